"""Workloads of the operators around an MXFP4 expert block, through the library's public entry points.

Five kinds of call: routing from softmax or sigmoid scores with groups and a balance bias, the residual norm
between two blocks, quantisation to microscaled 4-bit floats and back, the grouped product of quantised tokens with
quantised experts, and the product of a few unquantised tokens with quantised experts.  With `own` false, `run`
computes them with elementary torch operations.

Microscaled arrays stand for [rows, K] numbers as two uint8 tensors: codes [rows, K / 2] (two e2m1 codes a byte, the
even column in the low nibble) and scales [rows, K / 32] (one e8m0 exponent per 32 columns).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token of a step: 256 experts in 8 groups, sigmoid scores with a balance bias
        dict(name="route-1-sigmoid-groups", kind="route", T=1, E=256, k=8, score="sigmoid", n_group=8, topk_group=4, group_score="top2", bias=True,
             norm=True, scale=2.5, masked=0.0, ties=False),
        # a prompt through a softmax router without groups, a few experts masked out, logits that a bf16 router left with ties
        dict(name="route-2047-softmax", kind="route", T=2047, E=60, k=4, score="softmax", n_group=1, topk_group=1, group_score="max", bias=False,
             norm=False, scale=1.0, masked=0.05, ties=True),
        # a batch of long prompts, the widest router
        dict(name="route-16384-sigmoid-groups", kind="route", T=16384, E=256, k=8, score="sigmoid", n_group=8, topk_group=4, group_score="top2",
             bias=True, norm=True, scale=2.5, masked=0.0, ties=False),
        # one token between two layers: six slots joined by their gate weights, fp32 residual stream
        dict(name="norm-1", kind="norm", T=1, d=2048, k=6, act="bf16", res="f32", post=False, gate=None, scale=1.0),
        # a prompt between two layers: four slots, norm after the block, a gate per channel
        dict(name="norm-4096", kind="norm", T=4096, d=2048, k=4, act="bf16", res="bf16", post=True, gate="channel", scale=0.5),
        # activations of an odd-sized prompt in fp32
        dict(name="quantize-173-f32", kind="quantize", rows=173, K=1408, act="f32"),
        # expert weights at load time
        dict(name="quantize-weights", kind="quantize", rows=8 * 2816, K=2048, act="bf16"),
        # a short odd-sized prompt through the gate/up product of a DeepSeek-V2-Lite-shaped layer
        dict(name="product-173-swiglu", kind="product", T=173, E=64, k=6, N=2816, K=2048, slots=False, swiglu=True, out="bf16", skew=0.0),
        # a prompt through the gate/up product of a Qwen1.5-MoE-shaped layer
        dict(name="product-2048-swiglu", kind="product", T=2048, E=60, k=4, N=2816, K=2048, slots=False, swiglu=True, out="bf16", skew=0.5),
        # a long prompt through the down product of a dense first layer
        dict(name="product-4096-dense", kind="product", T=4096, E=1, k=1, N=2048, K=10944, slots=False, swiglu=False, out="f32", skew=0.0),
        # one token through the gate/up product of a DeepSeek-V2-Lite-shaped layer
        dict(name="matvec-1-swiglu", kind="matvec", T=1, E=64, k=6, N=2816, K=2048, slots=False, swiglu=True, act="bf16"),
        # a decode batch of 16 through the routed down product, one row of intermediates for every slot
        dict(name="matvec-16-slots", kind="matvec", T=16, E=64, k=6, N=2048, K=1408, slots=True, swiglu=False, act="f32"),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choice(["route", "norm", "quantize", "product", "product", "matvec"])
    act = rng.choice(["bf16", "bf16", "f32"])
    if kind == "route":
        n_group = rng.choice([1, 1, 2, 4, 8])
        size = log(4, 256 // n_group)
        topk_group = rng.randint(1, n_group)
        return dict(kind=kind, T=log(1, 16384), E=n_group * size, k=rng.randint(1, min(16, topk_group * size)), score=rng.choice(["softmax", "sigmoid"]),
                    n_group=n_group, topk_group=topk_group, group_score=rng.choice(["max", "top2"]), bias=rng.random() < 0.6, norm=rng.random() < 0.5,
                    scale=rng.choice([1.0, 2.5]), masked=rng.choice([0.0, 0.0, 0.05]), ties=rng.random() < 0.3)
    if kind == "norm":
        return dict(kind=kind, T=log(1, 2500), d=32 * log(4, 64), k=rng.randint(1, 6), act=act, res=rng.choice(["bf16", "f32"]), post=rng.random() < 0.5,
                    gate=rng.choice([None, "channel", "token"]), scale=rng.choice([1.0, 0.5]))
    if kind == "quantize":
        return dict(kind=kind, rows=log(1, 8192), K=32 * log(1, 128), act=act)
    N, K, swiglu = 32 * log(4, 100), 32 * log(4, 100), rng.random() < 0.5
    E = rng.choice([1, log(4, 96)])
    k = 1 if E == 1 else rng.randint(1, min(8, E))
    slots = k > 1 and rng.random() < 0.4
    if kind == "matvec":
        return dict(kind=kind, T=log(1, 16), E=E, k=k, N=N, K=K, slots=slots, swiglu=swiglu, act=act)
    return dict(kind=kind, T=log(1, 1024), E=E, k=k, N=N, K=K, slots=slots, swiglu=swiglu, out=rng.choice(["bf16", "bf16", "f32"]),
                skew=rng.choice([0.0, 0.0, 0.5]))


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + tag * 7919 + 29) & 0x7FFFFFFF)
    return g


def _rand(seed, tag, *shape):
    return torch.randn(shape, generator=_gen(seed, tag), device=DEV)


def _hidden(seed, tag, *shape):
    """Hidden states: unit normal, one channel in 256 ten times as large."""
    x = _rand(seed, tag, *shape)
    x[..., torch.randperm(shape[-1], generator=_gen(seed, tag + 50), device=DEV)[: max(1, shape[-1] // 256)]] *= 10.0
    return x


def _inputs(c, seed):
    s = {"case": c}
    if c["kind"] == "route":
        z = _rand(seed, 1, c["T"], c["E"])
        if c["ties"]:
            z = z.bfloat16().float()
        if c["masked"]:
            z[torch.rand(z.shape, generator=_gen(seed, 2), device=DEV) < c["masked"]] = -math.inf
        s["logits"] = z
        s["bias"] = _rand(seed, 3, c["E"]) * 0.05 if c["bias"] else None
    elif c["kind"] == "norm":
        T, d, act = c["T"], c["d"], DT[c["act"]]
        s["y"] = _hidden(seed, 1, T, c["k"], d).to(act)
        s["slot_w"] = torch.rand((T, c["k"]), generator=_gen(seed, 2), device=DEV) * (2.0 / c["k"])
        s["res"] = (_hidden(seed, 3, T, d) * 3.0).to(DT[c["res"]])
        s["pre"] = (1.0 + 0.1 * _rand(seed, 4, d)).to(act)
        s["post"] = (1.0 + 0.1 * _rand(seed, 5, d)).to(act) if c["post"] else None
        s["gate"] = None if c["gate"] is None else (0.5 + 0.2 * (_rand(seed, 6, d) if c["gate"] == "channel" else _rand(seed, 6, T, d))).to(act)
    elif c["kind"] == "quantize":
        s["x"] = (_hidden(seed, 1, c["rows"], c["K"]) * 0.02).to(DT[c["act"]])
    else:
        T, E, k, N, K = (c[n] for n in ("T", "E", "k", "N", "K"))
        s["w_codes"], s["w_scales"] = _quantize(_rand(seed, 1, E, N, K) * 0.02)
        s["x"] = _hidden(seed, 2, *((T, k, K) if c["slots"] else (T, K))).to(DT[c["act"]] if c["kind"] == "matvec" else torch.bfloat16)
        # distinct experts for a token, as a router's top-k gives them; skew: popular experts
        pop = _rand(seed, 3, E) * c.get("skew", 0.0)
        s["idx"] = (_rand(seed, 4, T, E) + pop).topk(k, dim=1).indices.to(torch.int32) if E > 1 else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2512_12990_amd import binding as B
        s["ctx"] = B.Ctx(0, workspace_bytes=0)
    return s


# --------------------------------------------------------------------------------------- one pass
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2512_12990_amd import binding as B
    c, ctx = s["case"], s["ctx"]
    if c["kind"] == "route":
        idx, w = B.smoe_route_scores(ctx, c["k"], logits=s["logits"], score=c["score"], n_group=c["n_group"], topk_group=c["topk_group"],
                                     group_score=c["group_score"], bias=s["bias"], norm_topk=c["norm"], routed_scale=c["scale"])
        return {"idx": idx, "w": w}
    if c["kind"] == "norm":
        res, x = B.smoe_residual_norm(ctx, s["res"], y=s["y"], slot_w=s["slot_w"], post_w=s["post"], gate=s["gate"], scale=c["scale"], pre_w=s["pre"],
                                      eps=1e-6)
        return {"res": res, "x": x}
    if c["kind"] == "quantize":
        return {"x": B.smoe_mx_dequantize(ctx, B.smoe_mx_quantize(ctx, s["x"]))}
    w = B.Mx(s["w_codes"], s["w_scales"])
    if c["kind"] == "matvec":
        return {"y": B.smoe_mx_matvec(ctx, w, s["x"], idx=s["idx"], swiglu=c["swiglu"])}
    return {"y": B.smoe_mx_product(ctx, w, B.smoe_mx_quantize(ctx, s["x"]), idx=s["idx"], swiglu=c["swiglu"], out_dtype=DT[c["out"]])}


def _quantize(x):
    """(codes, scales): exponent of a block = exponent of its largest magnitude - 2, values to the nearest of 0 .5 1 1.5 2 3 4 6, ties to the even code."""
    v = x.float().reshape(*x.shape[:-1], -1, 32)
    _, e = torch.frexp(v.abs().amax(-1))                       # largest = mantissa in [1/2, 1) * 2^e
    big = v.abs().amax(-1)
    X = torch.where(big > 0, (e - 3).clamp(-127, 127), torch.full_like(e, -127))
    inv = ((127 - X) << 23).to(torch.int32).view(torch.float32)            # 2^-X
    m = (v * inv[..., None]).abs()
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)).to(torch.uint8)
    code = code + (torch.signbit(v).to(torch.uint8) << 3)
    code = code.reshape(*x.shape[:-1], -1, 2)
    return code[..., 0] | (code[..., 1] << 4), (X + 127).to(torch.uint8)


def _values(codes, scales):
    """fp32 values that microscaled codes stand for."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    v = table[torch.stack([codes & 15, codes >> 4], -1).long()].reshape(*scales.shape, 32)
    scale = torch.where(scales > 0, (scales.to(torch.int32) << 23), torch.full_like(scales, 1 << 6, dtype=torch.int32) << 16).view(torch.float32)
    return (v * scale[..., None]).reshape(*codes.shape[:-1], -1)


def _swiglu(y):
    g, u = y[..., 0::2], y[..., 1::2]
    return g / (1.0 + torch.exp(-g)) * u


def _plain(s):
    c = s["case"]
    if c["kind"] == "route":
        return _plain_route(c, s["logits"].double(), s["bias"])
    if c["kind"] == "norm":
        b = (s["y"].float() * s["slot_w"][..., None]).sum(1)
        if s["post"] is not None:
            b = b * torch.rsqrt(b.square().mean(-1, keepdim=True) + 1e-6) * s["post"].float()
        if s["gate"] is not None:
            b = b * s["gate"].float()
        h = s["res"].float() + c["scale"] * b
        x = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6) * s["pre"].float()
        return {"res": h.to(s["res"].dtype), "x": x.to(s["y"].dtype)}
    if c["kind"] == "quantize":
        return {"x": _values(*_quantize(s["x"]))}
    x = s["x"].float() if c["kind"] == "matvec" else _values(*_quantize(s["x"]))
    idx, T, k = s["idx"], c["T"], c["k"]
    if idx is None:
        y = (x.reshape(T, -1) @ _values(s["w_codes"], s["w_scales"])[0].t())[:, None]
    elif T * k <= 96:
        # few rows: the selected experts' matrices, one for each row
        w = _values(s["w_codes"][idx.long()], s["w_scales"][idx.long()])
        x = x if c["slots"] else x[:, None].expand(T, k, -1)
        y = torch.matmul(w, x[..., None].contiguous())[..., 0]
    else:
        # rows sorted by expert, every expert's padded to the largest number of rows
        flat = idx.reshape(-1).long()
        order = torch.argsort(flat, stable=True)
        count = torch.bincount(flat, minlength=c["E"])
        cap = int(count.max())
        first = torch.cumsum(count, 0) - count
        at = flat[order] * cap + torch.arange(T * k, device=DEV) - first[flat[order]]
        rows = x.reshape(-1, c["K"])[order if c["slots"] else order // k]
        padded = torch.zeros((c["E"] * cap, c["K"]), device=DEV).index_copy_(0, at, rows).reshape(c["E"], cap, -1)
        out = torch.bmm(padded, _values(s["w_codes"], s["w_scales"]).transpose(1, 2).contiguous()).reshape(c["E"] * cap, -1)
        y = torch.empty((T * k, c["N"]), device=DEV).index_copy_(0, order, out[at]).reshape(T, k, -1)
    y = _swiglu(y) if c["swiglu"] else y
    return {"y": y.to(DT[c["out"] if c["kind"] == "product" else c["act"]])}


def _plain_route(c, z, bias):
    T, E, g = c["T"], c["E"], c["n_group"]
    if c["score"] == "sigmoid":
        p = 1.0 / (1.0 + torch.exp(-z))
    else:
        # a row without any finite logit has no scores
        p = torch.where(z > -math.inf, torch.exp(z - z.amax(-1, keepdim=True)), 0.0)
        p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
    sel = p if bias is None else p + bias.double()
    # stable descending sorts: equal values keep the order of their indices
    if g > 1:
        best = sel.reshape(T, g, -1).sort(dim=-1, descending=True, stable=True).values
        score = best[..., 0] + (best[..., 1] if c["group_score"] == "top2" and E // g > 1 else 0.0)
        rank = score.sort(dim=-1, descending=True, stable=True).indices.argsort(-1)
        sel = sel.masked_fill((rank >= c["topk_group"]).repeat_interleave(E // g, -1), -math.inf)
    idx = sel.sort(dim=-1, descending=True, stable=True).indices[:, : c["k"]]
    w = p.gather(1, idx)
    if c["norm"]:
        total = w.sum(-1, keepdim=True)
        w = torch.where(total > 0, w / total, torch.zeros_like(w))
    return {"idx": idx.to(torch.int32), "w": (w * c["scale"]).float()}


# -------------------------------------------------------------------------------- in 64 bits, apart
def _grid64(x):
    """What quantisation leaves of x, in 64 bits: the step of a magnitude in [1, 6] is half its power of two, below 1 it is 1/2."""
    v = x.double().reshape(-1, 32)
    X = torch.floor(torch.log2(v.abs().amax(-1, keepdim=True)))
    big = v.abs().amax(-1, keepdim=True)
    X = X + (torch.exp2(X + 1) <= big).double() - (torch.exp2(X) > big).double()           # log2 rounds next to a power of two
    unit = torch.exp2((X - 2).clamp(-127, 127))
    m = v.abs() / unit
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0).double())
    q = torch.sign(v) * (torch.round(m / step) * step).clamp(max=6.0) * unit
    return torch.where(big > 0, q, torch.zeros_like(q)).reshape(x.shape)


def _weights64(codes, scales):
    """sign, exponent and mantissa of every e2m1 code taken apart."""
    n = torch.stack([codes & 15, codes >> 4], -1).reshape(*scales.shape, 32).double()
    sign, n = 1.0 - 2.0 * torch.floor(n / 8), torch.remainder(n, 8)
    e, m = torch.floor(n / 2), torch.remainder(n, 2)
    v = torch.where(e > 0, torch.exp2(e - 1) * (1 + m / 2), m / 2) * sign
    return (v * torch.exp2(scales.double() - 127)[..., None]).reshape(*codes.shape[:-1], -1)


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "route":
        z = s["logits"].double()
        p = torch.sigmoid(z) if c["score"] == "sigmoid" else torch.nan_to_num(torch.softmax(z, -1))
        sel = (p if s["bias"] is None else p + s["bias"].double()).cpu().tolist()
        w = torch.zeros((c["T"], c["k"]), dtype=torch.float64)
        p, size = p.cpu(), c["E"] // c["n_group"]
        for t in range(c["T"]):
            groups = []
            for g in range(c["n_group"]):
                top = sorted(sel[t][g * size:(g + 1) * size], reverse=True)
                groups.append((-(top[0] if c["group_score"] == "max" else sum(top[:2])), g))
            allowed = {g for _, g in sorted(groups)[: c["topk_group"]]} if c["n_group"] > 1 else {0}
            chosen = sorted((-sel[t][e], e) for e in range(c["E"]) if e // size in allowed)[: c["k"]]
            row = p[t, [e for _, e in chosen]]
            w[t] = row / (row.sum() if c["norm"] and row.sum() > 0 else 1.0) * c["scale"]
        return {"idx": None, "w": w}
    if c["kind"] == "norm":
        b = sum(s["y"][:, j].double() * s["slot_w"][:, j, None].double() for j in range(c["k"]))
        rms = lambda v: v / torch.sqrt((v * v).sum(-1, keepdim=True) / c["d"] + 1e-6)
        b = rms(b) * s["post"].double() if c["post"] else b
        h = s["res"].double() + c["scale"] * (b if c["gate"] is None else b * s["gate"].double())
        return {"res": h, "x": rms(h) * s["pre"].double()}
    if c["kind"] == "quantize":
        return {"x": _grid64(s["x"])}
    T, k, N = c["T"], c["k"], c["N"]
    x = (s["x"].double() if c["kind"] == "matvec" else _grid64(s["x"])).reshape(T, -1, c["K"])
    y = torch.empty((T, k, N), dtype=torch.float64, device=DEV)
    for e in range(c["E"]):
        at = (s["idx"] == e).nonzero(as_tuple=True) if s["idx"] is not None else (torch.arange(T, device=DEV), torch.zeros(T, dtype=torch.long, device=DEV))
        if len(at[0]):
            w = _weights64(s["w_codes"][e], s["w_scales"][e])
            y[at] = torch.mm(x[at[0], at[1] if c["slots"] else torch.zeros_like(at[1])], w.t())
    return {"y": y[..., 0::2] * torch.sigmoid(y[..., 0::2]) * y[..., 1::2] if c["swiglu"] else y}


# ------------------------------------------------------------------------------ unavoidable work
def work(c):
    size = {"f32": 4, "bf16": 2}
    if c["kind"] == "route":
        return {"bytes": c["T"] * (4 * c["E"] + 8 * c["k"]) + (4 * c["E"] if c["bias"] else 0), "flops": c["T"] * c["E"] * 4}
    if c["kind"] == "norm":
        a, r, n = size[c["act"]], size[c["res"]], c["T"] * c["d"]
        vectors = 1 + c["post"] + (c["gate"] == "channel") + (c["T"] if c["gate"] == "token" else 0)
        return {"bytes": n * (c["k"] * a + 2 * r + a) + vectors * c["d"] * a + 4 * c["T"] * c["k"], "flops": n * (2 * c["k"] + 8)}
    if c["kind"] == "quantize":
        # there and back: the source read, codes and scales written and read, fp32 written
        return {"bytes": c["rows"] * c["K"] * (size[c["act"]] + 2 * 17 / 32 + 4), "flops": c["rows"] * c["K"] * 4}
    T, E, k, N, K = (c[n] for n in ("T", "E", "k", "N", "K"))
    rows = T * k
    used = E * (1.0 - (1.0 - k / E) ** T)                                # experts that a uniform routing reaches
    out = rows * (N // 2 if c["swiglu"] else N) * size[c["out"] if c["kind"] == "product" else c["act"]]
    x = (rows if c["slots"] else T) * K * (2 if c["kind"] == "product" else size[c["act"]])
    return {"bytes": used * N * K * 17 / 32 + x + out + 4 * rows, "flops": 2.0 * rows * N * K}
