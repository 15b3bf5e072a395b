"""Score routing, residual norm and microscaled floats on the GPU against their definition in 64 bits."""
import itertools

import numpy as np
import pytest
import torch

from oracle import block_oracle as O
from paper_2512_12990_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U32 = 2.0 ** -24                       # half a step of fp32, relative
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx():
    c = B.Ctx(0, workspace_bytes=0)
    yield c
    c.close()


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def np64(t):
    return t.detach().cpu().double().numpy()


def close(got, want, tol):
    """|got - want| <= tol everywhere, NaN where the definition has NaN."""
    got = np64(got)
    assert got.shape == want.shape
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    bad = ~(np.abs(got - want) <= tol) & ~nan
    assert not bad.any(), "%d of %d off, worst %.3g times the tolerance" % (bad.sum(), bad.size, np.max(np.where(bad, np.abs(got - want) / tol, 0)))


# ------------------------------------------------------------------------------------------ routing
def check_route(ctx, z, k, **kw):
    bias = kw.get("bias")
    idx, w = B.smoe_route_scores(ctx, k, logits=dev(z), score=kw.get("score", "softmax"), n_group=kw.get("ng", 1), topk_group=kw.get("tg", 1),
                                 group_score=kw.get("gs", "max"), bias=None if bias is None else dev(bias), norm_topk=kw.get("norm", False),
                                 routed_scale=kw.get("scale", 1.0))
    ri, rw = O.route_scores(z, k, kw.get("score", "softmax"), kw.get("ng", 1), kw.get("tg", 1), kw.get("gs", "max"), bias, kw.get("norm", False),
                            kw.get("scale", 1.0))
    got = idx.cpu().numpy()
    if not np.array_equal(got, ri):
        # Each binary64 score carries the exponential's last bit, a sum's and a quotient's: 1 + 1/2 + 1/2 units of 2^-53 relative to a score of at most 1,
        # and half a unit of the sum with the bias.  Two exact values nearer than 2^-51 may come out in either order, or equal.
        s = O.scores(z, kw.get("score", "softmax")) + (0.0 if bias is None else bias.astype(np.float64))
        assert (np.sort(got, 1)[:, 1:] > np.sort(got, 1)[:, :-1]).all()
        assert np.abs(np.take_along_axis(s, got.astype(np.int64), 1) - np.take_along_axis(s, ri, 1)).max() <= 2.0 ** -51
    close(w, rw, np.abs(rw) * 2 * U32 + 1e-45)             # one rounding from 64 bits, and a subnormal's step


@pytest.mark.parametrize("score, bias, norm", itertools.product(["softmax", "sigmoid"], [False, True], [False, True]))
@pytest.mark.parametrize("T, E, k, ng, tg, gs", [
    (1, 1, 1, 1, 1, "max"), (1, 256, 8, 8, 4, "top2"), (3, 64, 6, 1, 1, "max"), (130, 60, 4, 1, 1, "max"), (37, 160, 6, 8, 3, "max"), (5, 256, 16, 64, 4, "top2"),
    (9, 65, 16, 5, 2, "top2"), (17, 63, 3, 63, 3, "top2"), (70, 200, 7, 2, 1, "top2"), (4, 16, 16, 4, 4, "max"),
])
def test_route_scores(ctx, T, E, k, ng, tg, gs, score, bias, norm):
    rng = np.random.default_rng(T * 1000 + E)
    z = rng.standard_normal((T, E)).astype(np.float32) * 2
    b = (rng.standard_normal(E) * 0.1).astype(np.float32) if bias else None
    check_route(ctx, z, k, score=score, bias=b, norm=norm, ng=ng, tg=tg, gs=gs, scale=2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("ng, tg", [(1, 1), (8, 3)])
def test_route_scores_ties_masks_and_nan(ctx, score, ng, tg):
    rng = np.random.default_rng(5)
    E, k = 128, 6
    z = np.round(rng.standard_normal((24, E)) * 2).astype(np.float32) / 2             # many equal scores
    z[0] = 0.0
    z[1] = -np.inf                                                                    # nothing left
    z[2] = -np.inf
    z[2, 77] = 1.0
    z[3, 5], z[3, 9] = np.inf, np.inf
    z[4] = np.finfo(np.float32).min                                                   # a mask of the type's lowest value
    z[5, ::2] = np.finfo(np.float32).min
    z[6] = 1e30
    z[7] = -0.0
    z[7, ::3] = 0.0
    z[8, 11] = np.nan
    z[9] = np.nan
    z[10] = 1e-40
    for norm in (False, True):
        check_route(ctx, z, k, score=score, ng=ng, tg=tg, gs="top2", norm=norm)
    check_route(ctx, z[:8], k, score=score, ng=ng, tg=tg, gs="top2", bias=np.round(rng.standard_normal(E)).astype(np.float32), norm=True)
    b = np.zeros(E, np.float32)
    b[: E // 2] = -np.inf
    check_route(ctx, z[10:], k, score=score, ng=ng, tg=tg, gs="max", bias=b)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E, ng, tg, gs, k", [(256, 8, 4, "top2", 8), (64, 1, 1, "max", 6), (128, 4, 2, "max", 5), (64, 64, 7, "max", 7), (256, 2, 1, "top2", 16), (40, 1, 1, "max", 3),
                                              (256, 64, 9, "max", 8), (32, 4, 3, "top2", 8)])
def test_route_scores_close_decisions(ctx, E, ng, tg, gs, k, score):
    """Keys a few units in the last place apart, equal ones, saturated ones: the order is that of the binary64 scores."""
    rng = np.random.default_rng(E + ng)
    z = np.empty((2100, E), np.float32)                                              # (from 2049 tokens on fp32 keys decide where they can)
    z[600:] = rng.standard_normal((1500, E)) * 2
    z[:200] = rng.standard_normal((200, E)) * 2
    z[200:300] = 1.0 + rng.integers(-2, 3, size=(100, E)) * 2.0 ** -23               # neighbours in fp32
    z[300:340] = rng.standard_normal((40, E)) * 1e-12                                 # apart in fp32, scores equal to 1e-12
    z[340:400] = 12 + rng.random((60, E)) * 30                                        # sigmoids next to 1 and equal to it
    z[400:450] = -70 + rng.random((50, E))
    z[450:500] = np.round(rng.standard_normal((50, E)) * 4) / 4
    z[500:550] = rng.standard_normal((50, E))
    z[500:550][rng.random((50, E)) < 0.4] = -np.inf
    z[550:600] = rng.standard_normal((50, E)) * 1000
    b = (rng.standard_normal(E) * 0.05).astype(np.float32)
    near = b.copy()
    near[1::2] = near[::2] + np.float32(1e-8)                                         # pairs that a bias sets apart by less than fp32 holds next to 1
    wide = (rng.standard_normal(E) * 30).astype(np.float32)
    for bias, norm in ((None, False), (None, True), (b, True), (near, False), (wide, False)):
        check_route(ctx, z, k, score=score, ng=ng, tg=tg, gs=gs, bias=bias, norm=norm)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("T, E, d", [(1, 64, 256), (300, 64, 96), (600, 200, 2048), (1200, 16, 520), (5, 8, 13000), (1100, 30, 8192)])
def test_route_scores_from_activations(ctx, T, E, d, act):
    """The mat-vec's logits are smoe_route's, bit for bit; the choice is that of these logits."""
    g = torch.Generator().manual_seed(T + E)
    x = torch.randn((T, d), generator=g).to(DT[act]).cuda()
    wr = (torch.randn((E, d), generator=g) * 0.05).cuda()
    k = min(6, E)
    kw = dict(score="sigmoid", norm_topk=True)
    idx, w = B.smoe_route_scores(ctx, k, x=x, w_router=wr, **kw)
    if d < 8000:
        z = B.smoe_route(ctx, k, x=x, w_router=wr, want_logits=True)[2]
        i2, w2 = B.smoe_route_scores(ctx, k, logits=z, **kw)
        assert torch.equal(idx, i2) and torch.equal(w, w2)
    # sums of d products in fp32 are off by at most d * 2^-24 * sum |w x|; the chosen set may differ only among scores that near
    z64 = np64(x) @ np64(wr).T
    off = d * U32 * (np.abs(np64(x)) @ np.abs(np64(wr)).T).max()
    best = -np.sort(-z64, axis=1)[:, :k]
    got = np.take_along_axis(z64, idx.cpu().numpy().astype(np.int64), 1)
    assert np.abs(got - best).max() <= 2 * off


@pytest.mark.parametrize("E, d, act", [(64, 2048, "bf16"), (256, 520, "f32"), (7, 96, "bf16")])
def test_route_scores_one_token_with_a_workspace(ctx, E, d, act):
    """The mat-vec spread over the device, logits in the workspace: the bits of the call without one."""
    g = torch.Generator().manual_seed(E)
    c = B.Ctx(0)
    for _ in range(3):
        x, wr = torch.randn((1, d), generator=g).to(DT[act]).cuda(), (torch.randn((E, d), generator=g) * 0.05).cuda()
        a = B.smoe_route_scores(c, 3, x=x, w_router=wr, score="sigmoid", norm_topk=True)
        b = B.smoe_route_scores(ctx, 3, x=x, w_router=wr, score="sigmoid", norm_topk=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c.close()


# ------------------------------------------------------------------------------------ residual norm
def check_norm(ctx, T, d, k, act="bf16", res="f32", post=False, gate=None, pre=True, slot_w=True, scale=1.0, eps=1e-6, with_res=True, with_y=True, x=True,
               in_place=False, data=None, seed=0):
    g = torch.Generator().manual_seed(seed + T * 131 + d)
    r = lambda *s: torch.randn(s, generator=g)
    t = dict(res=(r(T, d) * 3).to(DT[res]) if with_res else None, y=r(T, k, d).to(DT[act]) if with_y else None,
             slot_w=torch.rand((T, k), generator=g) if slot_w and with_y else None, post_w=(1 + 0.1 * r(d)).to(DT[act]) if post else None,
             gate=None if gate is None else r(*((d,) if gate == "channel" else (T, d))).to(DT[act]), pre_w=(1 + 0.1 * r(d)).to(DT[act]) if pre else None)
    if data is not None:
        data(t)
    n = {a: None if v is None else np64(v) for a, v in t.items()}
    h, xo = O.residual_norm(n["res"], n["y"], n["slot_w"], n["post_w"], n["gate"], scale, n["pre_w"], eps)
    c = {a: None if v is None else v.cuda() for a, v in t.items()}
    out = c["res"] if in_place else None
    got_h, got_x = B.smoe_residual_norm(ctx, c.pop("res"), scale=scale, eps=eps, res_out=out, want_x=x, act_dtype=DT[act], **c)
    assert got_h.dtype == DT[res if with_res else act] and (not in_place or got_h is out)
    # Sums of squares: a thread adds at most 32 of them, then 6 steps over the wave and 16 over the work-group: 54 roundings, halved by the root; the mean,
    # eps, root and division 4 more: a norm's factor is off by 32 units.  b: k + 1 roundings of the largest partial sum; post norm, gate, scale: 5.
    a = 0.0
    if n["y"] is not None:
        a = (np.abs(n["y"]) * (1 if n["slot_w"] is None else np.abs(n["slot_w"])[..., None])).sum(1) * (k + 1) * U32
        if n["post_w"] is not None:
            b = (n["y"] * (1 if n["slot_w"] is None else n["slot_w"][..., None])).sum(1)
            f = 1 / np.sqrt((b * b).mean(-1, keepdims=True) + eps)
            # error of b, and of its norm: |d f / f| <= |d b| |b| / mean b^2 (Cauchy-Schwarz: rms of the errors over rms of b)
            rel = np.sqrt((a * a).mean(-1, keepdims=True)) * f + 32 * U32
            a = (a * f + np.abs(b) * f * rel) * np.abs(n["post_w"])
            a = a + np.abs(b * f * n["post_w"]) * 3 * U32
        step = 1.0 if n["gate"] is None else np.abs(n["gate"])
        a = a * step * abs(scale) + np.abs(h - (0 if n["res"] is None else n["res"])) * 3 * U32
    a = a + np.abs(h) * U32
    close(got_h, h, a + np.abs(h) * HALF[res if with_res else act] * 1.01 + 1e-37)
    if x:
        f = 1 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
        rel = np.sqrt((a * a).mean(-1, keepdims=True)) * f + 32 * U32
        p = 1.0 if n["pre_w"] is None else np.abs(n["pre_w"])
        close(got_x, xo, (a * f + np.abs(h) * f * rel) * p * 1.01 + np.abs(xo) * (HALF[act] + 2 * U32) * 1.01 + 1e-37)
    else:
        assert got_x is None


@pytest.mark.parametrize("act, res", itertools.product(["f32", "bf16"], ["f32", "bf16"]))
@pytest.mark.parametrize("T, d, k", [(1, 2048, 6), (5, 8, 1), (7, 504, 3), (6, 512, 2), (3, 520, 1), (2, 2056, 5), (4, 4096, 2), (3, 4104, 24), (2, 8192, 1), (2, 8200, 4), (1, 16384, 3),
                                     (301, 128, 2)])
def test_residual_norm(ctx, T, d, k, act, res):
    check_norm(ctx, T, d, k, act, res)
    check_norm(ctx, T, d, k, act, res, post=True, gate="channel", scale=0.5)


@pytest.mark.parametrize("kw", [
    dict(gate="token", scale=-2.0), dict(pre=False), dict(slot_w=False), dict(with_res=False), dict(with_y=False), dict(x=False), dict(in_place=True),
    dict(post=True, eps=0.0), dict(with_y=False, pre=False, in_place=True), dict(with_res=False, x=False, post=True),
])
@pytest.mark.parametrize("d", [64, 1408])
def test_residual_norm_options(ctx, kw, d):
    check_norm(ctx, 11, d, 0 if not kw.get("with_y", True) else 2, act="bf16", res="bf16" if not kw.get("with_res", True) else "f32", **kw)


def test_residual_norm_zero_rows_and_large_values(ctx):
    def zero(t):
        t["y"][1] = 0
        t["res"][1] = 0
        t["slot_w"][2] = 0                                   # a token that no slot serves
        t["res"][3] *= 1e15
    check_norm(ctx, 6, 512, 3, post=True, data=zero)
    def nan(t):
        t["y"][2, 1, 7] = float("nan")
    check_norm(ctx, 6, 2048, 3, data=nan)
    h, x = B.smoe_residual_norm(ctx, torch.zeros((0, 64), device="cuda"), y=torch.zeros((0, 2, 64), device="cuda"))
    assert h.shape == (0, 64) and x.shape == (0, 64)


# ---------------------------------------------------------------------------------- quantise and back
@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 32), (3, 64), (173, 1408), (2, 5, 96), (1031, 2048), (7, 8192)])
def test_mx_quantize_and_back(ctx, shape, act):
    g = torch.Generator().manual_seed(shape[-1])
    x = torch.randn(shape, generator=g) * torch.exp2(torch.randint(-20, 20, shape[:-1] + (1,), generator=g).float())
    x = x.to(DT[act])
    m = B.smoe_mx_quantize(ctx, x.cuda())
    codes, scales = O.mx_quantize(np64(x))
    assert np.array_equal(m.scales.cpu().numpy(), scales) and np.array_equal(m.codes.cpu().numpy(), codes)
    for out in ("f32", "bf16"):                              # e2m1 times a power of two: exact in both
        assert np.array_equal(np64(B.smoe_mx_dequantize(ctx, m, DT[out])), O.mx_values(codes, scales))
    into = B.Mx(torch.full_like(m.codes, 77), torch.full_like(m.scales, 77))
    assert B.smoe_mx_quantize(ctx, x.cuda(), out=into) is into
    assert torch.equal(into.codes, m.codes) and torch.equal(into.scales, m.scales)


def test_mx_quantize_borders(ctx):
    """Every border of the grid with its two neighbours, at every exponent of fp32, subnormal blocks, zeros, infinities and NaN."""
    half = np.array([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7], np.float64)
    rows = []
    for e in range(-149, 126):
        v = np.concatenate([half, -half]) * 2.0 ** e
        v = np.minimum(v, 3.4e38).astype(np.float32)
        rows += [v, np.nextafter(v, np.float32(0)), np.nextafter(v, np.float32(3.4e38))]
    x = np.stack(rows)
    for bad in (np.nan, -np.nan, np.inf, -np.inf):
        row = x[300].copy()
        row[13] = bad
        x = np.concatenate([x, row[None]])
    x = np.concatenate([x, np.zeros((1, 32), np.float32), -np.zeros((1, 32), np.float32)])
    m = B.smoe_mx_quantize(ctx, dev(x))
    codes, scales = O.mx_quantize(x)
    assert np.array_equal(m.scales.cpu().numpy(), scales)
    assert np.array_equal(m.codes.cpu().numpy(), codes)
    got, want = np64(B.smoe_mx_dequantize(ctx, m)), O.mx_values(codes, scales)
    assert np.array_equal(got, want, equal_nan=True)


def test_mx_dequantize_every_code_and_scale(ctx):
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(1, 16, 16), (256, 1, 1)).reshape(256, 256)
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, 1)
    want = O.mx_values(codes, scales)
    got = np64(B.smoe_mx_dequantize(ctx, B.Mx(dev(codes), dev(scales))))
    with np.errstate(over="ignore"):
        assert np.array_equal(got, want.astype(np.float32).astype(np.float64), equal_nan=True)


def test_mx_empty(ctx):
    m = B.smoe_mx_quantize(ctx, torch.zeros((0, 64), device="cuda"))
    assert m.codes.shape == (0, 32) and B.smoe_mx_dequantize(ctx, m).shape == (0, 64)


# ----------------------------------------------------------------------------------------- products
def mx_random(rng, *shape, spread=1):
    """Codes and scales whose products with each other add up without rounding: multiples of 2^-2 times small powers of two."""
    codes = rng.integers(0, 256, size=shape[:-1] + (shape[-1] // 2,)).astype(np.uint8)
    scales = rng.integers(127 - spread, 128 + spread, size=shape[:-1] + (shape[-1] // 32,)).astype(np.uint8)
    return codes, scales


def experts(rng, T, k, E, how):
    if E == 1:
        return np.zeros((T, k), np.int32)
    if how == "one":
        return np.full((T, k), E - 1, np.int32)
    if how == "outside":
        return rng.integers(-3, E + 3, size=(T, k)).astype(np.int32)
    return np.stack([rng.choice(E, size=k, replace=k > E) for _ in range(T)]).astype(np.int32)


PRODUCTS = [  # T, k, E, N, K
    (1, 1, 1, 16, 32), (1, 6, 64, 64, 256), (3, 2, 5, 48, 96), (33, 1, 1, 272, 128), (64, 4, 7, 256, 64), (65, 2, 3, 96, 1408), (129, 1, 1, 528, 544),
    (200, 6, 40, 128, 320), (257, 2, 2, 80, 2048), (500, 3, 9, 512, 160), (1025, 1, 1, 64, 288),
]


@pytest.mark.parametrize("T, k, E, N, K", PRODUCTS)
@pytest.mark.parametrize("how, slots", [("any", False), ("any", True), ("one", False), ("outside", True)])
def test_mx_product_exact(ctx, T, k, E, N, K, how, slots):
    """Sums that fp32 holds without rounding: the product has to be exact, whatever the order of the sum."""
    rng = np.random.default_rng(T * 7 + N + K)
    w, x = mx_random(rng, E, N, K), mx_random(rng, *((T, k, K) if slots else (T, K)))
    idx = experts(rng, T, k, E, how)
    plain = E == 1 and k == 1 and how == "any"
    want = O.product(O.mx_values(*w), O.mx_values(*x), idx, False)
    assert K * 36 * 4 < 2 ** 24 / 16                           # multiples of 2^-4 below 2^20
    W, X = B.Mx(*map(dev, w)), B.Mx(*map(dev, x))
    i = None if plain and not slots else dev(idx)
    assert np.array_equal(np64(B.smoe_mx_product(ctx, W, X, idx=i, out_dtype=torch.float32)), want)
    got = B.smoe_mx_product(ctx, W, X, idx=i)
    assert torch.equal(got.cpu(), torch.from_numpy(want).float().bfloat16())
    # the gate and up columns of the SwiGLU are the same sums; silu in fp32: exponential, sum, quotient, product, two units each
    want = O.product(O.mx_values(*w), O.mx_values(*x), idx, True)
    for out in ("f32", "bf16"):
        got = B.smoe_mx_product(ctx, W, X, idx=i, swiglu=True, out_dtype=DT[out])
        close(got, want, np.abs(want) * (8 * U32 + HALF[out]) + 1e-30)


@pytest.mark.parametrize("T, k, E, N, K, slots", [
    (1600, 1, 1, 2064, 544, False), (1590, 1, 1, 2048, 160, False), (4100, 1, 1, 2064, 288, False), (4097, 1, 1, 2048, 1280, False), (4096, 1, 1, 2064, 800, False),
    (1000, 2, 3, 1600, 256, True), (1700, 4, 9, 1040, 1056, False), (2000, 3, 5, 2064, 96, True), (3000, 2, 2, 1536, 2304, False),
    (5000, 4, 7, 48, 96, False), (4600, 2, 3, 2064, 160, True), (1024, 4, 250, 32, 64, False), (1025, 4, 250, 32, 64, False), (4096, 1, 2, 32, 64, False), (8192, 1, 3, 2048, 64, False),
])
def test_mx_product_larger_tiles(ctx, T, k, E, N, K, slots):
    """Enough rows for the tiles of 64 and of 128 slots; odd counts, and all lengths of a last stage (1 to 7 blocks, none); slots that work-groups find
    themselves (up to 4096 or 8192) and slots listed before."""
    rng = np.random.default_rng(T + K)
    w, x = mx_random(rng, E, N, K), mx_random(rng, *((T, k, K) if slots else (T, K)))
    idx = experts(rng, T, k, E, "any")
    want = O.product(O.mx_values(*w), O.mx_values(*x), idx, False)
    W, X, i = B.Mx(*map(dev, w)), B.Mx(*map(dev, x)), dev(idx) if E > 1 else None
    assert np.array_equal(np64(B.smoe_mx_product(ctx, W, X, idx=i, out_dtype=torch.float32)), want)
    assert torch.equal(B.smoe_mx_product(ctx, W, X, idx=i).cpu(), torch.from_numpy(want).float().bfloat16())
    want = O.silu(want[..., 0::2]) * want[..., 1::2]
    for out in ("f32", "bf16"):
        got = B.smoe_mx_product(ctx, W, X, idx=i, swiglu=True, out_dtype=DT[out])
        close(got, want, np.abs(want) * (8 * U32 + HALF[out]) + 1e-30)


@pytest.mark.parametrize("T, k, E, N, K", [(100, 4, 16, 160, 2048), (40, 1, 1, 64, 10944), (2, 2, 300 // 2, 32, 65536)])
def test_mx_product_of_quantised_numbers(ctx, T, k, E, N, K):
    rng = np.random.default_rng(K)
    w = O.mx_quantize(rng.standard_normal((E, N, K)).astype(np.float32) * 0.02) if E * N * K < 4e7 else mx_random(rng, E, N, K, spread=3)
    x = rng.standard_normal((T, K)).astype(np.float32)
    x[:, ::97] *= 30
    idx = experts(rng, T, k, E, "any")
    X = B.smoe_mx_quantize(ctx, dev(x))
    used, local = np.unique(idx, return_inverse=True)
    wv, xv = O.mx_values(w[0][used], w[1][used]), O.mx_values(*O.mx_quantize(x))
    local = local.reshape(idx.shape)
    want = O.product(wv, xv, local, False)
    # exact products, one rounding (up to a whole step) per addition, K of them one after the other at worst
    tol = O.product(np.abs(wv), np.abs(xv), local, False) * K * 2 * U32
    close(B.smoe_mx_product(ctx, B.Mx(*map(dev, w)), X, idx=dev(idx), out_dtype=torch.float32), want, tol)


def test_mx_product_scales(ctx):
    """Scales at both ends, NaN blocks, and blocks that do not exist behind an odd number of blocks."""
    rng = np.random.default_rng(3)
    N, K, T = 32, 96, 40
    w, x = mx_random(rng, 1, N, K), mx_random(rng, T, K)
    w[1][0, :, 0], x[1][:, 0] = 254, 1                       # 2^127 * 2^-126
    w[1][0, 1, 1], x[1][:, 1] = 0, 127 + 120                 # 2^-127 * 2^120
    w[1][0, 0, 1] = 127
    w[1][0, 2:, 1], x[1][3, 1] = 7, 127
    w[1][0, 5, 2] = 255
    x[1][7, 2] = 255
    wv, xv = O.mx_values(*w), O.mx_values(*x)
    want = O.product(wv, xv, None, False)
    tol = O.product(np.abs(wv), np.abs(xv), None, False) * K * 2 * U32
    got = B.smoe_mx_product(ctx, B.Mx(*map(dev, w)), B.Mx(*map(dev, x)), out_dtype=torch.float32)
    assert np.isnan(want[:, 0, 5]).all() and np.isnan(want[7]).all()
    with np.errstate(over="ignore"):
        big = np.abs(want) > 3e38
    want[big], tol[big] = 0, 1
    close(torch.where(dev(big), torch.zeros_like(got), got), want, np.where(np.isnan(tol), 0, tol))


def test_mx_product_buffers_and_scratch(ctx):
    rng = np.random.default_rng(9)
    w, x = mx_random(rng, 6, 64, 128), mx_random(rng, 2100, 128)
    idx = experts(rng, 2100, 3, 6, "any")
    W, X, i = B.Mx(*map(dev, w)), B.Mx(*map(dev, x)), dev(idx)
    want = B.smoe_mx_product(ctx, W, X, idx=i)
    scratch = torch.full((B.smoe_mx_product_bytes(2100, 3, 6, 64),), 255, dtype=torch.uint8, device="cuda")
    wide = torch.full((2102, 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    got = B.smoe_mx_product(ctx, W, X, idx=i, scratch=scratch, y=wide[1:2101])
    assert got.data_ptr() == wide[1:2101].data_ptr() and torch.equal(got, want)
    assert (wide[0] == 7).all() and (wide[2101] == 7).all()
    with pytest.raises(B.SmoeError):
        B.smoe_mx_product(ctx, W, X, idx=i, scratch=scratch[:1024])
    assert B.smoe_mx_product(ctx, W, B.Mx(X.codes[:0], X.scales[:0]), idx=i[:0]).shape == (0, 3, 64)
    flat = B.Mx(W.codes[2], W.scales[2])
    assert torch.equal(B.smoe_mx_product(ctx, flat, X), B.smoe_mx_product(ctx, W, X, idx=torch.full((2100, 1), 2, dtype=torch.int32, device="cuda")))


MATVECS = [(1, 1, 1, 16, 32), (1, 6, 64, 64, 2048), (16, 1, 1, 48, 1408), (16, 16, 5, 32, 96), (5, 3, 9, 16, 160), (7, 2, 2, 208, 544), (16, 6, 64, 32, 128), (2, 4, 4, 16, 65536)]


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("T, k, E, N, K", MATVECS)
@pytest.mark.parametrize("how, slots", [("any", False), ("any", True), ("one", True), ("outside", False)])
def test_mx_matvec_exact(ctx, T, k, E, N, K, how, slots, act):
    rng = np.random.default_rng(T * 7 + N + K)
    w = mx_random(rng, E, N, K)
    x = rng.integers(-8, 9, size=(T, k, K) if slots else (T, K)).astype(np.float32) / 4
    idx = experts(rng, T, k, E, how)
    want = O.product(O.mx_values(*w), x.astype(np.float64), idx, False)
    assert np.abs(want).max() < 2 ** 19 and K * 12 * 2 < 2 ** 24 / 8       # multiples of 2^-4 (0.5 * 0.5 * 0.25), partial sums below 2^20
    W, X = B.Mx(*map(dev, w)), dev(x, DT[act])
    i = None if E == 1 and k == 1 and not slots else dev(idx)
    got = B.smoe_mx_matvec(ctx, W, X, idx=i)
    assert torch.equal(got.cpu(), torch.from_numpy(want).float().to(DT[act]))
    want = O.product(O.mx_values(*w), x.astype(np.float64), idx, True)
    close(B.smoe_mx_matvec(ctx, W, X, idx=i, swiglu=True), want, np.abs(want) * (8 * U32 + HALF[act]) + 1e-30)


def test_mx_matvec_takes_fp32_whole(ctx):
    """All 24 bits of an fp32 activation count, at every exponent; NaN and infinities come through."""
    rng = np.random.default_rng(4)
    N, K = 16, 128
    codes = np.zeros((1, N, K // 2), np.uint8)
    for n in range(N):
        codes[0, n, n * 4] = 2                               # weight 1 at column 8 n
    W = B.Mx(dev(codes), dev(np.full((1, N, K // 32), 127, np.uint8)))
    x = (rng.standard_normal((16, K)) * np.exp2(rng.integers(-60, 60, size=(16, K)))).astype(np.float32)
    got = np64(B.smoe_mx_matvec(ctx, W, dev(x)))[:, 0]
    assert np.array_equal(got, x[:, ::8].astype(np.float64))
    x[0] = 1.0
    x[0, 0], x[1] = np.finfo(np.float32).max, 0.0
    x[2, 8] = np.nan
    x[3, 8] = np.inf
    got = np64(B.smoe_mx_matvec(ctx, W, dev(x)))[:, 0]
    assert got[0, 0] == np.finfo(np.float32).max and (got[1] == 0).all() and np.isnan(got[2]).all()
    assert got[3, 1] == np.inf and np.isnan(got[3, 0])        # 1 * inf; 0 * inf in every other row


def test_mx_matvec_scales(ctx):
    rng = np.random.default_rng(8)
    w = mx_random(rng, 1, 16, 64)
    w[1][0, :, 0] = np.arange(110, 126)
    w[1][0, 3, 1] = 255
    x = rng.standard_normal((4, 64)).astype(np.float32)
    want = O.product(O.mx_values(*w), x.astype(np.float64), None, False)
    tol = O.product(np.abs(O.mx_values(*w)), np.abs(x.astype(np.float64)), None, False) * 64 * 2 * U32
    got = B.smoe_mx_matvec(ctx, B.Mx(*map(dev, w)), dev(x))
    close(got, want, np.where(np.isnan(tol), 0, tol))
    assert np.isnan(want[:, 0, 3]).all()


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 4])
def test_mx_matvec_ends_of_the_range(ctx, T, act):
    """Every code at the largest and smallest scales; activations down to the smallest."""
    N, K = 16, 64
    codes, scales = np.zeros((1, N, K // 2), np.uint8), np.full((1, N, 2), 127, np.uint8)
    codes[0, :, 0] = np.arange(16)                           # row n: code n at column 0
    for byte in (0, 1, 127, 250, 252, 253, 254):
        scales[0, :, 0] = byte
        W = B.Mx(dev(codes), dev(scales))
        w = O.mx_values(codes, scales)[0, :, 0]
        inf = np.abs(w) >= 2.0 ** 128
        for e in (-149, -133, -120, -110, 0, 100):
            x = torch.zeros(T, K)
            x[:, 0] = torch.tensor(1.5 + 2.0 ** -10 + 2.0 ** -23) * 2.0 ** max(e, -126) * 2.0 ** min(e + 126, 0)
            x = x.to(DT[act])
            want = np64(x)[0, 0] * w
            over = np.abs(want) > 3.3e38                     # (mantissas 1.5 and 2.25: none close to 2^128)
            # two additions (up to a step each), the activation's lost bits (bf16 has none there), the result's rounding and its smallest step
            tol = np.abs(want) * (4 * U32 + HALF[act]) + np.abs(w) * (2.0 ** -133 if act == "f32" else 0) + 2.0 ** (-133 if act == "bf16" else -149)
            got = np64(B.smoe_mx_matvec(ctx, W, x.cuda())).reshape(T, N)
            for row in got:
                assert not np.isfinite(row[inf]).any(), (byte, e)
                assert np.array_equal(row[over & ~inf], np.sign(want[over & ~inf]) * np.inf), (byte, e)
                fine = ~over & ~inf
                assert (np.abs(row - want)[fine] <= tol[fine]).all(), (byte, e)


@pytest.mark.parametrize("T", [1, 5])
def test_matvec_against_product(ctx, T):
    """Activations that quantise without loss: both products see the same numbers."""
    rng = np.random.default_rng(T)
    w = mx_random(rng, 8, 96, 256)
    x = mx_random(rng, T, 256)
    idx = dev(experts(rng, T, 3, 8, "any"))
    W, X = B.Mx(*map(dev, w)), B.Mx(*map(dev, x))
    a = B.smoe_mx_product(ctx, W, X, idx=idx)
    b = B.smoe_mx_matvec(ctx, W, B.smoe_mx_dequantize(ctx, X, torch.bfloat16), idx=idx)
    assert torch.equal(a, b)


# ---------------------------------------------------------------------------------- used together
def block(ctx, h, p, k, few):
    """One MoE block: norm, logits, routing, gate/up product with SwiGLU, down product, residual norm of the next block."""
    h, x = B.smoe_residual_norm(ctx, h, pre_w=p["pre"], act_dtype=torch.bfloat16)
    idx, w = B.smoe_route_scores(ctx, k, x=x, w_router=p["router"], score="sigmoid", n_group=4, topk_group=2, group_score="top2", bias=p["bias"],
                                 norm_topk=True, routed_scale=2.5)
    if few:
        y = B.smoe_mx_matvec(ctx, p["down"], B.smoe_mx_matvec(ctx, p["up"], x, idx=idx, swiglu=True), idx=idx)
    else:
        mid = B.smoe_mx_product(ctx, p["up"], B.smoe_mx_quantize(ctx, x), idx=idx, swiglu=True)
        y = B.smoe_mx_product(ctx, p["down"], B.smoe_mx_quantize(ctx, mid), idx=idx)
    return (*B.smoe_residual_norm(ctx, h, y=y, slot_w=w, post_w=p["post"], gate=p["gate"], scale=0.7, pre_w=p["pre"]), idx, w, x, y)


def block_params(seed, E=16, d=256, f=192):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)
    up, down = O.mx_quantize(r(E, 2 * f, d).numpy() * 0.05), O.mx_quantize(r(E, d, f).numpy() * 0.05)
    v = lambda t: t.bfloat16().cuda()
    return dict(pre=v(1 + 0.1 * r(d)), post=v(1 + 0.1 * r(d)), gate=v(r(d)), router=(r(E, d) * 0.1).cuda(), bias=(r(E) * 0.05).cuda(),
                up=B.Mx(*map(dev, up)), down=B.Mx(*map(dev, down))), g


@pytest.mark.parametrize("T, few", [(1, True), (7, True), (7, False), (150, False)])
def test_block(ctx, T, few):
    k, d = 4, 256
    p, g = block_params(T)
    h0 = torch.randn((T, d), generator=g).cuda()
    h, x2, idx, w, x, y = block(ctx, h0, p, k, few)
    # every stage against the definition from the stage's own inputs
    up, down = (O.mx_values(p[n].codes.cpu().numpy(), p[n].scales.cpu().numpy()) for n in ("up", "down"))
    i = idx.cpu().numpy()
    xq = np64(x) if few else O.mx_values(*O.mx_quantize(np64(x)))
    mid = torch.from_numpy(O.product(up, xq, i, True)).float().bfloat16()
    mid = np64(mid) if few else O.mx_values(*O.mx_quantize(np64(mid)))
    want = O.product(down, mid, i, False)
    # a value of `mid` on a border may round to its neighbour, a step of at most 2^-7 (bf16) or a third (4 bits): rare, so held to the norm
    assert np.linalg.norm(np64(y) - want) <= (2.0 ** -7 if few else 2.0 ** -5) * np.linalg.norm(want)
    hw, xw = O.residual_norm(np64(h0), np64(y), np64(w), np64(p["post"]), np64(p["gate"]), 0.7, np64(p["pre"]), 1e-6)
    assert np.linalg.norm(np64(h) - hw) <= 1e-5 * np.linalg.norm(hw) and np.linalg.norm(np64(x2) - xw) <= 2.0 ** -8 * np.linalg.norm(xw)


def test_block_in_a_graph(ctx):
    """Captured once, replayed on new contents, with eager calls of other sizes between the replays."""
    p, g = block_params(3)
    s = torch.cuda.Stream()
    c = B.Ctx(0, stream=s, workspace_bytes=0)
    h0 = torch.zeros((40, 256), device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        block(c, h0, p, 4, False)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        out = block(c, h0, p, 4, False)
    for rep in range(4):
        new = torch.randn((40, 256), generator=g)
        h0.copy_(new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = block(ctx, new.cuda(), p, 4, False)
        block(ctx, torch.randn((130 + rep, 256), device="cuda"), p, 4, False)
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)
    c.close()


def test_calls_on_another_stream(ctx):
    """A context of its own stream: ordered by events, its results are those of the default stream."""
    p, g = block_params(4)
    s = torch.cuda.Stream()
    c = B.Ctx(0, stream=s, workspace_bytes=0)
    h0 = torch.randn((33, 256), generator=g).cuda()
    want = block(ctx, h0, p, 4, False)
    for _ in range(3):
        s.wait_stream(torch.cuda.current_stream())
        got = block(c, h0, p, 4, False)
        torch.cuda.current_stream().wait_stream(s)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    c.close()
