"""Score routing, residual norm and microscaled products where numbers, sizes and kernel variants reach their ends."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as O
from paper_2512_12990_amd import binding as B
from test_gpu_block_ops import DT, HALF, U32, dev, mx_random, np64

pytestmark = pytest.mark.gpu

TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133}      # smallest step of the type


@pytest.fixture(scope="module")
def ctx():
    c = B.Ctx(0, workspace_bytes=0)
    yield c
    c.close()


# ------------------------------------------------------------------------------------------ SwiGLU
UPS = np.array([1.0, -1.0, 1.5e10, -2.5e20, 1.25e30, 3e38, 1e-20, -3e38])
GATES = np.array([-60, -75.9, -76.1, -76.3, -80, -86, -87.2, -87.5, -88, -88.6, -88.8, -89, -95, -100, -104, -110,
                  -120, -130, -140, -150, -160, -170, -175, -180, -185, -190, -195, -200, -206, -210, -250, -3e38])


def check_swiglu(got, g, u, out):
    """silu(g) * u; the kernel's own bound is 9 half steps of fp32, and the result is rounded once more."""
    g, u = np.broadcast_arrays(g, u)
    with np.errstate(over="ignore"):
        want = g / (1.0 + np.exp(-g)) * u
    tol = np.abs(want) * (9 * U32 + HALF[out]) + TINY[out]
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), [(float(a), float(b), float(c), float(d)) for a, b, c, d in zip(g[bad], u[bad], got[bad], want[bad])][:5]


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_matvec_swiglu_far_below_zero(ctx, act):
    """Gates from -60 on down: silu(g) is no fp32 number there or a subnormal one, silu(g) * u still is."""
    N, K = 16, 32
    codes = np.zeros((1, N, K // 2), np.uint8)
    codes[0, 0::2, 0] = 2                                    # every gate row: weight 1 at column 0
    for i in range(8):
        codes[0, 2 * i + 1, (8 + i) // 2] = 2 << (4 * (i % 2))      # up row i: weight 1 at column 8 + i
    W = B.Mx(dev(codes), dev(np.full((1, N, 1), 127, np.uint8)))
    for at in (0, 16):
        x = torch.zeros(16, K, dtype=torch.float64)
        x[:, 0] = torch.from_numpy(GATES[at:at + 16])
        x[:, 8:16] = torch.from_numpy(UPS)
        x = x.to(DT[act])
        got = np64(B.smoe_mx_matvec(ctx, W, x.cuda(), swiglu=True))[:, 0]
        x = np64(x)
        check_swiglu(got, x[:, :1], x[:, 8:16], act)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("T, N", [(72, 16), (1600, 2064), (4100, 2064)])
def test_product_swiglu_far_below_zero(ctx, T, N, out):
    """The same in the product of quantised numbers, in each tile shape: a gate is the sum of codes times 16 and of codes times a half.  With many rows three
    in four have ordinary gates, next to them and in waves of their own."""
    grid = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
    gates = [((4, 1, 0), (0, 0)), ((4, 1, .5), (0, 0)), ((4, 1.5, 0), (0, 0)), ((4, 1.5, 0), (1.5, 0)), ((4, 1.5, 0), (2, 0)), ((6, 0, 0), (0, 0)),
             ((6, 1.5, 0), (0, 0)), ((6, 3, 0), (1, 0)), ((6, 4, 1), (3, 0)), ((6, 6, 0), (0, 0)), ((6, 6, .5), (4, 1)), ((6, 6, 6), (0, 0))]
    ups = [(1, 127), (1.5, 127 + 30), (-6, 127 + 60), (3, 127 + 100), (-4, 127 + 120), (1, 127 - 60)]
    code = lambda v: int(np.nonzero(grid == abs(v))[0][0]) + (8 if v < 0 else 0)
    K = 96
    wn = np.zeros((N, K), np.uint8)                          # codes, one a column
    wn[0::2, [0, 1, 2, 32, 33]] = 2
    wn[1::2, 64] = 2
    xn, xs, g, u = [], [], [], []
    for coarse, fine in gates:
        for v, byte in ups:
            row = np.zeros(K, np.uint8)
            row[:3], row[32:34], row[64] = [code(-c) for c in coarse], [code(-c) for c in fine], code(v)
            xn.append(row)
            xs.append([131, 126, byte])
            g.append(-16.0 * sum(coarse) - 0.5 * sum(fine))
            u.append(v * 2.0 ** (byte - 127))
    if T > 72:
        at = np.random.default_rng(T).integers(0, len(g), size=T)
        xn, xs, g, u = ([v[i] for i in at] for v in (xn, xs, g, u))
        for t in range(T):
            if t % 4 or t > T // 2:
                xn[t] = xn[t].copy()
                xn[t][:3] &= 8                               # gates of -4 and more
                g[t] = -0.5 * sum(float(grid[n & 7]) for n in xn[t][32:34])
    pack = lambda n: np.ascontiguousarray(n[..., 0::2] | (n[..., 1::2] << 4))
    W = B.Mx(dev(pack(wn)), dev(np.full((N, 3), 127, np.uint8)))
    X = B.Mx(dev(pack(np.stack(xn))), dev(np.array(xs, np.uint8)))
    got = np64(B.smoe_mx_product(ctx, W, X, swiglu=True, out_dtype=DT[out]))[:, 0]
    check_swiglu(got, np.array(g)[:, None] + np.zeros((1, N // 2)), np.array(u)[:, None] + np.zeros((1, N // 2)), out)


# ------------------------------------------------------------------------------------ largest launches
def room_for(nbytes):
    """Skips where the device has not that much free memory."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < nbytes:
        pytest.skip("needs %d GB of free device memory" % (nbytes >> 30))


@pytest.mark.parametrize("T, d", [(1 << 22, 8200), ((1 << 20) + 3, 8200), ((1 << 20) + 1, 520), (1 << 22, 512)])
def test_residual_norm_most_rows(ctx, T, d):
    """More rows than one launch takes: every token is served once, the last ones too."""
    room_for(T * d * 4 + (8 << 30))
    res = torch.ones((T, d), dtype=torch.bfloat16, device="cuda")
    at = sorted({0, 1, (1 << 20) - 1, 1 << 20, T // 2 + 5, T - 2, T - 1} & set(range(T)))
    rows = torch.randn((len(at), d), generator=torch.Generator().manual_seed(d)).bfloat16()
    res[torch.tensor(at, device="cuda")] = rows.cuda()
    out, x = B.smoe_residual_norm(ctx, res, res_out=res)
    assert out is res
    i = torch.tensor(at, device="cuda")
    want = np64(rows)
    assert np.array_equal(np64(res[i]), want)
    # sum of squares: at most 54 roundings, halved by the root, and 4 of mean, eps, root and division; then the result's own and the type's
    want = want / np.sqrt((want * want).mean(-1, keepdims=True) + 1e-6)
    got = np64(x[i])
    assert (np.abs(got - want) <= np.abs(want) * (33 * U32 + HALF["bf16"])).all()
    x[i] = 1.0                                               # everywhere else 1 / sqrt(1 + 1e-6) is 1 in bfloat16
    for a in range(0, T, 1 << 18):
        assert (x[a:a + (1 << 18)] == 1.0).all()


@pytest.mark.parametrize("act, res", [("bf16", "f32"), ("f32", "bf16")])
def test_residual_norm_most_rows_with_everything(ctx, act, res):
    """Every operand moves on with the rows: the last rows are those of a call on them alone."""
    T, d, k = (1 << 21) + 3, 16, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    y, w, gate, h = r(T, k, d).to(DT[act]), r(T, k), r(T, d).to(DT[act]), r(T, d).to(DT[res])
    kw = dict(post_w=r(d).to(DT[act]), pre_w=r(d).to(DT[act]), scale=0.5)
    out = B.smoe_residual_norm(ctx, h, y=y, slot_w=w, gate=gate, **kw)
    for a, b in ((0, 8), ((1 << 20) - 8, 1 << 20), (1 << 20, (1 << 20) + 8), (T - 11, T)):
        part = B.smoe_residual_norm(ctx, h[a:b].clone(), y=y[a:b].clone(), slot_w=w[a:b].clone(), gate=gate[a:b].clone(), **kw)
        assert torch.equal(out[0][a:b], part[0]) and torch.equal(out[1][a:b], part[1])
    kw["gate"] = gate[0]
    out = B.smoe_residual_norm(ctx, h, y=y, slot_w=w, **kw)
    part = B.smoe_residual_norm(ctx, h[-9:].clone(), y=y[-9:].clone(), slot_w=w[-9:].clone(), **kw)
    assert torch.equal(out[0][-9:], part[0]) and torch.equal(out[1][-9:], part[1])


@pytest.mark.parametrize("T, d, act", [(1 << 22, 7400, "f32"), ((1 << 20) + 3, 14700, "bf16"), ((1 << 21) + 5, 6000, "f32")])
def test_route_scores_from_activations_most_tokens(ctx, T, d, act):
    """One or two wide tokens to a work-group, and more work-groups than one launch takes."""
    size = T * d * (4 if act == "f32" else 2)
    room_for(size + (4 << 30))
    x = torch.zeros((T, d), dtype=DT[act], device="cuda")
    at = sorted({0, 1, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, T // 2 + 5, T - 2, T - 1} & set(range(T)))
    x[torch.tensor(at, device="cuda"), 3] = 1.0
    wr = torch.zeros((3, d), device="cuda")
    wr[:, 3] = torch.tensor([0.0, 1.0, 3.0])                 # logits 0 everywhere (a tie: expert 0, then 1), or 0, 1, 3
    idx, w = B.smoe_route_scores(ctx, 2, x=x, w_router=wr, score="softmax")
    del x
    other = torch.ones(T, dtype=torch.bool, device="cuda")
    other[torch.tensor(at, device="cuda")] = False
    assert (idx[other] == torch.tensor([0, 1], device="cuda")).all() and (w[other] == torch.tensor(1.0 / 3.0)).all()
    s = np.exp([0.0, 1.0, 3.0]) / np.exp([0.0, 1.0, 3.0]).sum()
    assert (idx[~other] == torch.tensor([2, 1], device="cuda")).all()
    assert (np.abs(np64(w[~other]) - s[[2, 1]]) <= s[[2, 1]] * 2 * U32).all()


# ------------------------------------------------------------------------------- formats, graphs
def test_mx_dequantize_every_code_and_scale_to_bf16(ctx):
    """A power of two with one more bit: exact in bfloat16 down to its subnormals, infinite from 2^128 on."""
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(1, 16, 16), (256, 1, 1)).reshape(256, 256)
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, 1)
    want = O.mx_values(codes, scales)
    big = np.abs(want) >= 2.0 ** 128
    want[big] = np.copysign(np.inf, want[big])
    assert np.array_equal(np64(B.smoe_mx_dequantize(ctx, B.Mx(dev(codes), dev(scales)), torch.bfloat16)), want, equal_nan=True)


def test_first_product_of_a_context_is_captured():
    """A context's first call of the widest tile asks for its LDS while a graph is captured; replays on new contents, with eager work between them."""
    rng = np.random.default_rng(2)
    T, N, K = 4100, 2064, 128
    w, x = mx_random(rng, N, K), mx_random(rng, T, K)
    W, X = B.Mx(*map(dev, w)), B.Mx(*map(dev, x))
    s = torch.cuda.Stream()
    c = B.Ctx(0, stream=s, workspace_bytes=0)
    y = torch.zeros((T, 1, N), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.smoe_mx_product(c, W, X, y=y)
    for _ in range(3):
        x = mx_random(rng, T, K)
        X.codes.copy_(dev(x[0]))
        X.scales.copy_(dev(x[1]))
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = O.product(O.mx_values(*w)[None], O.mx_values(*x), None, False)
        assert torch.equal(y.cpu(), torch.from_numpy(want).float().bfloat16())
        B.smoe_mx_quantize(c, torch.randn(64, 64, device="cuda"))
        torch.cuda.synchronize()
    c.close()
