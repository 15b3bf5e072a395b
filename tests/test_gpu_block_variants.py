"""Every kernel variant of the products around MXFP4 experts and of the score routing, against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import block_cases
from oracle import block_oracle as O
from paper_2512_12990_amd import binding as B
from test_gpu_block_ops import DT, HALF, U32, check_route, close, dev, experts, mx_random, np64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Ctx(0, workspace_bytes=0)
    yield c
    c.close()


def used_values(w, idx, E):
    """(values of the experts that idx names, idx among them); an index outside counts as the nearest expert."""
    used, local = np.unique(np.clip(idx, 0, E - 1), return_inverse=True)
    return O.mx_values(w[0][used], w[1][used]), local.reshape(idx.shape)


def silu_product(y):
    with np.errstate(over="ignore"):
        return O.silu(y[..., 0::2]) * y[..., 1::2]


def swiglu_close(got, want, out):
    # gate and up are exact sums; silu(g) * u is off by at most 9 half steps of fp32, then comes the result's rounding (in products of normal size)
    close(got, want, np.abs(want) * (9 * U32 + HALF[out]) + 1e-30)


# ------------------------------------------------------------------------------------------- matvec
@pytest.mark.parametrize("how, slots", [("any", False), ("any", True), ("one", True), ("outside", False)])
@pytest.mark.parametrize("T, k, E, N, K", block_cases.MATVEC_FOUR_TILES + block_cases.MATVEC_ONE_TILE)
def test_matvec_forms_exact(ctx, T, k, E, N, K, how, slots):
    """Sums that fp32 holds without rounding have to be exact, whatever their order."""
    rng = np.random.default_rng(T * 7 + N + K)
    w = mx_random(rng, E, N, K)
    x = rng.integers(-8, 9, size=(T, k, K) if slots else (T, K)).astype(np.float32) / 4
    idx = experts(rng, T, k, E, how)
    values, local = used_values(w, idx, E)
    want = O.product(values, x.astype(np.float64), local, False)
    assert K * 12 * 2 < 2 ** 24 / 16                         # multiples of 2^-4, partial sums below 2^20
    W = B.Mx(*map(dev, w))
    i = None if E == 1 and k == 1 and not slots else dev(idx)
    for act in ("f32", "bf16"):
        X = dev(x, DT[act])
        got = B.smoe_mx_matvec(ctx, W, X, idx=i)
        assert torch.equal(got.cpu(), torch.from_numpy(want).float().to(DT[act]))
        swiglu_close(B.smoe_mx_matvec(ctx, W, X, idx=i, swiglu=True), silu_product(want), act)


@pytest.mark.parametrize("T", [1, 2, 16])
def test_matvec_four_tiles_takes_fp32_whole(ctx, T):
    """All 24 bits of an fp32 activation count, at every exponent; infinities and NaN come through."""
    rng = np.random.default_rng(4)
    N, K = 8208, 96
    codes = np.zeros((N, K // 2), np.uint8)
    col = (np.arange(N) * 7) % K
    codes[np.arange(N), col // 2] = 2 << (4 * (col % 2))      # row n: weight 1 at column 7 n % K
    W = B.Mx(dev(codes), dev(np.full((N, K // 32), 127, np.uint8)))
    x = (rng.standard_normal((T, K)) * np.exp2(rng.integers(-60, 60, size=(T, K)))).astype(np.float32)
    assert np.array_equal(np64(B.smoe_mx_matvec(ctx, W, dev(x)))[:, 0], x[:, col].astype(np.float64))
    x[0] = 0.0
    x[0, 7], x[-1, 14] = np.inf, np.nan
    got = np64(B.smoe_mx_matvec(ctx, W, dev(x)))[:, 0]
    if T > 1:
        assert (got[0, col == 7] == np.inf).all()
        assert np.isnan(got[0, col != 7]).all()               # 0 * inf
    assert np.isnan(got[-1]).all()


# ------------------------------------------------------------------------------------------ product
CASES = [c for group in (block_cases.PRODUCT_SEARCH, block_cases.PRODUCT_LIST, block_cases.PRODUCT_PLAIN) for pair in group for c in pair]


@pytest.mark.parametrize("T, k, E, N, K, how", [(*c, how) for c in CASES for how in ("any", "outside", "skewed") if how == "any" or c[2] > 1])
def test_product_variants_exact(ctx, T, k, E, N, K, how):
    rng = np.random.default_rng(T * 7 + N + K)
    slots = how == "outside"
    w, x = mx_random(rng, E, N, K), mx_random(rng, *((T, k, K) if slots else (T, K)))
    if how == "skewed":                                      # one expert with most of the slots, some with none, the same one twice for a token
        idx = np.where(rng.random((T, k)) < 0.7, E // 2, rng.integers(0, max(1, E // 3), size=(T, k))).astype(np.int32)
    else:
        idx = experts(rng, T, k, E, how)
    values, local = used_values(w, idx, E)
    want = O.product(values, O.mx_values(*x), local, False)
    assert K * 36 * 4 < 2 ** 24 / 16                         # multiples of 2^-4, partial sums below 2^20
    W, X = B.Mx(*map(dev, w)), B.Mx(*map(dev, x))
    i = dev(idx) if E > 1 else None
    exact = torch.from_numpy(want)
    assert torch.equal(B.smoe_mx_product(ctx, W, X, idx=i, out_dtype=torch.float32).cpu(), exact.float())
    assert torch.equal(B.smoe_mx_product(ctx, W, X, idx=i).cpu(), exact.float().bfloat16())
    del exact
    swiglu_close(B.smoe_mx_product(ctx, W, X, idx=i, swiglu=True), silu_product(want), "bf16")


@pytest.mark.parametrize("T, k, E, N, K", [(5, 2, 6, 48, 65536), (40, 1, 1, 64, 10944), (33, 1, 1, 32, 65504), (300, 2, 3, 144, 10976), (1600, 1, 1, 2064, 10944), (4100, 1, 1, 2064, 5472)])
def test_product_of_long_rows_exact(ctx, T, k, E, N, K):
    """Numbers up to 1 without scales: sums of up to 65536 products are multiples of 1/4 that fp32 holds, so a column lost anywhere shows."""
    rng = np.random.default_rng(K + T)
    def small(*shape):
        n = rng.integers(0, 3, size=shape, dtype=np.uint8) + 8 * rng.integers(0, 2, size=shape, dtype=np.uint8)      # 0, 1/2, 1 and their negatives
        return n[..., 0::2] | (n[..., 1::2] << 4), np.full(shape[:-1] + (shape[-1] // 32,), 127, np.uint8)
    w, x = small(E, N, K), small(T, K)
    idx = experts(rng, T, k, E, "any")
    assert K * 4 < 2 ** 24
    W, X = B.Mx(*map(dev, w)), B.Mx(*map(dev, x))
    got = np64(B.smoe_mx_product(ctx, W, X, idx=dev(idx) if E > 1 else None, out_dtype=torch.float32))
    # (fp32 sums of the definition are exact for the same reason)
    wv, xv = (O.mx_values(*m).astype(np.float32) for m in (w, x))
    for e in range(E):
        t, j = np.nonzero(idx == e)
        assert np.array_equal(got[t, j], (xv[t] @ wv[e].T).astype(np.float64)), e


# ------------------------------------------------------------------------------------------ routing
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E, ng, tg, k", block_cases.ROUTE_PART_LANES + block_cases.ROUTE_ODD_GROUPS)
def test_route_scores_of_any_number_of_experts(ctx, E, ng, tg, k, score):
    """Lanes without experts, groups of any size: plain logits, ties, neighbours in fp32, masks, large ones."""
    rng = np.random.default_rng(E + ng)
    z = rng.standard_normal((block_cases.ROUTE_TOKENS, E)).astype(np.float32) * 2
    z[:60] = 1.0 + rng.integers(-2, 3, size=(60, E)) * 2.0 ** -23
    z[60:120] = np.round(rng.standard_normal((60, E)) * 4) / 4
    z[120:160] = -70 + rng.random((40, E))
    z[160:200] = 12 + rng.random((40, E)) * 30
    z[200:260][rng.random((60, E)) < 0.4] = -np.inf
    z[260] = -np.inf
    z[261:300] = rng.standard_normal((39, E)) * 1000
    z[300:320] = -20 - 50 * rng.random((20, E))               # below what stands for a lane without experts
    b = (rng.standard_normal(E) * 0.05).astype(np.float32)
    check_route(ctx, z, k, score=score, ng=ng, tg=tg, gs="max", norm=False, scale=2.5)
    check_route(ctx, z, k, score=score, ng=ng, tg=tg, gs="top2", bias=b - 3.0, norm=True)
