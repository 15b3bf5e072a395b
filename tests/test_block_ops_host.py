"""CPU-only tests of score routing, residual norm and microscaled floats: pins of their oracle, and every refusal of the C
entries (made before any device call, so a context of zeros will do)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import block_oracle as O
from paper_2512_12990_amd import binding as B

P = 1 << 20                      # an aligned address that no refused call looks at


@pytest.fixture(scope="module")
def ctx():
    buf = C.create_string_buffer(1 << 14)
    yield C.addressof(buf)
    del buf


# ------------------------------------------------------------------------------------ oracle's pins
def test_quantiser_pins():
    x = np.zeros((1, 64))
    x[0, :16] = [0, .25, .26, .75, .74, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, 6.0, 7.9, -0.25, -0.75, -7.0]
    x[0, 32:36] = [0.75, 0.125, -0.0625, 0.09375]
    codes, scales = O.mx_quantize(x)
    assert scales.tolist() == [[127, 124]]
    # ties to the even code; magnitudes above 6 saturate
    want = [0, 0, .5, 1, .5, 1, 2, 2, 4, 4, 6, 6, 6, 0, -1, -6]
    v = O.mx_values(codes, scales)
    assert v[0, :16].tolist() == want
    assert v[0, 32:36].tolist() == [0.75, 0.125, -0.0625, 0.125]     # unit 1/8; 0.09375 is 0.75 units, a tie that goes to 1
    assert codes[0, 0] == 0x00 and codes[0, 1] == 0x21            # even column in the low nibble
    assert codes[0, 6] & 0xF0 == 0x80 and codes[0, 7] == 0xFA       # -0.25 keeps its sign as -0; -1, -6 are codes 10 and 15


def test_quantiser_edges():
    x = np.zeros((6, 32))
    x[1, 3] = 2.0 ** -130
    x[2, 0] = 3.0e38
    x[3, 7] = np.nan
    x[4, 9] = -np.inf
    x[5] = 2.0 ** -149
    codes, scales = O.mx_quantize(x)
    assert scales[:, 0].tolist() == [0, 0, 252, 255, 255, 0]
    v = O.mx_values(codes, scales)
    assert (v[0] == 0).all() and v[1, 3] == 0.0 and np.isnan(v[3]).all() and np.isnan(v[4]).all() and (v[5] == 0).all()
    assert v[2, 0] == 6 * 2.0 ** 125                                # 3e38 = 7.05 * 2^125


def test_routing_pins():
    z = np.log(np.array([[1.0, 2.0, 3.0, 4.0]], np.float32)).astype(np.float32)
    idx, w = O.route_scores(z, 2, "softmax", 1, 1, "max", None, False, 1.0)
    assert idx.tolist() == [[3, 2]] and np.allclose(w, [[0.4, 0.3]], atol=1e-7)
    idx, w = O.route_scores(z, 2, "softmax", 1, 1, "max", np.array([0.35, 0, 0, 0], np.float32), True, 2.0)
    assert idx.tolist() == [[0, 3]] and np.allclose(w, [[0.4, 1.6]], atol=1e-6)
    # groups: the largest stands in the first group, the largest pair in the second
    z = np.array([[5.0, 0.0, 4.0, 4.0]], np.float32)
    assert O.route_scores(z, 1, "softmax", 2, 1, "max", None, False, 1.0)[0].tolist() == [[0]]
    assert O.route_scores(z, 1, "sigmoid", 2, 1, "top2", None, False, 1.0)[0].tolist() == [[2]]
    z = np.full((1, 4), -np.inf, np.float32)
    idx, w = O.route_scores(z, 2, "softmax", 1, 1, "max", None, True, 1.0)
    assert idx.tolist() == [[0, 1]] and w.tolist() == [[0.0, 0.0]]


def test_norm_pins():
    h, x = O.residual_norm(np.array([[3.0, 4.0]]), np.array([[[1.0, 0.0], [0.0, 1.0]]]), np.array([[2.0, 4.0]]), None, None, 0.5, np.array([1.0, 2.0]), 0.0)
    assert h.tolist() == [[4.0, 6.0]]
    assert np.allclose(x, [[4 / 26 ** 0.5, 12 / 26 ** 0.5]])


# ------------------------------------------------------------------------------------------ refusals
def _route(ctx, **kw):
    a = dict(T=4, E=8, k=2, d=0, logits=P, x=None, act=0, wr=None, score=0, ng=1, tg=1, gs=0, bias=None, norm=0, scale=1.0, idx=P, w=P)
    a.update(kw)
    return B.lib().smoe_route_scores(ctx, *a.values())


@pytest.mark.parametrize("kw, rc", [
    (dict(idx=None), -1), (dict(w=None), -1), (dict(logits=None), -1), (dict(logits=None, x=P), -1), (dict(act=2), -1), (dict(score=2), -1),
    (dict(gs=2), -1), (dict(score=-1), -1), (dict(T=-1), -2), (dict(T=(1 << 22) + 1), -2), (dict(E=0), -2), (dict(E=257), -2), (dict(k=0), -2), (dict(k=9), -2),
    (dict(E=64, k=17), -2), (dict(ng=3), -2), (dict(ng=0), -2), (dict(E=256, ng=128), -2), (dict(ng=4, tg=0), -2), (dict(ng=4, tg=5), -2),
    (dict(ng=4, tg=1, k=3), -2), (dict(logits=None, x=P, wr=P, d=0), -2), (dict(logits=P + 4), -3), (dict(bias=P + 8), -3), (dict(idx=P + 4), -3),
    (dict(w=P + 4), -3), (dict(logits=None, x=P, wr=P, act=1, d=64000), -4),
])
def test_route_scores_refuses(ctx, kw, rc):
    assert _route(ctx, **kw) == rc


def test_zero_tokens_and_null_context(ctx):
    assert _route(ctx, T=0, logits=None, idx=None, w=None) == 0 and _route(None) == -1
    assert _norm(ctx, T=0, y=None, res=None, ro=None, xo=None) == 0 and _norm(None) == -1
    assert _quant(ctx, rows=0, src=None, codes=None, scales=None) == (0, 0) and _quant(None) == (-1, -1)
    assert _product(ctx, T=0, x=None, idx=None, y=None) == 0 and _product(None) == -1
    assert _matvec(ctx, T=0, x=None, idx=None, y=None) == 0 and _matvec(None) == -1


def _norm(ctx, **kw):
    a = dict(T=4, d=64, k=2, y=P, sw=P, post=P, gate=P, gr=0, scale=1.0, res=2 * P, pre=P, eps=1e-6, act=0, rd=0, ro=3 * P, xo=4 * P)
    a.update(kw)
    return B.lib().smoe_residual_norm(ctx, *a.values())


@pytest.mark.parametrize("kw, rc", [
    (dict(ro=None, xo=None), -1), (dict(y=None, k=0, sw=None, post=None, gate=None, res=None), -1), (dict(y=None), -1), (dict(k=0), -1),
    (dict(y=None, k=0), -1), (dict(act=2), -1), (dict(rd=-1), -1), (dict(gr=2), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
    (dict(xo=2 * P), -1), (dict(xo=P), -1), (dict(xo=3 * P), -1), (dict(ro=P), -1), (dict(T=-1), -2), (dict(d=0), -2), (dict(d=60), -2),
    (dict(d=16392), -2), (dict(k=25), -2), (dict(k=-1), -2), (dict(T=(1 << 22) + 1), -2),
    (dict(y=P + 2), -3), (dict(sw=P + 4), -3), (dict(post=P + 8), -3), (dict(gate=P + 1), -3), (dict(res=P + 4), -3), (dict(pre=P + 4), -3), (dict(ro=P + 4), -3),
    (dict(xo=P + 4), -3),
])
def test_residual_norm_refuses(ctx, kw, rc):
    assert _norm(ctx, **kw) == rc


def _quant(ctx, **kw):
    a = dict(rows=4, K=64, src=P, dt=0, codes=P, scales=P)
    a.update(kw)
    lib = B.lib()
    return (lib.smoe_mx_quantize(ctx, a["rows"], a["K"], a["src"], a["dt"], a["codes"], a["scales"]),
            lib.smoe_mx_dequantize(ctx, a["rows"], a["K"], a["codes"], a["scales"], a["src"], a["dt"]))


@pytest.mark.parametrize("kw, rc", [
    (dict(src=None), -1), (dict(codes=None), -1), (dict(scales=None), -1), (dict(dt=3), -1), (dict(rows=-1), -2), (dict(K=0), -2), (dict(K=48), -2),
    (dict(rows=1 << 30), -2), (dict(src=P + 8), -3), (dict(codes=P + 4), -3), (dict(scales=P + 1), -3),
])
def test_mx_quantize_refuses(ctx, kw, rc):
    assert _quant(ctx, **kw) == (rc, rc)


def _product(ctx, **kw):
    a = dict(E=4, N=64, K=64, wc=P, ws=P, T=3000, k=2, x=P, xs=P, slots=0, idx=P, sg=0, dt=0, scratch=P, nbytes=1 << 20, y=P)
    a.update(kw)
    return B.lib().smoe_mx_product(ctx, *a.values())


@pytest.mark.parametrize("kw, rc", [
    (dict(wc=None), -1), (dict(ws=None), -1), (dict(x=None), -1), (dict(xs=None), -1), (dict(y=None), -1), (dict(scratch=None), -1), (dict(slots=2), -1),
    (dict(sg=2), -1), (dict(dt=2), -1), (dict(E=0), -2), (dict(E=257), -2), (dict(N=0), -2), (dict(N=24), -2), (dict(N=(1 << 20) + 16), -2), (dict(K=0), -2),
    (dict(K=48), -2), (dict(K=65568), -2), (dict(N=1 << 20, K=8192), -2), (dict(T=-1), -2), (dict(k=0), -2), (dict(k=17), -2),
    (dict(T=1 << 21, k=4, nbytes=1 << 40), -2), (dict(T=1 << 20, K=4096, nbytes=1 << 40), -2), (dict(idx=None), -2), (dict(idx=None, E=1), -2),
    (dict(T=1 << 20, k=4, N=1 << 20, nbytes=1 << 40), -2),
    (dict(wc=P + 8), -3), (dict(ws=P + 8), -3), (dict(x=P + 8), -3), (dict(xs=P + 8), -3), (dict(idx=P + 8), -3), (dict(scratch=P + 8), -3), (dict(y=P + 8), -3),
    (dict(nbytes=64), -4),
])
def test_mx_product_refuses(ctx, kw, rc):
    assert _product(ctx, **kw) == rc


def test_mx_product_bytes():
    n = C.c_size_t()
    lib = B.lib()
    assert lib.smoe_mx_product_bytes(5, 2, 4, 64, None) == -1
    for args in [(-1, 2, 4, 64), (5, 0, 4, 64), (5, 17, 4, 64), (5, 2, 0, 64), (5, 2, 257, 64), (1 << 22, 2, 4, 64), (5, 2, 4, 0), (5, 2, 4, 24)]:
        assert lib.smoe_mx_product_bytes(*args, C.byref(n)) == -2
    # the slots listed by expert and, for each tile, a record; none where there are few
    assert B.smoe_mx_product_bytes(2048, 4, 60, 2816) >= 2048 * 4 * 4
    assert B.smoe_mx_product_bytes(3000, 2, 4, 64) >= 6000 * 4
    assert B.smoe_mx_product_bytes(0, 4, 60, 64) == 0 and B.smoe_mx_product_bytes(1024, 4, 60, 64) == 0
    assert B.smoe_mx_product_bytes(1025, 4, 60, 64) > 0


def _matvec(ctx, **kw):
    a = dict(E=4, N=64, K=64, wc=P, ws=P, T=5, k=2, x=P, dt=0, slots=0, idx=P, sg=0, y=2 * P)
    a.update(kw)
    return B.lib().smoe_mx_matvec(ctx, *a.values())


@pytest.mark.parametrize("kw, rc", [
    (dict(wc=None), -1), (dict(ws=None), -1), (dict(x=None), -1), (dict(y=None), -1), (dict(y=P), -1), (dict(slots=2), -1), (dict(sg=-1), -1), (dict(dt=2), -1),
    (dict(E=0), -2), (dict(E=257), -2), (dict(N=24), -2), (dict(K=48), -2), (dict(T=17), -2), (dict(T=-1), -2), (dict(k=17), -2), (dict(idx=None), -2),
    (dict(wc=P + 8), -3), (dict(ws=P + 8), -3), (dict(x=P + 8), -3), (dict(idx=P + 8), -3), (dict(y=P + 8), -3),
])
def test_mx_matvec_refuses(ctx, kw, rc):
    assert _matvec(ctx, **kw) == rc


class _FakeCtx:
    device, h, raw_stream = 0, None, 0


@pytest.mark.parametrize("call", [
    lambda c: B.smoe_route_scores(c, 2, logits=torch.zeros(4, 8), score="tanh"),
    lambda c: B.smoe_route_scores(c, 2, logits=torch.zeros(4, 8), group_score="mean"),
    lambda c: B.smoe_route_scores(c, 2, logits=torch.zeros(4, 8, dtype=torch.float64)),
    lambda c: B.smoe_route_scores(c, 2, logits=torch.zeros(4, 8)),                                   # on the CPU
    lambda c: B.smoe_route_scores(c, 2),
    lambda c: B.smoe_route_scores(c, 2, x=torch.zeros(4, 8)),
    lambda c: B.smoe_residual_norm(c, None),
    lambda c: B.smoe_residual_norm(c, torch.zeros(4, 64, dtype=torch.float16)),
    lambda c: B.smoe_residual_norm(c, torch.zeros(4, 64), act_dtype=torch.float16),
    lambda c: B.smoe_mx_quantize(c, torch.zeros(32)),
    lambda c: B.smoe_mx_quantize(c, torch.zeros(())),
    lambda c: B.smoe_mx_quantize(c, torch.zeros(4, 0)),
    lambda c: B.smoe_mx_quantize(c, torch.zeros(4, 48)),
    lambda c: B.smoe_mx_quantize(c, torch.zeros(4, 64, dtype=torch.float16)),
    lambda c: B.smoe_mx_dequantize(c, B.Mx(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))),
    lambda c: B.smoe_mx_matvec(c, B.Mx(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)), torch.zeros(4, 64)),
    lambda c: B.smoe_mx_matvec(c, B.Mx(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)), torch.zeros(())),
])
def test_binding_refuses(call, monkeypatch):
    monkeypatch.setattr(B, "_stream_now", lambda device: 0)              # (no device to ask here)
    with pytest.raises(B.SmoeError):
        call(_FakeCtx())
