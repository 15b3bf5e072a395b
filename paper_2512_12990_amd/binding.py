"""Thin ctypes binding of libslicemoe.so: argument marshalling only.

Every function has the name and meaning of the C entry point in include/slicemoe.h; torch
tensors are used for device memory and the current stream only.  There is no CPU fallback:
if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import NamedTuple, Optional

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libslicemoe.so")

F32, BF16 = 0, 1
_DT = {torch.float32: F32, torch.bfloat16: BF16, "f32": F32, "bf16": BF16}


class SmoeError(RuntimeError):
    pass


class BankDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("n_experts", "d_model", "d_ff", "group", "b_high", "b_low", "w_dtype", "scale_dtype", "symmetric")]


class CacheStats(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("msb_hit", "msb_miss", "lsb_hit", "lsb_miss")]


class SystemSpec(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("flash_gbit_s", "dram_gbit_s", "xpu_tops", "flash_pj_bit", "dram_pj_bit",
                                          "xpu_tops_w")]


class Cost(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("flash_bits", "dram_bits", "ops", "energy_j", "latency_s", "miss_rate_high")]


_lib = None

EXPORTS = [
    "smoe_workspace_bytes", "smoe_ctx_create", "smoe_ctx_destroy", "smoe_strerror", "smoe_last_hip_error", "smoe_ctx_timing",
    "smoe_ctx_timing_read", "smoe_stream_read", "smoe_ctx_single_launch", "smoe_ctx_single_launch_status",
    "smoe_bank_bytes", "smoe_bank_create", "smoe_bank_destroy", "smoe_quantize_slice", "smoe_export_codes",
    "smoe_route", "smoe_expert_ffn", "smoe_decode_layer", "smoe_decode_layer_multi", "smoe_static_scratch_bytes", "smoe_decode_layer_static",
    "smoe_prefill_bytes", "smoe_prefill_tiles", "smoe_prefill_histogram", "smoe_topn_slices",
    "smoe_cache_create", "smoe_cache_destroy", "smoe_cache_init_order", "smoe_cache_snapshot",
    "smoe_cache_access", "smoe_cache_snapshot_all", "smoe_cache_access_all", "smoe_cache_stats_get", "smoe_cache_order",
    "smoe_system_spec_paper", "smoe_cost_model",
    "smoe_route_scores", "smoe_residual_norm", "smoe_mx_quantize", "smoe_mx_dequantize", "smoe_mx_product_bytes", "smoe_mx_product",
    "smoe_mx_matvec",
]


# Argument types of the calls a decode or prefill loop makes (p pointer or handle, i int, l long long, f float, z size_t): with
# them ctypes converts plain numbers and addresses itself, which costs a third of building an object per argument (a
# one-token step of a tiny layer is as long as its host work).
_SIGNATURES = {
    "smoe_quantize_slice": "ppiippp",
    "smoe_route": "piiiippippifppp",
    "smoe_expert_ffn": "ppppiipppfpipp",
    "smoe_decode_layer": "ppppiipppifpfpipppp",
    "smoe_decode_layer_static": "ppppiipppifpfpipppp",
    "smoe_decode_layer_multi": "pppipiippifpfpipppp",
    "smoe_prefill_histogram": "pppipiippifpipzpppp",
    "smoe_route_scores": "piiiippipiiiipifpp",
    "smoe_residual_norm": "piiippppifppfiipp",
    "smoe_mx_quantize": "plipipp",
    "smoe_mx_dequantize": "plipppi",
    "smoe_mx_product_bytes": "iiiip",
    "smoe_mx_product": "piiippiippipiipzp",
    "smoe_mx_matvec": "piiippiipiipip",
}
_CT = {"p": C.c_void_p, "i": C.c_int, "l": C.c_longlong, "f": C.c_float, "z": C.c_size_t}


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise SmoeError("libslicemoe.so is not built: run `python -m paper_2512_12990_amd.build` "
                            "(there is no CPU fallback)")
        handle = C.CDLL(LIB_PATH)
        handle.smoe_strerror.restype = C.c_char_p
        handle.smoe_strerror.argtypes = [C.c_int]
        for name in EXPORTS:
            getattr(handle, name)            # fail loudly on a missing symbol
        for name, sig in _SIGNATURES.items():
            getattr(handle, name).argtypes = [_CT[c] for c in sig]
        _lib = handle                        # last: another host thread must not see it without its signatures
    return _lib


def _chk(rc: int, what: str, ctx=None):
    if rc != 0:
        msg = lib().smoe_strerror(rc).decode()
        if ctx is not None and rc == -5:
            msg += " (hipError %d)" % lib().smoe_last_hip_error(ctx)
        raise SmoeError("%s failed: %s [%d]" % (what, msg, rc))


def _p(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA/HIP tensors"
    return t.data_ptr()


def smoe_workspace_bytes(tokens: int, k: int, d_ff: int, n_shared: int = 0, shared_d_ff: int = 0) -> int:
    n = C.c_size_t()
    _chk(lib().smoe_workspace_bytes(C.c_int(tokens), C.c_int(k), C.c_int(d_ff), C.c_int(n_shared), C.c_int(shared_d_ff),
                                    C.byref(n)), "smoe_workspace_bytes")
    return n.value


class Ctx:
    """A library context; the torch tensor `workspace` owns the device workspace it borrows."""

    def __init__(self, device: int = 0, stream: Optional[torch.cuda.Stream] = None, workspace_bytes: int = 4 << 20):
        self.device = device
        s = stream if stream is not None else torch.cuda.current_stream(device)
        self._stream = s
        self.raw_stream, self.torch_device = s.cuda_stream, torch.device("cuda", device)
        self.workspace, base = None, 0
        if workspace_bytes:                       # 0: a context for the calls that need no workspace
            self.workspace = torch.empty(workspace_bytes + 256, dtype=torch.uint8, device="cuda:%d" % device)
            base = self.workspace.data_ptr() + (-self.workspace.data_ptr()) % 256
        self.h = C.c_void_p()
        _chk(lib().smoe_ctx_create(C.c_int(device), C.c_void_p(s.cuda_stream), C.c_void_p(base),
                                   C.c_size_t(workspace_bytes), C.byref(self.h)), "smoe_ctx_create")

    def timing(self, enable: bool):
        _chk(lib().smoe_ctx_timing(self.h, C.c_int(int(enable))), "smoe_ctx_timing")

    def timing_read(self):
        """(gateup_us_sum, down_us_sum, n_calls) since the last read; synchronises."""
        g, d, n = C.c_double(), C.c_double(), C.c_int()
        _chk(lib().smoe_ctx_timing_read(self.h, C.byref(g), C.byref(d), C.byref(n)), "smoe_ctx_timing_read", self.h)
        return g.value, d.value, n.value

    def single_launch(self, enable: bool, spin_limit: int = 0):
        """One kernel launch per decode call where the case fits (see smoe_ctx_single_launch)."""
        _chk(lib().smoe_ctx_single_launch(self.h, C.c_int(int(enable)), C.c_int(spin_limit)), "smoe_ctx_single_launch", self.h)

    def single_launch_status(self):
        """(decode calls that took the single launch, work-groups that gave up waiting); synchronises."""
        n, t = C.c_longlong(), C.c_uint()
        _chk(lib().smoe_ctx_single_launch_status(self.h, C.byref(n), C.byref(t)), "smoe_ctx_single_launch_status", self.h)
        return n.value, t.value

    def close(self):
        if self.h:
            lib().smoe_ctx_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def smoe_bank_bytes(desc: BankDesc) -> int:
    n = C.c_size_t()
    _chk(lib().smoe_bank_bytes(C.byref(desc), C.byref(n)), "smoe_bank_bytes")
    return n.value


class Bank:
    """A sliced expert store; the torch tensor `store` owns the device memory."""

    def __init__(self, ctx: Ctx, n_experts, d_model, d_ff, group, w_dtype="f32", scale_dtype="f32", b_high=8, b_low=4,
                 symmetric=False):
        self.ctx = ctx
        self.desc = BankDesc(n_experts, d_model, d_ff, group, b_high, b_low, _DT[w_dtype], _DT[scale_dtype], int(symmetric))
        self.nbytes = smoe_bank_bytes(self.desc)
        self.store = torch.empty(self.nbytes + 256, dtype=torch.uint8, device="cuda:%d" % ctx.device)
        off = (-self.store.data_ptr()) % 256
        self._base = self.store.data_ptr() + off
        self.h = C.c_void_p()
        _chk(lib().smoe_bank_create(ctx.h, C.byref(self.desc), C.c_void_p(self._base), C.c_size_t(self.nbytes),
                                    C.byref(self.h)), "smoe_bank_create", ctx.h)

    def close(self):
        if self.h:
            lib().smoe_bank_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def smoe_quantize_slice(ctx: Ctx, bank: Bank, e0: int, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor):
    """w_gate/w_up [n, d_ff, d_model], w_down [n, d_model, d_ff] on the device, dtype = bank w_dtype."""
    n = w_gate.shape[0]
    d, f = bank.desc.d_model, bank.desc.d_ff
    assert tuple(w_gate.shape) == (n, f, d) and tuple(w_up.shape) == (n, f, d) and tuple(w_down.shape) == (n, d, f)
    want = torch.float32 if bank.desc.w_dtype == F32 else torch.bfloat16
    assert w_gate.dtype == want and w_up.dtype == want and w_down.dtype == want
    _chk(lib().smoe_quantize_slice(ctx.h, bank.h, e0, n, _p(w_gate), _p(w_up), _p(w_down)),
         "smoe_quantize_slice", ctx.h)


def smoe_export_codes(ctx: Ctx, bank: Bank, expert: int, matrix: int):
    """Returns dict(q, msb, lsb [N,K] uint8; zp [N,ng] uint8; scale [N,ng] fp32) as numpy arrays."""
    d, f, G = bank.desc.d_model, bank.desc.d_ff, bank.desc.group
    N, K = (d, f) if matrix == 2 else (f, d)
    ng = -(-K // G)
    out = dict(q=np.empty((N, K), np.uint8), msb=np.empty((N, K), np.uint8), lsb=np.empty((N, K), np.uint8),
               zp=np.empty((N, ng), np.uint8), scale=np.empty((N, ng), np.float32))
    ptr = lambda a: a.ctypes.data_as(C.c_void_p)
    _chk(lib().smoe_export_codes(ctx.h, bank.h, C.c_int(expert), C.c_int(matrix), ptr(out["q"]), ptr(out["msb"]),
                                 ptr(out["lsb"]), ptr(out["zp"]), ptr(out["scale"])), "smoe_export_codes", ctx.h)
    return out


def smoe_route(ctx: Ctx, k: int, logits: Optional[torch.Tensor] = None, x: Optional[torch.Tensor] = None,
               w_router: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, norm_topk: bool = False,
               routed_scale: float = 1.0, want_logits: bool = False):
    dev = "cuda:%d" % ctx.device
    if logits is not None:
        T, E = logits.shape
        d = 0
        act = F32
    else:
        T, d = x.shape
        E = w_router.shape[0]
        act = _DT[x.dtype]
    idx = torch.empty((T, k), dtype=torch.int32, device=dev)
    w = torch.empty((T, k), dtype=torch.float32, device=dev)
    zout = torch.empty((T, E), dtype=torch.float32, device=dev) if want_logits else None
    _chk(lib().smoe_route(ctx.h, T, E, k, d, _p(logits), _p(x), act,
                          _p(w_router), _p(bias), int(norm_topk), routed_scale, _p(zout),
                          _p(idx), _p(w)), "smoe_route", ctx.h)
    return (idx, w, zout) if want_logits else (idx, w)


def smoe_expert_ffn(ctx: Ctx, routed: Optional[Bank], shared: Optional[Bank], x: torch.Tensor, idx, w, slice_mask,
                    tau_head: float = 0.0, shared_gate_w=None, add_residual: bool = False, y=None, prec_out=None):
    k = 0 if idx is None else idx.numel()
    if y is None:
        y = torch.empty_like(x)
    _chk(lib().smoe_expert_ffn(ctx.h, routed.h if routed else None, shared.h if shared else None, _p(x),
                               _DT[x.dtype], k, _p(idx), _p(w), _p(slice_mask),
                               tau_head, _p(shared_gate_w), int(add_residual), _p(y),
                               _p(prec_out)), "smoe_expert_ffn", ctx.h)
    return y


def smoe_decode_layer(ctx: Ctx, routed: Bank, shared: Optional[Bank], x: torch.Tensor, k: int, logits=None,
                      w_router=None, bias=None, norm_topk: bool = False, routed_scale: float = 1.0, slice_mask=None,
                      tau_head: float = 0.0, shared_gate_w=None, add_residual: bool = False, y=None, idx_out=None,
                      w_out=None, prec_out=None):
    if y is None:
        y = torch.empty_like(x)
    _chk(lib().smoe_decode_layer(ctx.h, routed.h, shared.h if shared else None, _p(x), _DT[x.dtype],
                                 k, _p(logits), _p(w_router), _p(bias), int(norm_topk),
                                 routed_scale, _p(slice_mask), tau_head, _p(shared_gate_w),
                                 int(add_residual), _p(y), _p(idx_out), _p(w_out), _p(prec_out)),
         "smoe_decode_layer", ctx.h)
    return y


def smoe_static_scratch_bytes() -> int:
    n = C.c_size_t()
    _chk(lib().smoe_static_scratch_bytes(C.byref(n)), "smoe_static_scratch_bytes")
    return n.value


def smoe_decode_layer_static(ctx: Ctx, routed: Bank, shared: Optional[Bank], x: torch.Tensor, k: int, y: torch.Tensor,
                             logits=None, w_router=None, bias=None, norm_topk: bool = False, routed_scale: float = 1.0,
                             slice_mask=None, tau_head: float = 0.0, shared_gate_w=None, add_residual: bool = False,
                             idx_out=None, w_out=None, prec_out=None):
    """smoe_decode_layer over the library's static workspace; the caller passes every buffer (y included)."""
    _chk(lib().smoe_decode_layer_static(ctx.h, routed.h, shared.h if shared else None, _p(x), _DT[x.dtype],
                                        k, _p(logits), _p(w_router), _p(bias), int(norm_topk),
                                        routed_scale, _p(slice_mask), tau_head, _p(shared_gate_w),
                                        int(add_residual), _p(y), _p(idx_out), _p(w_out), _p(prec_out)),
         "smoe_decode_layer_static", ctx.h)
    return y


def smoe_decode_layer_multi(ctx: Ctx, routed: Bank, shared: Optional[Bank], x: torch.Tensor, k: int, logits: torch.Tensor,
                            bias=None, norm_topk: bool = False, routed_scale: float = 1.0, slice_mask=None,
                            tau_head: float = 0.0, shared_gate_w=None, add_residual: bool = False, y=None, idx_out=None,
                            w_out=None, prec_out=None):
    T = x.shape[0]
    if y is None:
        y = torch.empty_like(x)
    _chk(lib().smoe_decode_layer_multi(ctx.h, routed.h, shared.h if shared else None, T, _p(x),
                                       _DT[x.dtype], k, _p(logits), _p(bias), int(norm_topk),
                                       routed_scale, _p(slice_mask), tau_head, _p(shared_gate_w),
                                       int(add_residual), _p(y), _p(idx_out), _p(w_out), _p(prec_out)),
         "smoe_decode_layer_multi", ctx.h)
    return y


def smoe_prefill_bytes(T, E, k, d_model, d_ff, shared_d_ff=0) -> int:
    n = C.c_size_t()
    _chk(lib().smoe_prefill_bytes(C.c_int(T), C.c_int(E), C.c_int(k), C.c_int(d_model), C.c_int(d_ff),
                                  C.c_int(shared_d_ff), C.byref(n)), "smoe_prefill_bytes")
    return n.value


def smoe_prefill_tiles(routed: BankDesc, shared: Optional[BankDesc], T: int, k: int, n_cu: int):
    """(token rows of the tallest tile of the routed experts, of the shared experts, shared tiles in the routed launches)"""
    r, s, j = C.c_int(), C.c_int(), C.c_int()
    _chk(lib().smoe_prefill_tiles(C.byref(routed), C.byref(shared) if shared is not None else None, C.c_int(T), C.c_int(k), C.c_int(n_cu),
                                  C.byref(r), C.byref(s), C.byref(j)), "smoe_prefill_tiles")
    return r.value, s.value, bool(j.value)


def smoe_prefill_histogram(ctx: Ctx, routed: Bank, shared: Optional[Bank], x: torch.Tensor, k: int, logits=None,
                           w_router=None, norm_topk=False, routed_scale=1.0, shared_gate_w=None, add_residual=False,
                           scratch: Optional[torch.Tensor] = None):
    T, d = x.shape
    E = routed.desc.n_experts
    dev = x.device
    need = smoe_prefill_bytes(T, E, k, d, routed.desc.d_ff, shared.desc.d_ff if shared else 0)
    if scratch is None:
        scratch = torch.empty(need, dtype=torch.uint8, device=dev)
    y = torch.empty_like(x)
    idx = torch.empty((T, k), dtype=torch.int32, device=dev)
    w = torch.empty((T, k), dtype=torch.float32, device=dev)
    hist = torch.empty((E,), dtype=torch.int32, device=dev)     # bit pattern of uint32 counts
    _chk(lib().smoe_prefill_histogram(ctx.h, routed.h, shared.h if shared else None, T, _p(x),
                                      _DT[x.dtype], k, _p(logits), _p(w_router),
                                      int(norm_topk), routed_scale, _p(shared_gate_w),
                                      int(add_residual), _p(scratch), scratch.numel(), _p(y),
                                      _p(idx), _p(w), _p(hist)), "smoe_prefill_histogram", ctx.h)
    return y, idx, w, hist


# ---- scores, norms and microscaled 4-bit floats ---------------------------------------------------
SCORES = {"softmax": 0, "sigmoid": 1}
GROUP_SCORES = {"max": 0, "top2": 1}


_ACTS = {torch.float32, torch.bfloat16}
_F32, _BF16, _I32, _U8 = {torch.float32}, {torch.bfloat16}, {torch.int32}, {torch.uint8}
_ONE = {torch.float32: _F32, torch.bfloat16: _BF16}
# the current stream's address; the public call, which builds an object, where torch (without GPU support) lacks the shorter one
_stream_now = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_empty = torch.empty


def _arg(ok: bool, what: str):
    if not ok:
        raise SmoeError("invalid argument: " + what)


def _t(ctx: Ctx, name: str, t: torch.Tensor, dtypes, shape=None) -> int:
    """Address of a tensor after the checks that the C entry cannot make."""
    if t.dtype in dtypes and (shape is None or t.shape == shape) and t.get_device() == ctx.device and t.is_contiguous():
        return t.data_ptr()
    if t.dtype not in dtypes:
        raise SmoeError("%s: dtype %s" % (name, t.dtype))
    if shape is not None and t.shape != shape:
        raise SmoeError("%s: shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    raise SmoeError("%s: must be contiguous on device %d of the context" % (name, ctx.device))


def _tensors(values):
    for v in values:
        if isinstance(v, torch.Tensor):
            yield v
        elif isinstance(v, (tuple, list)):
            yield from _tensors(v)


def _on_stream(f):
    """Runs a call with the context's stream as torch's current one, so that what it allocates belongs to that stream.  Where the caller's is another,
    the tensors that the call uses are kept from reuse until its work on the context's stream is done, and what it returns until
    the caller's work on its own stream is; the order of the two streams' work is the caller's."""
    @functools.wraps(f)
    def call(ctx, *args, **kw):
        if _stream_now(ctx.device) == ctx.raw_stream:
            return f(ctx, *args, **kw)
        caller = torch.cuda.current_stream(ctx.device)
        for t in _tensors((args, tuple(kw.values()))):
            if t.is_cuda:
                t.record_stream(ctx._stream)
        with torch.cuda.stream(ctx._stream):
            out = f(ctx, *args, **kw)
        for t in _tensors((out,)):
            t.record_stream(caller)
        return out
    return call


@_on_stream
def smoe_route_scores(ctx: Ctx, k: int, logits: Optional[torch.Tensor] = None, x: Optional[torch.Tensor] = None,
                      w_router: Optional[torch.Tensor] = None, score: str = "softmax", n_group: int = 1, topk_group: int = 1,
                      group_score: str = "max", bias: Optional[torch.Tensor] = None, norm_topk: bool = False, routed_scale: float = 1.0):
    """(idx int32 [T, k], w float32 [T, k]); logits float32 [T, E], or x [T, d] and w_router float32 [E, d]."""
    if score not in SCORES or group_score not in GROUP_SCORES:
        raise SmoeError("invalid argument: score %r, group_score %r" % (score, group_score))
    if logits is not None:
        _arg(logits.dim() == 2, "logits [T, E]")
        T, E = logits.shape
        d, act, lp, xp, wp = 0, F32, _t(ctx, "logits", logits, _F32), None, None
    else:
        _arg(x is not None and w_router is not None and x.dim() == 2 and w_router.dim() == 2, "logits, or x [T, d] and w_router [E, d]")
        (T, d), E = x.shape, w_router.shape[0]
        lp, xp, wp = None, _t(ctx, "x", x, _ACTS), _t(ctx, "w_router", w_router, _F32, (E, d))
        act = _DT[x.dtype]
    bp = None if bias is None else _t(ctx, "bias", bias, _F32, (E,))
    _arg(k > 0, "k")
    like = x if logits is None else logits
    idx, w = like.new_empty((T, k), dtype=torch.int32), like.new_empty((T, k), dtype=torch.float32)
    rc = lib().smoe_route_scores(ctx.h, T, E, k, d, lp, xp, act, wp, SCORES[score], n_group, topk_group, GROUP_SCORES[group_score], bp,
                                 norm_topk, routed_scale, idx.data_ptr(), w.data_ptr())
    if rc:
        _chk(rc, "smoe_route_scores", ctx.h)
    return idx, w


@_on_stream
def smoe_residual_norm(ctx: Ctx, res: Optional[torch.Tensor], y: Optional[torch.Tensor] = None, slot_w: Optional[torch.Tensor] = None,
                       post_w: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None, scale: float = 1.0,
                       pre_w: Optional[torch.Tensor] = None, eps: float = 1e-6, res_out: Optional[torch.Tensor] = None, want_x: bool = True,
                       act_dtype: Optional[torch.dtype] = None):
    """(res_out [T, d], x [T, d] or None).  y [T, k, d] or [T, d]; without y the act dtype is pre_w's or `act_dtype`; without
    res the residual has the act dtype.  res_out may be res (in place)."""
    if y is not None:
        ys = y.shape
        _arg(len(ys) in (2, 3), "y [T, k, d] or [T, d]")
        T, d, k, act = ys[0], ys[-1], ys[1] if len(ys) == 3 else 1, y.dtype
    else:
        _arg(res is not None and res.dim() == 2, "y, or res [T, d]")
        T, d = res.shape
        k, act = 0, act_dtype or (pre_w.dtype if pre_w is not None else res.dtype)
    if act not in _ACTS or (act_dtype is not None and act_dtype != act):
        raise SmoeError("invalid argument: act dtype %s" % act)
    acts = _ONE[act]
    yp = None if y is None else _t(ctx, "y", y, acts)
    rp = None if res is None else _t(ctx, "res", res, _ACTS, (T, d))
    sp = None if slot_w is None else _t(ctx, "slot_w", slot_w, _F32, (T, k))
    op = None if post_w is None else _t(ctx, "post_w", post_w, acts, (d,))
    pp = None if pre_w is None else _t(ctx, "pre_w", pre_w, acts, (d,))
    gr = gate is not None and gate.dim() == 2
    gp = None if gate is None else _t(ctx, "gate", gate, acts, (T, d) if gr else (d,))
    rd = act if res is None else res.dtype
    if res_out is None:
        res_out = _empty((T, d), dtype=rd, device=ctx.torch_device) if res is None else torch.empty_like(res)
        ro = res_out.data_ptr()
    else:
        rd = res_out.dtype if res is None else rd
        ro = _t(ctx, "res_out", res_out, _ACTS if res is None else _ONE[rd], (T, d))
    x, xo = None, None
    if want_x:
        x = torch.empty_like(res_out) if rd == act else res_out.new_empty((T, d), dtype=act)
        xo = x.data_ptr()
    rc = lib().smoe_residual_norm(ctx.h, T, d, k, yp, sp, op, gp, gr, scale, rp, pp, eps, _DT[act], _DT[rd], ro, xo)
    if rc:
        _chk(rc, "smoe_residual_norm", ctx.h)
    return res_out, x


class Mx(NamedTuple):
    """Microscaled 4-bit floats [..., K]: codes uint8 [..., K/2], scales uint8 [..., K/32] (see slicemoe.h)."""
    codes: torch.Tensor
    scales: torch.Tensor


def _mx(ctx: Ctx, name: str, m: Mx):
    """(codes address, scales address, shape of the codes)"""
    c, s = m
    cp, sp = _t(ctx, name + ".codes", c, _U8), _t(ctx, name + ".scales", s, _U8)
    cs, ss = c.shape, s.shape
    if len(cs) < 2 or cs[:-1] != ss[:-1] or cs[-1] != 16 * ss[-1] or not cs[-1]:
        raise SmoeError("%s: codes %s and scales %s do not belong together" % (name, tuple(cs), tuple(ss)))
    return cp, sp, cs


@_on_stream
def smoe_mx_quantize(ctx: Ctx, src: torch.Tensor, out: Optional[Mx] = None) -> Mx:
    """src [..., K] float32 or bfloat16, at least two-dimensional."""
    _arg(src.dim() >= 2 and src.shape[-1] % 32 == 0 and src.shape[-1] > 0, "src [..., K], K a multiple of 32")
    *lead, K = src.shape
    sp = _t(ctx, "src", src, _ACTS)
    if out is None:
        out = Mx(src.new_empty((*lead, K // 2), dtype=torch.uint8), src.new_empty((*lead, K // 32), dtype=torch.uint8))
        cp, ep = out[0].data_ptr(), out[1].data_ptr()
    else:
        cp, ep, shape = _mx(ctx, "out", out)
        _arg(shape == (*lead, K // 2), "out: shape")
    rc = lib().smoe_mx_quantize(ctx.h, src.numel() // K, K, sp, _DT[src.dtype], cp, ep)
    if rc:
        _chk(rc, "smoe_mx_quantize", ctx.h)
    return out


@_on_stream
def smoe_mx_dequantize(ctx: Ctx, m: Mx, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    cp, sp, (*lead, half) = _mx(ctx, "m", m)
    _arg(dtype in _ACTS, "dtype")
    out = m[0].new_empty((*lead, 2 * half), dtype=dtype)
    rc = lib().smoe_mx_dequantize(ctx.h, out.numel() // (2 * half), 2 * half, cp, sp, out.data_ptr(), _DT[dtype])
    if rc:
        _chk(rc, "smoe_mx_dequantize", ctx.h)
    return out


@functools.lru_cache(maxsize=4096)
def smoe_mx_product_bytes(T: int, k: int, E: int, N: int) -> int:
    n = C.c_size_t()
    _chk(lib().smoe_mx_product_bytes(T, k, E, N, C.byref(n)), "smoe_mx_product_bytes")
    return n.value


def _mx_args(ctx: Ctx, w: Mx, x_shape, idx: Optional[torch.Tensor]):
    """(codes, scales, E, N, T, k, x_slots, idx address) of a product; x_shape [T, K / 2] or [T, k, K / 2], w [E, N, K] or [N, K]."""
    wc, ws, shape = _mx(ctx, "w", w)
    nx = len(x_shape)
    if len(shape) not in (2, 3) or nx not in (2, 3) or shape[-1] != x_shape[-1]:
        raise SmoeError("invalid argument: w [E, N, K] or [N, K], x [T, K] or [T, k, K]")
    E, N = (1, shape[0]) if len(shape) == 2 else shape[:2]
    T = x_shape[0]
    if idx is None:
        _arg(nx == 2 or x_shape[1] == 1, "x [T, K] without idx")
        return wc, ws, E, N, T, 1, nx == 3, None
    _arg(idx.dim() == 2, "idx [T, k]")
    k = idx.shape[1]
    _arg(nx == 2 or x_shape[1] == k, "x [T, k, K] with the k of idx")
    return wc, ws, E, N, T, k, nx == 3, _t(ctx, "idx", idx, _I32, (T, k))


@_on_stream
def smoe_mx_product(ctx: Ctx, w: Mx, x: Mx, idx: Optional[torch.Tensor] = None, swiglu: bool = False, out_dtype: torch.dtype = torch.bfloat16,
                    scratch: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [T, k, N] (N / 2 with swiglu); w [E, N, K] or [N, K], x [T, K] or [T, k, K], idx int32 [T, k] or None (one matrix, k = 1)."""
    xc, xs, x_shape = _mx(ctx, "x", x)
    wc, ws, E, N, T, k, slots, ip = _mx_args(ctx, w, x_shape, idx)
    if out_dtype not in _ACTS:
        raise SmoeError("invalid argument: out_dtype %s" % out_dtype)
    shape = (T, k, N // 2 if swiglu else N)
    sp, size = None, 0
    if scratch is not None:
        sp, size = _t(ctx, "scratch", scratch, _U8), scratch.numel()
    elif ip is not None and T:
        size = smoe_mx_product_bytes(T, k, E, N)
        if size:
            scratch = x[0].new_empty(size)
            sp = scratch.data_ptr()
    if y is None:
        y = x[0].new_empty(shape, dtype=out_dtype)
        yp = y.data_ptr()
    else:
        yp = _t(ctx, "y", y, _ONE[out_dtype], shape)
    rc = lib().smoe_mx_product(ctx.h, E, N, 2 * x_shape[-1], wc, ws, T, k, xc, xs, slots, ip, swiglu, _DT[out_dtype], sp, size, yp)
    if rc:
        _chk(rc, "smoe_mx_product", ctx.h)
    return y


@_on_stream
def smoe_mx_matvec(ctx: Ctx, w: Mx, x: torch.Tensor, idx: Optional[torch.Tensor] = None, swiglu: bool = False,
                   y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [T, k, N] (N / 2 with swiglu) of x's dtype, T <= 16; w, idx as in smoe_mx_product, x [T, K] or [T, k, K]."""
    xp = _t(ctx, "x", x, _ACTS)
    xs = x.shape
    _arg(len(xs) > 1, "x [T, K] or [T, k, K]")
    wc, ws, E, N, T, k, slots, ip = _mx_args(ctx, w, xs[:-1] + (xs[-1] // 2,), idx)
    shape = (T, k, N // 2 if swiglu else N)
    if y is None:
        y = x.new_empty(shape)
        yp = y.data_ptr()
    else:
        yp = _t(ctx, "y", y, _ONE[x.dtype], shape)
    rc = lib().smoe_mx_matvec(ctx.h, E, N, xs[-1], wc, ws, T, k, xp, _DT[x.dtype], slots, ip, swiglu, yp)
    if rc:
        _chk(rc, "smoe_mx_matvec", ctx.h)
    return y


# ---- host-only calls ----------------------------------------------------------------------------
def smoe_topn_slices(hist: np.ndarray, n: int) -> np.ndarray:
    hist = np.ascontiguousarray(hist, dtype=np.uint32)
    L, E = hist.shape
    out = np.empty(max(1, min(n, 2 * L * E)), np.uint32)
    cnt = C.c_int()
    _chk(lib().smoe_topn_slices(hist.ctypes.data_as(C.c_void_p), C.c_int(L), C.c_int(E), C.c_int(n),
                                out.ctypes.data_as(C.c_void_p), C.byref(cnt)), "smoe_topn_slices")
    return out[: cnt.value].copy()


def smoe_system_spec_paper() -> SystemSpec:
    spec = SystemSpec()
    _chk(lib().smoe_system_spec_paper(C.byref(spec)), "smoe_system_spec_paper")
    return spec


def smoe_cost_model(spec: SystemSpec, stats: dict, msb_slice_bytes: int, lsb_slice_bytes: int, ops: float) -> dict:
    st = CacheStats(stats["msb_hit"], stats["msb_miss"], stats["lsb_hit"], stats["lsb_miss"])
    out = Cost()
    _chk(lib().smoe_cost_model(C.byref(spec), C.byref(st), C.c_uint64(msb_slice_bytes), C.c_uint64(lsb_slice_bytes),
                               C.c_double(ops), C.byref(out)), "smoe_cost_model")
    return {n: getattr(out, n) for n, _ in Cost._fields_}


class Cache:
    def __init__(self, L: int, E: int, capacity: int):
        self.L, self.E, self.cap = L, E, capacity
        self.h = C.c_void_p()
        _chk(lib().smoe_cache_create(C.c_int(L), C.c_int(E), C.c_int(capacity), C.byref(self.h)), "smoe_cache_create")

    def init_order(self, slice_ids):
        a = np.ascontiguousarray(slice_ids, dtype=np.uint32)
        _chk(lib().smoe_cache_init_order(self.h, a.ctypes.data_as(C.c_void_p), C.c_int(a.size)), "smoe_cache_init_order")

    def snapshot(self, layer: int, beta: float):
        mask = np.empty(self.E, np.uint8)
        bias = np.empty(self.E, np.float32)
        _chk(lib().smoe_cache_snapshot(self.h, C.c_int(layer), C.c_float(beta), mask.ctypes.data_as(C.c_void_p),
                                       bias.ctypes.data_as(C.c_void_p)), "smoe_cache_snapshot")
        return mask, bias

    def access(self, layer: int, idx, want_high):
        i = np.ascontiguousarray(idx, dtype=np.int32)
        wh = np.ascontiguousarray(want_high, dtype=np.uint8)
        _chk(lib().smoe_cache_access(self.h, C.c_int(layer), C.c_int(i.size), i.ctypes.data_as(C.c_void_p),
                                     wh.ctypes.data_as(C.c_void_p)), "smoe_cache_access")

    def snapshot_all(self, beta: float, mask_out: np.ndarray, bias_out: Optional[np.ndarray] = None):
        """Masks (uint8 [L, E]) and routing bias (float32 [L, E]) of all layers into the caller's arrays."""
        assert mask_out.dtype == np.uint8 and mask_out.flags.c_contiguous and mask_out.size == self.L * self.E
        bp = None
        if bias_out is not None:
            assert bias_out.dtype == np.float32 and bias_out.flags.c_contiguous and bias_out.size == self.L * self.E
            bp = bias_out.ctypes.data_as(C.c_void_p)
        _chk(lib().smoe_cache_snapshot_all(self.h, C.c_float(beta), mask_out.ctypes.data_as(C.c_void_p), bp),
             "smoe_cache_snapshot_all")

    def access_all(self, idx: np.ndarray, k: int, want_high: Optional[np.ndarray] = None):
        """One token's selections in all layers: idx int32 [L, stride >= k] (C-contiguous), want_high uint8 [L, k]."""
        assert idx.dtype == np.int32 and idx.flags.c_contiguous and idx.shape[0] == self.L and idx.shape[1] >= k
        wp = None
        if want_high is not None:
            wh = np.ascontiguousarray(want_high, dtype=np.uint8)
            assert wh.size == self.L * k
            wp = wh.ctypes.data_as(C.c_void_p)
        _chk(lib().smoe_cache_access_all(self.h, C.c_int(k), idx.ctypes.data_as(C.c_void_p), C.c_int(idx.shape[1]), wp),
             "smoe_cache_access_all")

    def stats(self) -> dict:
        s = CacheStats()
        _chk(lib().smoe_cache_stats_get(self.h, C.byref(s)), "smoe_cache_stats_get")
        return dict(msb_hit=s.msb_hit, msb_miss=s.msb_miss, lsb_hit=s.lsb_hit, lsb_miss=s.lsb_miss)

    def order(self) -> list:
        out = np.empty(max(1, self.cap), np.uint32)
        n = C.c_int()
        _chk(lib().smoe_cache_order(self.h, out.ctypes.data_as(C.c_void_p), C.c_int(self.cap), C.byref(n)),
             "smoe_cache_order")
        return out[: n.value].tolist()

    def close(self):
        if self.h:
            lib().smoe_cache_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
