"""Sizes of kernel launches at the ends of the documented ranges, on the CPU: the HIP calls that a launch makes are replaced by ones that
record it.  A launch takes fewer than 2^32 threads along each axis, at most 1024 in a work-group and at most 160 KB of LDS."""
import json
import os
import subprocess
import sys

import pytest

import block_cases
from paper_2512_12990_amd import binding as B

SHIM = r"""
#include <stddef.h>
#include <stdint.h>
typedef struct { uint32_t x, y, z; } dim3;
static dim3 g_grid, g_block;
static size_t g_lds;
static uint32_t g_log[64][7];
static int g_n;
int launches(uint32_t* out) { int n = g_n; for (int i = 0; i < n; i++) for (int j = 0; j < 7; j++) out[7 * i + j] = g_log[i][j]; g_n = 0; return n; }
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, void* s) { g_grid = g; g_block = b; g_lds = lds; return 0; }
int __hipPopCallConfiguration(dim3* g, dim3* b, size_t* lds, void** s) { *g = g_grid; *b = g_block; *lds = g_lds; *s = 0; return 0; }
int hipLaunchKernel(const void* f, dim3 g, dim3 b, void** args, size_t lds, void* s) {
  if (g_n < 64) { uint32_t v[7] = {g.x, g.y, g.z, b.x, b.y, b.z, (uint32_t)lds}; for (int j = 0; j < 7; j++) g_log[g_n][j] = v[j]; g_n++; }
  return 0;
}
int hipGetLastError(void) { return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipSetDevice(int d) { return 0; }
int hipFuncSetAttribute(const void* f, int a, int v) { return 0; }
"""

RUN = r"""
import ctypes as C, json, sys
shim = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)              # found before the HIP runtime that the library links
lib = C.CDLL(sys.argv[2])
signatures, calls = json.loads(sys.argv[3])
ct = {"p": C.c_void_p, "i": C.c_int, "l": C.c_longlong, "f": C.c_float, "z": C.c_size_t}
ctx = C.c_void_p()
assert lib.smoe_ctx_create(0, None, None, C.c_size_t(0), C.byref(ctx)) == 0
log, out = (C.c_uint32 * 448)(), []
for name, args in calls:
    f = getattr(lib, name)
    f.argtypes = [ct[c] for c in signatures[name]]
    rc = f(ctx, *args)
    n = shim.launches(log)
    out.append((rc, [list(log[7 * i:7 * i + 7]) for i in range(n)]))
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    d = tmp_path_factory.mktemp("shim")
    src, so = str(d / "shim.c"), str(d / "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", so, src], check=True)

    def run(calls):
        arg = json.dumps(({n: B._SIGNATURES[n] for n, _ in calls}, calls))
        r = subprocess.run([sys.executable, "-c", RUN, so, os.path.abspath(B.LIB_PATH), arg], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return json.loads(r.stdout)
    return run


P = 1 << 20                      # an aligned address that no kernel gets to see
BIG = 1 << 22


def check(launches, calls):
    """Every call is accepted and its launches fit; the number of work-groups of each call's launches."""
    n = []
    for (name, args), (rc, log) in zip(calls, launches(calls)):
        assert rc == 0 and log, (name, args, rc)
        for gx, gy, gz, bx, by, bz, lds in log:
            assert max(gx * bx, gy * by, gz * bz) < 1 << 32 and min(gx, gy, gz) > 0 and bx * by * bz <= 1024 and lds <= 160 * 1024, (name, args, log)
        n.append(sum(v[0] * v[1] * v[2] for v in log))
    return n


@pytest.mark.parametrize("T", [1, 5, BIG - 1, BIG])
def test_residual_norm(launches, T):
    calls = [["smoe_residual_norm", [T, d, 0, None, None, None, None, 0, 1.0, P, None, 1e-6, act, res, 2 * P, 3 * P]]
             for d in (8, 512, 520, 2048, 2056, 4096, 4104, 8192, 8200, 16384) for act in (0, 1) for res in (0, 1)]
    for (_, args), n in zip(calls, check(launches, calls)):
        assert n * (4 if args[1] <= 512 else 1) >= T         # four rows a work-group, or one


@pytest.mark.parametrize("T", [1, 300, 600, 2047, BIG - 1, BIG])
def test_route_scores(launches, T):
    def call(E, k, d, logits, act, ng=1):
        return ["smoe_route_scores", [T, E, k, d, P if logits else None, None if logits else P, act, None if logits else P, 1, ng, ng, 1, None, 1, 1.0, P, P]]
    given = [call(E, 4, 0, True, 0, ng) for E, ng in ((4, 1), (60, 1), (63, 1), (64, 8), (128, 8), (160, 8), (200, 1), (256, 1), (256, 64))]
    for n in check(launches, given):
        assert n * 16 >= T                                   # four waves of four tokens or of one
    # widths on both sides of where 8, 4, 2 tokens and 1 still fit a work-group
    work = [call(E, 1, d, False, act) for E in (1, 64, 256) for act in (0, 1) for d in (64, 1500, 3400, 3700, 6500, 7400, 12000, 13600)]
    work += [call(E, 1, d, False, 1) for E in (1, 64, 256) for d in (14700, 24000, 27000)]
    for n in check(launches, work):
        assert n * 8 >= T


def test_mx_quantize(launches):
    calls = [[n, [rows, K, P, 0, P, P] if n == "smoe_mx_quantize" else [rows, K, P, P, P, 1]]
             for rows, K in ((1, 32), (3, 96), (1 << 29, 32), (1 << 18, 1 << 16), ((1 << 34) // 96, 96)) for n in ("smoe_mx_quantize", "smoe_mx_dequantize")]
    for (_, args), n in zip(calls, check(launches, calls)):
        assert n * 256 * 8 >= args[0] * args[1]


def test_mx_product(launches):
    calls = [["smoe_mx_product", [E, N, K, P, P, T, k, P, P, slots, P if E > 1 or k > 1 else None, 1, 0, P, 1 << 40, P]]
             for T, k, E, N, K, slots in ((1, 1, 1, 16, 32, 0), (1, 16, 256, 1 << 20, 32, 0), (BIG, 1, 1, 8192, 32, 0), (BIG, 1, 256, 8192, 32, 0), (1 << 18, 16, 256, 8192, 64, 1),
                                          (2048, 16, 256, 1 << 20, 4064, 0), (32768, 1, 1, 1 << 20, 4064, 0), (BIG, 1, 3, 16, 992, 0), (16, 1, 256, 1 << 20, 4064, 0), (100, 2, 256, 65536, 65504, 1))]
    check(launches, calls)


def test_mx_matvec(launches):
    calls = [["smoe_mx_matvec", [E, N, K, P, P, T, k, P, act, 0, P if E > 1 or k > 1 else None, 0, 2 * P]]
             for T, k, E, N, K in ((1, 1, 1, 16, 32), (16, 16, 256, 1 << 20, 4064), (16, 1, 1, 1 << 20, 4064), (1, 16, 256, 1 << 20, 32), (16, 16, 3, 65504, 65536), (5, 1, 256, 48, 65536))
             for act in (0, 1)]
    check(launches, calls)


# ---------------------------------------------------------------- which variants the GPU tests' sizes reach
def test_matvec_sizes_reach_both_forms(launches):
    def forms(cases):
        calls = [["smoe_mx_matvec", [E, N, K, P, P, T, k, P, act, 0, P if E > 1 or k > 1 else None, 0, 2 * P]] for T, k, E, N, K in cases for act in (0, 1)]
        return {log[0][3] for _, log in launches(calls)}
    assert forms(block_cases.MATVEC_FOUR_TILES) == {256} and forms(block_cases.MATVEC_ONE_TILE) == {512}


def test_product_sizes_reach_every_tile(launches):
    def forms(group, idx):
        calls = [["smoe_mx_product", [E, N, K, P, P, T, k, P, P, 0, P if idx else None, 0, 0, P, 1 << 40, P]] for pair in group for T, k, E, N, K in pair]
        return [(len(log), log[-1][3], log[-1][6]) for _, log in launches(calls)]
    # six kernels: three shapes, which threads and LDS tell apart, of two alignments; a launch more where slots are listed before
    search, listed, plain = forms(block_cases.PRODUCT_SEARCH, True), forms(block_cases.PRODUCT_LIST, True), forms(block_cases.PRODUCT_PLAIN, False)
    assert len({f[1:] for f in search}) == 6 and [f[1:] for f in listed] == [f[1:] for f in search] == [f[1:] for f in plain]
    assert {f[0] for f in search} == {1} and {f[0] for f in listed} == {2} and {f[0] for f in plain} == {1}


def test_route_sizes_reach_both_forms(launches):
    T = block_cases.ROUTE_TOKENS
    def tokens_of_a_work_group(cases):
        calls = [["smoe_route_scores", [T, E, k, 0, P, None, 0, None, 1, ng, tg, 1, None, 1, 1.0, P, P]] for E, ng, tg, k in cases]
        return {-(-T // log[0][0]) for _, log in launches(calls)}
    assert tokens_of_a_work_group(block_cases.ROUTE_PART_LANES) == {16} and tokens_of_a_work_group(block_cases.ROUTE_ODD_GROUPS) == {4}
