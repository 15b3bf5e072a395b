"""Sizes of kernel launches at the ends of the documented ranges, on the CPU: the HIP calls that a launch makes are replaced by ones that
record it.  A launch takes fewer than 2^32 threads along each axis and at most 1024 in a work-group."""
import json
import os
import subprocess
import sys

import pytest

from paper_2512_12990_amd import binding as B

SHIM = r"""
#include <stddef.h>
#include <stdint.h>
typedef struct { uint32_t x, y, z; } dim3;
static dim3 g_grid, g_block;
static uint32_t g_log[64][6];
static int g_n;
int launches(uint32_t* out) { int n = g_n; for (int i = 0; i < n; i++) for (int j = 0; j < 6; j++) out[6 * i + j] = g_log[i][j]; g_n = 0; return n; }
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, void* s) { g_grid = g; g_block = b; return 0; }
int __hipPopCallConfiguration(dim3* g, dim3* b, size_t* lds, void** s) { *g = g_grid; *b = g_block; *lds = 0; *s = 0; return 0; }
int hipLaunchKernel(const void* f, dim3 g, dim3 b, void** args, size_t lds, void* s) {
  if (g_n < 64) { uint32_t v[6] = {g.x, g.y, g.z, b.x, b.y, b.z}; for (int j = 0; j < 6; j++) g_log[g_n][j] = v[j]; g_n++; }
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
log, out = (C.c_uint32 * 384)(), []
for name, args in calls:
    f = getattr(lib, name)
    f.argtypes = [ct[c] for c in signatures[name]]
    rc = f(ctx, *args)
    n = shim.launches(log)
    out.append((rc, [list(log[6 * i:6 * i + 6]) for i in range(n)]))
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
    """Every call is accepted and its launches fit; the number of work-groups of each call's last launch."""
    n = []
    for (name, args), (rc, log) in zip(calls, launches(calls)):
        assert rc == 0 and log, (name, args, rc)
        for gx, gy, gz, bx, by, bz in log:
            assert max(gx * bx, gy * by, gz * bz) < 1 << 32 and min(gx, gy, gz) > 0 and bx * by * bz <= 1024, (name, args, log)
        n.append(gx * gy * gz)
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
