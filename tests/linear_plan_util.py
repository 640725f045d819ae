"""The cut of the linear layers' tensor-core products (csrc/linear_plan.h, host code), compiled for the tests."""
import ctypes
import functools
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_16308_b200", "csrc")
SOURCE = """
#include "linear_plan.h"
static int put(dbs::LgPlan p, int *out) { out[0] = p.cg; out[1] = p.nt; out[2] = p.c; return 0; }
extern "C" int gemm(int sms, int64_t tokens, int64_t width, int out_cols, int64_t kb, int arrays, int aligned, int *out) {
    return put(dbs::plan_gemm(sms, tokens, width, out_cols, kb, arrays, aligned != 0), out);
}
extern "C" int weights(int sms, int64_t tokens, int64_t m, int64_t n, int products, int *out) { return put(dbs::plan_weights(sms, tokens, m, n, products), out); }
extern "C" int tiles(int *out) {
    int n = 0;
#define ONE(NT, C) out[2 * n] = NT; out[2 * n++ + 1] = C;
    LG_TILES(ONE)
    return n;
}
"""


@functools.cache
def _lib():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "plan.cpp"), os.path.join(d, "plan.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, src, "-o", so], check=True)
        lib = ctypes.CDLL(so)
    i64, i32 = ctypes.c_int64, ctypes.c_int
    lib.gemm.argtypes = [i32, i64, i64, i32, i64, i32, i32, ctypes.c_void_p]
    lib.weights.argtypes = [i32, i64, i64, i64, i32, ctypes.c_void_p]
    return lib


def _plan(f, *args):
    out = (ctypes.c_int * 3)()
    f(*args, out)
    return tuple(out)


def blocks(v):
    return -(-v // 64)


# each returns (thread blocks that work on one tile, tokens of a tile, thread blocks that share its K)
def forward(m, n, t, arrays, aligned, sms=148):
    return _plan(_lib().gemm, sms, t, m, 128, blocks(n), arrays, int(aligned))


def gated(m, n, t, arrays, aligned, sms=148):
    return _plan(_lib().gemm, sms, t, m, 64, blocks(n), arrays, int(aligned))


def gradient_of_x(m, n, t, layers, aligned, sms=148):
    return _plan(_lib().gemm, sms, t, n, 128, blocks(m) * layers, 0, int(aligned))


def gradient_of_weights(m, n, t, layers, sms=148):
    return _plan(_lib().weights, sms, t, m, n, layers)


def tiles():
    """the tiles of one thread block that are built, (tokens, thread blocks that share K)"""
    out = (ctypes.c_int * 64)()
    n = _lib().tiles(out)
    return [(out[2 * k], out[2 * k + 1]) for k in range(n)]
