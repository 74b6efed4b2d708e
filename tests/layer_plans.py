"""What a product by residues does at a time, and its bytes (csrc/gt_shape.hpp), compiled for the CPU."""
import collections
import ctypes as C
import functools
import os
import subprocess
import tempfile

from shapes import CSRC, SIMDS

SOURCE = r"""
#include "gt_shape.hpp"
extern "C" void plan(u64 M, u64 N, u64 K, int small, u64 *out)
{
    const RnsPlan p = rns_plan(M, N, K, small ? RNS_LIMIT_SMALL : RNS_LIMIT);
    out[0] = p.rows; out[1] = p.cols; out[2] = p.keep; out[3] = p.whole;
}
extern "C" u64 bytes(u64 simds, u64 M, u64 N, u64 K, u64 keep)
{
    const RnsSizes z = rns_sizes(simds, M, N, K);
    return z.abytes + z.bbytes + keep * z.rbytes;
}
"""
Plan = collections.namedtuple("Plan", "rows cols keep whole")


@functools.lru_cache(None)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        src, so = os.path.join(tmp, "layer_plans.cpp"), os.path.join(tmp, "layer_plans.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, "-o", so, src], check=True)
        L = C.CDLL(so)
    u64 = C.c_uint64
    L.plan.argtypes, L.plan.restype = [u64, u64, u64, C.c_int, C.c_void_p], None
    L.bytes.argtypes, L.bytes.restype = [u64] * 5, u64
    return L


def plan(M, N, K, small=False):
    out = (C.c_uint64 * 4)()
    _lib().plan(M, N, K, int(small), out)
    return Plan(*out)


def workspace(M, N, K, small=False):
    """The most bytes of residues of any part of such a product."""
    p = plan(M, N, K, small)
    sides = lambda n, step: {min(n, step), n % step or min(n, step)}  # noqa: E731
    return max(_lib().bytes(SIMDS, m, n, K, p.keep) for m in sides(M, p.rows) for n in sides(N, p.cols))
