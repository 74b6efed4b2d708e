"""The rules of the gated layer and of linear attention (csrc/gt_shape.hpp), compiled for the CPU."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

from shapes import CSRC, SIMDS

SOURCE = r"""
#include "gt_shape.hpp"
extern "C" int few(u64 simds, u64 n) { return gated_few(simds, n); }
extern "C" int pairs(u64 simds, u64 chains) { return lin_pairs(simds, chains); }
extern "C" u32 per(u64 simds, u64 tiles) { return tiles_of_wave(simds, tiles); }
extern "C" void gated(u64 simds, u64 n, u64 *out)
{
    const FinShape s = gated_shape(simds, n);
    out[0] = s.per; out[1] = s.nbig; out[2] = s.waves;
}
extern "C" void pass(u64 nbh, u64 nc, u64 dk, u64 dv, int small, u64 *out)
{
    const LinPass p = lin_pass(nbh, nc, dk, dv, small ? RNS_LIMIT_SMALL : RNS_LIMIT);
    out[0] = p.nbh; out[1] = p.nch;
}
"""


@functools.lru_cache(None)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        src, so = os.path.join(tmp, "block_shapes.cpp"), os.path.join(tmp, "block_shapes.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, "-o", so, src], check=True)
        L = C.CDLL(so)
    u64, vp = C.c_uint64, C.c_void_p
    L.few.argtypes = L.pairs.argtypes = L.per.argtypes = [u64, u64]
    L.per.restype = C.c_uint32
    L.gated.argtypes, L.gated.restype = [u64, u64, vp], None
    L.pass_ = getattr(L, "pass")
    L.pass_.argtypes, L.pass_.restype = [u64] * 4 + [C.c_int, vp], None
    return L


def few(n):
    """Do n completions of a gated layer take a workgroup for 16?"""
    return bool(_lib().few(SIMDS, n))


def pairs(chains):
    """Do so many chains of states take two wavefronts each?"""
    return bool(_lib().pairs(SIMDS, chains))


def per(tiles):
    """Tiles of a wavefront."""
    return _lib().per(SIMDS, tiles)


def gated(n):
    """(tiles of a large wavefront, large wavefronts, wavefronts) of a completion of residues."""
    out = (C.c_uint64 * 3)()
    _lib().gated(SIMDS, n, out)
    return tuple(out)


def lin_pass(nbh, nc, dk, dv, small=False):
    """(heads, chunks) at a time."""
    out = (C.c_uint64 * 2)()
    _lib().pass_(nbh, nc, dk, dv, int(small), out)
    return tuple(out)
