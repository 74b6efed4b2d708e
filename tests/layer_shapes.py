"""The rules of the layers' products and completions (csrc/gt_shape.hpp), compiled for the CPU."""
import ctypes as C
import functools
import os
import subprocess
import tempfile

from shapes import CSRC, SIMDS

SOURCE = r"""
#include "gt_shape.hpp"
extern "C" int few(u64 simds, u64 M, u64 N, u64 K) { return few_rows(simds, M, N, K, K); }
extern "C" int apart(u64 rows, u64 din, u64 dout) { return few_rows_apart(rows, din, dout); }
extern "C" void few_split(u64 simds, u64 M, u64 N, u64 K, u64 *out)
{
    const FewShape s = few_shape(simds, M, N, K);
    out[0] = s.rows; out[1] = s.ntile; out[2] = s.ngrp; out[3] = s.nsplit; out[4] = s.per;
}
extern "C" void rmm(u64 simds, u64 M, u64 N, u64 *out)
{
    const RmmShape s = rmm_shape(simds, M, N);
    out[0] = s.wm; out[1] = s.wn; out[2] = s.ntm; out[3] = s.ntn;
}
extern "C" void fin(u64 simds, u64 n, u64 *out)
{
    const FinShape s = fin_shape(simds, n);
    out[0] = s.per; out[1] = s.nbig; out[2] = s.waves;
}
extern "C" int parts_pairs(u64 simds, u64 n) { return fin_pairs(simds, n); }
extern "C" int left(u64 simds, u64 M, u64 N, u64 K)
{
    const FewShape s = few_shape(simds, M, N, K);
    return s.rows == 16 && few_left(simds, s.ntile, s.ngrp, (K + 63) / 64);
}
extern "C" u64 rows_of_pass(u64 N) { return rns_rows(N); }
"""


@functools.lru_cache(None)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        src, so = os.path.join(tmp, "layer_shapes.cpp"), os.path.join(tmp, "layer_shapes.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, "-o", so, src], check=True)
        L = C.CDLL(so)
    u64, vp = C.c_uint64, C.c_void_p
    L.few.argtypes = [u64] * 4
    L.apart.argtypes = [u64] * 3
    L.few_split.argtypes, L.few_split.restype = [u64] * 4 + [vp], None
    L.rmm.argtypes, L.rmm.restype = [u64] * 3 + [vp], None
    L.fin.argtypes, L.fin.restype = [u64, u64, vp], None
    L.parts_pairs.argtypes = [u64] * 2
    L.left.argtypes = [u64] * 4
    L.rows_of_pass.argtypes, L.rows_of_pass.restype = [u64], u64
    return L


def few(M, N, K):
    """Does a product of M rows with weights K x N take the kernel of few rows (else products by residues)?"""
    return bool(_lib().few(SIMDS, M, N, K))


def apart(rows, din, dout):
    return bool(_lib().apart(rows, din, dout))


def _array(f, n, *args):
    out = (C.c_uint64 * n)()
    f(SIMDS, *args, out)
    return tuple(out)


def few_split(M, N, K):
    return _array(_lib().few_split, 5, M, N, K)


def rmm(M, N):
    """(wm, wn, row tiles, column tiles) of a product of residues."""
    return _array(_lib().rmm, 4, M, N)


def fin(n):
    """(tiles of a first wavefront, such wavefronts, wavefronts)"""
    return _array(_lib().fin, 3, n)


def parts_pairs(n):
    """Are n parts completed by two elements a lane?"""
    return bool(_lib().parts_pairs(SIMDS, n))


def left(M, N, K):
    """Are the few rows converted by a launch of their own?"""
    return bool(_lib().left(SIMDS, M, N, K))


def rows_of_pass(N):
    return _lib().rows_of_pass(N)
