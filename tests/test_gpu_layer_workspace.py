"""Layers in a small workspace (GT_FLAG_SMALL_WORKSPACE), which takes the passes of the largest products at small sizes: chunks whose residues are not kept, blocks of
columns and rows, against the oracle bit for bit."""
import numpy as np
import pytest

import plain_layers as pl
from test_gpu_layers import shared
from test_gpu_parity import mods, same, same_stats  # noqa: F401

pytestmark = pytest.mark.gpu

# rows, din, dout, all in several blocks of rows: blocks of columns; more chunks than are kept; four kept, then one; chunks and columns, odd; all residues kept
FORWARD = [(600, 130, 600), (300, 8300, 130), (200, 16500, 60), (261, 8200, 259), (500, 4100, 20)]
# the gradient of the weights over several chunks of rows
BACKWARD = [(9000, 140, 260), (4500, 20, 30), (700, 300, 257)]


def small(mods, seed):
    Oracle, gtree = mods
    return Oracle(seed), gtree.GTree(seed, flags=gtree.GT_FLAG_SMALL_WORKSPACE)


@pytest.mark.parametrize("rows,din,dout", FORWARD)
@pytest.mark.parametrize("relu,bias,res", [(False, False, True), (True, True, False)])
def test_dense_forward(mods, seed, rows, din, dout, relu, bias, res):
    o, g = small(mods, seed)
    rng = np.random.default_rng(rows + din)
    x, W = pl.fixed(rng, 16, 1.0, rows, din), pl.fixed(rng, 16, din ** -0.5, din, dout)
    b, r = (pl.fixed(rng, 16, 1.0, *s) if on else None for s, on in (((dout,), bias), ((rows, dout), res)))
    (xo, xg), (Wo, Wg), (bo, bg), (ro, rg) = (shared(o, g, a) for a in (x, W, b, r))
    layer = g.dense_create(Wg, din, dout, b=bg)
    for call in range(2):
        print("dense", rows, din, dout, relu, call, flush=True)
        yo, go = o.dense_forward(xo, Wo, rows, din, dout, b=bo, relu=relu, residual=ro)
        got = g.dense_forward(layer, xg, rows, relu=relu, residual=rg, want_gate=relu)
        same(got[0] if relu else got, yo, "y")
        if relu:
            same(got[1], go, "gate")
        same_stats(o, g)
    layer.close(); g.close()


@pytest.mark.parametrize("rows,din,dout", BACKWARD)
def test_dense_backward(mods, seed, rows, din, dout):
    o, g = small(mods, seed)
    rng = np.random.default_rng(rows)
    x, W, dy = pl.fixed(rng, 16, 1.0, rows, din), pl.fixed(rng, 16, 1.0, din, dout), pl.fixed(rng, 16, 0.1, rows, dout)
    (xo, xg), (Wo, Wg), (do, dg) = (shared(o, g, a) for a in (x, W, dy))
    layer = g.dense_create(Wg, din, dout)
    for call in range(2):
        print("backward", rows, din, dout, call, flush=True)
        for name, a, b in zip(("dx", "dW", "db"), g.dense_backward(layer, xg, dg, rows), o.dense_backward(xo, Wo, do, rows, din, dout)):
            same(a, b, name)
        same_stats(o, g)
    layer.close(); g.close()


def test_mixture_of_many_rows(mods, seed):
    o, g = small(mods, seed)
    rows, d, ff, E = 400, 130, 300, 4
    rng = np.random.default_rng(rows)
    x, Wr, W1, W2 = (shared(o, g, pl.fixed(rng, 16, 0.3, *s)) for s in ((rows, d), (d, E), (E, d, ff), (E, ff, d)))
    moe = g.moe_create(Wr[1], W1[1], W2[1], d, ff, E, 1, rows)
    for call in range(2):
        same(g.moe_forward(moe, x[1], rows), o.moe_forward(x[0], Wr[0], W1[0], W2[0], rows, d, ff, E, 1), "y")
        same_stats(o, g)
    moe.close(); g.close()
