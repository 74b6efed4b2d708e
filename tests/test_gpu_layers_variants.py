"""Layers on the GPU at the sizes that take products by residues, and backward passes both ways, against the CPU oracle bit for bit."""
import numpy as np
import pytest

import plain_layers as pl
from test_gpu_layers import check_backward, check_dense, shared
from test_gpu_parity import mods, pair, same, same_stats  # noqa: F401

pytestmark = pytest.mark.gpu

# rows, din, dout: odd sizes, a side within a tile, terms below a step and above a chunk, rows of more than a pass, all tiles of the product
RESIDUES = [(193, 1030, 260), (300, 640, 333), (1100, 130, 300), (4100, 22, 250), (1100, 1100, 40), (300, 4200, 70), (1000, 65, 1300), (16500, 3, 5),
            (200, 64, 5200), (500, 600, 300)]


@pytest.mark.parametrize("rows,din,dout", RESIDUES)
@pytest.mark.parametrize("relu,bias,res", [(False, False, True), (True, True, False)])
def test_dense_forward(mods, seed, rows, din, dout, relu, bias, res):
    check_dense(mods, seed, rows, din, dout, relu, bias, res, calls=2)


# few rows with many outputs
FEW_MANY = [(150, 64, 700), (129, 33, 641), (2, 40, 50000)]


@pytest.mark.parametrize("rows,din,dout", FEW_MANY)
@pytest.mark.parametrize("relu,bias,res", [(False, True, True), (True, True, False), (True, False, True)])
def test_few_rows_with_many_outputs(mods, seed, rows, din, dout, relu, bias, res):
    check_dense(mods, seed, rows, din, dout, relu, bias, res, calls=2)


# few rows, converted by a launch of their own
LEFT = [(180, 700, 1100), (65, 1030, 2045)]


@pytest.mark.parametrize("rows,din,dout", LEFT)
@pytest.mark.parametrize("relu,bias,res", [(False, False, True), (True, True, False)])
def test_rows_converted_ahead(mods, seed, rows, din, dout, relu, bias, res):
    check_dense(mods, seed, rows, din, dout, relu, bias, res, calls=2)


LEFT_BACKWARD = [(190, 1100, 700), (177, 1030, 1025)]


@pytest.mark.parametrize("rows,din,dout", LEFT_BACKWARD)
def test_gradient_rows_converted_ahead(mods, seed, rows, din, dout):
    check_backward(mods, seed, rows, din, dout, True, want=(True, False, True))


@pytest.mark.parametrize("f", [1, 8, 20])
@pytest.mark.parametrize("relu", [False, True])
def test_fraction_widths(mods, seed, f, relu):
    check_dense(mods, seed, 1100, 130, 300, relu, True, True, f=f, std=4.0)


@pytest.mark.parametrize("relu", [False, True])
def test_words_of_any_size(mods, seed, relu):
    o, g = pair(mods, seed)
    rng = np.random.default_rng(5)
    rows, din, dout = 300, 1100, 200
    x, W, b = (rng.integers(0, (1 << 64) - 1, size=s, dtype=np.uint64) for s in (rows * din, din * dout, dout))
    (xo, xg), (Wo, Wg), (bo, bg) = ((o.share(a), g.share_a(a)) for a in (x, W, b))
    layer = g.dense_create(Wg, din, dout, b=bg)
    same(g.dense_forward(layer, xg, rows, relu=relu), o.dense_forward(xo, Wo, rows, din, dout, b=bo, relu=relu)[0])
    layer.close(); g.close()


# few rows, products by residues: within a step of terms, a whole chunk, one more term
LARGEST = [(7, 64, 70), (200, 65, 70), (200, 4096, 20), (300, 4096, 20), (300, 4097, 20)]


@pytest.mark.parametrize("rows,din,dout", LARGEST)
def test_largest_words(mods, seed, rows, din, dout):
    """Components that are the smallest and the largest signed words in turn: the largest sums that limbs and residues have to tell apart."""
    o, g = pair(mods, seed)
    low, high = np.uint64(1 << 63), np.uint64((1 << 63) - 1)
    for a, b in ((low, low), (low, high), (high, high)):
        xc, wc = np.full((3, rows * din), a, dtype=np.uint64), np.full((3, din * dout), b, dtype=np.uint64)
        import torch
        Oracle, gtree = mods

        def on_gpu(c):
            t = torch.from_numpy(np.stack([c, np.roll(c, -1, 0)], 1).astype(np.int64)).to("cuda")
            return gtree.Shares(c.shape[1], t=t.contiguous())

        layer = g.dense_create(on_gpu(wc), din, dout)
        same(g.dense_forward(layer, on_gpu(xc), rows), o.dense_forward(xc, wc, rows, din, dout)[0], "y")
        dy = np.full((3, rows * dout), b, dtype=np.uint64)
        for got, want in zip(g.dense_backward(layer, on_gpu(xc), on_gpu(dy), rows), o.dense_backward(xc, wc, dy, rows, din, dout)):
            same(got, want)
        layer.close()
    g.close()


def test_planes_of_odd_alignment_and_in_place_residual(mods, seed):
    import torch
    Oracle, gtree = mods
    o, g = pair(mods, seed)
    rng = np.random.default_rng(6)
    rows, din, dout = 1100, 130, 301
    x, W, r = pl.fixed(rng, 16, 1.0, rows, din), pl.fixed(rng, 16, 0.3, din, dout), pl.fixed(rng, 16, 1.0, rows, dout)
    (xo, xg), (Wo, Wg), (ro, rg) = shared(o, g, x), shared(o, g, W), shared(o, g, r)

    def odd(s):
        t = torch.empty((3, 2, s.n + 3 - s.n % 2), dtype=torch.int64, device="cuda")[:, :, 1:s.n + 1]
        t.copy_(s.t)
        return gtree.Shares(s.n, t=t)

    layer, y = g.dense_create(odd(Wg), din, dout), odd(rg)
    gtree._chk(g.L.gt_dense_forward(g.ctx, layer.h, gtree._ref(odd(xg)), rows, 1, gtree._ref(y), gtree._ref(y), None), "gt_dense_forward")
    same(y, o.dense_forward(xo, Wo, rows, din, dout, relu=True, residual=ro)[0])
    same_stats(o, g)
    layer.close(); g.close()


# rows, din, dout: gradients side by side with both tiles and one after the other, dx apart, more rows than a chunk of terms
BACKWARD = [(3, 400, 330), (64, 512, 256), (65, 400, 330), (200, 70, 150), (1000, 1300, 65), (500, 90, 1), (5000, 20, 30)]


@pytest.mark.parametrize("rows,din,dout", BACKWARD)
@pytest.mark.parametrize("gated", [False, True])
def test_dense_backward(mods, seed, rows, din, dout, gated):
    check_backward(mods, seed, rows, din, dout, gated)


@pytest.mark.parametrize("rows,din,dout", [(300, 640, 333), (300, 70, 40)])
def test_gradient_of_the_input_alone(mods, seed, rows, din, dout):
    check_backward(mods, seed, rows, din, dout, True, want=(True, False, True))


# rows, d, ff, experts, top: products by residues at the first layer, at both
MIXTURES = [(200, 40, 450, 8, 2), (400, 130, 300, 4, 1)]
# rows converted by a launch of their own, the division beside the product
LEFT_MIXTURES = [(24, 340, 1024, 8, 2)]


@pytest.mark.parametrize("rows,d,ff,E,top", MIXTURES + LEFT_MIXTURES)
@pytest.mark.parametrize("bias", [False, True])
def test_mixture_of_many_rows(mods, seed, rows, d, ff, E, top, bias):
    o, g = pair(mods, seed)
    rng = np.random.default_rng(rows)
    x, Wr, W1, W2 = (pl.fixed(rng, 16, 0.3, *s) for s in ((rows, d), (d, E), (E, d, ff), (E, ff, d)))
    br, b1, b2 = (pl.fixed(rng, 16, 0.5, *s) if bias else None for s in ((E,), (E, ff), (E, d)))
    both = [shared(o, g, a) for a in (x, Wr, W1, W2, br, b1, b2)]
    so, sg = [t[0] for t in both], [t[1] for t in both]
    moe = g.moe_create(sg[1], sg[2], sg[3], d, ff, E, top, rows, br=sg[4], b1=sg[5], b2=sg[6])
    for n in (rows, 3, rows):                             # a call of few rows between
        yo = o.moe_forward(np.ascontiguousarray(so[0][:, :n * d]), *so[1:4], n, d, ff, E, top, br=so[4], b1=so[5], b2=so[6])
        yg = g.moe_forward(moe, g_rows(g, sg[0], n * d), n)
        same(yg, yo, "y")
        same_stats(o, g)
    moe.close(); g.close()


def g_rows(g, s, n):
    from paper_2305_00645_amd import gtree
    return gtree.Shares(n, t=s.t[:, :, :n].contiguous())
