"""The protocol of the layers (oracle) against Python integers, at the sizes and values where it can go wrong, and its message
counts; the binding's refusals that need no GPU."""
import ctypes as C

import numpy as np
import pytest

import plain_layers as pl
from oracle import Oracle
from paper_2305_00645_amd import gtree


def make(seed, f):
    return Oracle(seed, tau=f)


def dense(o, x, W, f, b=None, relu=False, res=None):
    rows, din, dout = x.shape[0], W.shape[0], W.shape[1]
    sh = [None if a is None else o.share(pl.words(a)) for a in (x, W, b, res)]
    return o.dense_forward(sh[0], sh[1], rows, din, dout, b=sh[2], relu=relu, residual=sh[3])


@pytest.mark.parametrize("f", [1, 2, 8, 13, 16, 20])
@pytest.mark.parametrize("relu", [False, True])
def test_rounding_at_its_borders(seed, f, relu):
    """One-term products, so that the sum is the first factor: around multiples of 2^f and of half of it, around zero, the smallest and
    largest sums allowed, with every fraction width."""
    o = make(seed, f)
    top = (1 << (f + 31)) if relu else 1 << 62
    half, one = 1 << (f - 1), 1 << f
    v = sorted({s * (m + d) for m in (0, half, one, one + half, 5 * one, 1 << 40 if not relu else 1 << (f + 20)) for d in (-2, -1, 0, 1, 2)
                for s in (1, -1)} | {top - half - 1, top - half - 2, -top, -top + 1, -top + half, -half, -half - 1})
    v = [t for t in v if -top <= t + half < top] + [0] * 5
    x = np.array(v, dtype=object)[:, None]
    y, gate = dense(o, x, np.array([[1]], dtype=object), f, relu=relu)
    want, bit = pl.forward(x, np.array([[1]], dtype=object), f, relu=relu)
    assert np.array_equal(o.rec(y), pl.words(want))
    if relu:
        assert np.array_equal(o.rec(gate), pl.words(bit))
    assert o.op_counter() == 3


@pytest.mark.parametrize("rows,din,dout", [(1, 1, 1), (1, 7, 3), (3, 1, 5), (2, 33, 17), (17, 5, 9), (0, 4, 3)])
@pytest.mark.parametrize("relu,bias,res", [(False, False, False), (True, True, False), (True, False, True), (False, True, True)])
def test_dense_forward(seed, rows, din, dout, relu, bias, res):
    f = 12
    rng = np.random.default_rng(rows * 100 + din)
    x, W = pl.fixed(rng, f, 1.0, rows, din), pl.fixed(rng, f, 1.0, din, dout)
    b = pl.fixed(rng, f, 1.0, dout) if bias else None
    r = pl.fixed(rng, f, 1.0, rows, dout) if res else None
    o = make(seed, f)
    y, gate = dense(o, x, W, f, b, relu, r)
    want, bit = pl.forward(x, W, f, b, relu, r)
    assert np.array_equal(o.rec(y), pl.words(want))
    if relu:
        assert np.array_equal(o.rec(gate), pl.words(bit))
    n = rows * dout
    bits = o.wire_bits()
    # opening to both others, the tree, the conversions, with ReLU the product
    assert bits[0][1] == n * (64 + (2 if relu else 1)) and bits[0][2] == n * (64 + (61 + 64 if relu else 30))
    assert o.stats()[0] == (8 if relu else 6)


@pytest.mark.parametrize("rows,din,dout,gated", [(1, 1, 1, True), (5, 3, 7, True), (4, 9, 2, False), (33, 6, 5, True)])
def test_dense_backward(seed, rows, din, dout, gated):
    f = 14
    rng = np.random.default_rng(rows)
    x, W, dy = pl.fixed(rng, f, 1.0, rows, din), pl.fixed(rng, f, 1.0, din, dout), pl.fixed(rng, f, 0.1, rows, dout)
    gate = rng.integers(0, 2, size=(rows, dout)).astype(object) if gated else None
    o = make(seed, f)
    sh = [None if a is None else o.share(pl.words(a)) for a in (x, W, dy, gate)]
    got = o.dense_backward(sh[0], sh[1], sh[2], rows, din, dout, gate=sh[3])
    for g, w in zip(got, pl.backward(x, W, dy, f, gate)):
        assert np.array_equal(o.rec(g), pl.words(w))


def test_gradient_against_differences(seed):
    """The gradients of loss = sum(dy * ReLU(x W + b)) against differences of the plain forward pass in real numbers: each is a rounded
    sum of rows (or columns) products, so it is off by at most half a unit of the last place; the difference quotient of a piecewise linear function
    is exact away from its kinks up to float64's rounding, which leaves 2^-f."""
    f, rows, din, dout = 16, 6, 4, 5
    rng = np.random.default_rng(3)
    x, W, b, dy = (pl.fixed(rng, f, 1.0, *s) for s in ((rows, din), (din, dout), (dout,), (rows, dout)))
    o = make(seed, f)
    sx, sW, sb, sdy = (o.share(pl.words(a)) for a in (x, W, b, dy))
    _, gate = o.dense_forward(sx, sW, rows, din, dout, b=sb, relu=True)
    got = [pl.signed(o.rec(t)).astype(np.float64) / 2 ** f for t in o.dense_backward(sx, sW, sdy, rows, din, dout, gate=gate)]
    xr, Wr, br, dr = (a.astype(np.float64) / 2 ** f for a in (x, W, b, dy))

    def loss(x_, W_, b_):
        return float((dr * np.maximum(x_ @ W_ + b_, 0)).sum())

    eps = 2.0 ** -20
    assert np.abs(xr @ Wr + br).min() > 64 * eps          # no kink near
    for k, a in enumerate((xr, Wr, br)):
        for i in np.ndindex(a.shape):
            up, down = a.copy(), a.copy()
            up[i] += eps
            down[i] -= eps
            args = [[xr, Wr, br] for _ in range(2)]
            args[0][k], args[1][k] = up, down
            diff = (loss(*args[0]) - loss(*args[1])) / (2 * eps)
            assert abs(got[k].reshape(a.shape)[i] - diff) <= 2.0 ** -f, (k, i)


@pytest.mark.parametrize("rows,d,ff,E,top", [(1, 3, 4, 1, 1), (2, 5, 3, 2, 1), (3, 4, 6, 5, 2), (2, 3, 5, 4, 4), (0, 3, 2, 2, 1)])
@pytest.mark.parametrize("bias", [False, True])
def test_moe(seed, rows, d, ff, E, top, bias):
    f = 13
    rng = np.random.default_rng(rows + E)
    x, Wr, W1, W2 = (pl.fixed(rng, f, 0.7, *s) for s in ((rows, d), (d, E), (E, d, ff), (E, ff, d)))
    br, b1, b2 = (pl.fixed(rng, f, 0.5, *s) if bias else None for s in ((E,), (E, ff), (E, d)))
    res = pl.fixed(rng, f, 1.0, rows, d)
    o = make(seed, f)
    sh = [None if a is None else o.share(pl.words(a)) for a in (x, Wr, W1, W2, br, b1, b2, res)]
    op = o.op_counter()
    y = o.moe_forward(*sh[:4], rows, d, ff, E, top, br=sh[4], b1=sh[5], b2=sh[6], residual=sh[7])
    assert o.op_counter() - op == 10 + f
    assert np.array_equal(o.rec(y), pl.words(pl.moe(x, Wr, W1, W2, f, top, br, b1, b2, res)))


def test_moe_ties_and_no_scores(seed):
    """Equal scores: the lower index; no positive score: gates of zero, so the layer adds nothing but the residual."""
    f, d, ff, E = 10, 2, 3, 4
    rng = np.random.default_rng(8)
    W1, W2, b2 = pl.fixed(rng, f, 1.0, E, d, ff), pl.fixed(rng, f, 1.0, E, ff, d), pl.fixed(rng, f, 1.0, E, d)
    x = np.array([[1 << f, 0], [-(1 << f), 0], [0, 0]], dtype=object)
    Wr = np.array([[1 << f] * E, [0] * E], dtype=object)
    o = make(seed, f)
    sh = [o.share(pl.words(a)) for a in (x, Wr, W1, W2, b2)]
    y = pl.signed(o.rec(o.moe_forward(*sh[:4], 3, d, ff, E, 2, b2=sh[4]))).reshape(3, d)
    assert np.array_equal(y, pl.moe(x, Wr, W1, W2, f, 2, None, None, b2, None))
    assert not y[1].any() and not y[2].any()


def test_refusals_without_a_gpu():
    L = gtree.load()
    h = C.c_void_p()
    assert L.gt_dense_create(None, None, None, 1, 1, C.byref(h)) == gtree.GT_EINVAL
    assert L.gt_dense_set(None, None, None, None) == gtree.GT_EINVAL
    assert L.gt_dense_forward(None, None, None, 0, 0, None, None, None) == gtree.GT_EINVAL
    assert L.gt_dense_backward(None, None, None, None, None, 0, None, None, None) == gtree.GT_EINVAL
    assert L.gt_moe_create(None, None, None, None, None, None, None, 1, 1, 1, 1, 1, C.byref(h)) == gtree.GT_EINVAL
    assert L.gt_moe_forward(None, None, None, 0, None, None) == gtree.GT_EINVAL
    assert L.gt_dense_destroy(None) == gtree.GT_EINVAL and L.gt_moe_destroy(None) == gtree.GT_EINVAL
    assert not h.value
