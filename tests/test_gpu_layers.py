"""Layers on the GPU against the CPU oracle: every share plane bit for bit, rounds and bytes; refusals."""
import numpy as np
import pytest

import plain_layers as pl
from test_gpu_parity import mods, pair, same, same_stats  # noqa: F401

pytestmark = pytest.mark.gpu


def shared(o, g, a):
    """The same sharing on both sides; None stays None."""
    if a is None:
        return None, None
    w = pl.words(a)
    return o.share(w), g.share_a(w)


def check_dense(mods, seed, rows, din, dout, relu, bias, res, f=16, calls=1, std=1.0, seed2=0):
    o, g = pair(mods, seed, tau=f)
    rng = np.random.default_rng(rows * 1009 + din * 31 + dout + seed2)
    x, W = pl.fixed(rng, f, std, rows, din), pl.fixed(rng, f, std * max(din, 1) ** -0.5, din, dout)
    b = pl.fixed(rng, f, std, dout) if bias else None
    r = pl.fixed(rng, f, std, rows, dout) if res else None
    (xo, xg), (Wo, Wg), (bo, bg), (ro, rg) = (shared(o, g, a) for a in (x, W, b, r))
    layer = g.dense_create(Wg, din, dout, b=bg)
    for call in range(calls):
        yo, go = o.dense_forward(xo, Wo, rows, din, dout, b=bo, relu=relu, residual=ro)
        got = g.dense_forward(layer, xg, rows, relu=relu, residual=rg, want_gate=relu)
        yg, gg = got if relu else (got, None)
        print("dense", rows, din, dout, relu, call, flush=True)
        same(yg, yo, "y")
        if relu:
            same(gg, go, "gate")
        same_stats(o, g)
    want, _ = pl.forward(x[:4], W, f, b, relu, None if r is None else r[:4])
    assert np.array_equal(g.rec(yg)[:want.size], pl.words(want))
    layer.close(); g.close()


SIZES = [(1, 1, 1), (1, 64, 64), (1, 1, 97), (1, 300, 1), (2, 65, 33), (7, 31, 130), (8, 64, 16), (9, 70, 48), (15, 129, 15), (16, 64, 32),
         (17, 63, 31), (31, 128, 64), (33, 294, 257), (64, 64, 64), (65, 96, 70), (100, 22, 16), (129, 33, 5), (267, 22, 3)]


@pytest.mark.parametrize("rows,din,dout", SIZES)
@pytest.mark.parametrize("relu,bias,res", [(False, False, True), (True, True, False)])
def test_dense_forward(mods, seed, rows, din, dout, relu, bias, res):
    check_dense(mods, seed, rows, din, dout, relu, bias, res, calls=2)


@pytest.mark.parametrize("f", [1, 2, 9, 13, 20])
@pytest.mark.parametrize("relu", [False, True])
def test_fraction_widths(mods, seed, f, relu):
    check_dense(mods, seed, 5, 40, 37, relu, True, True, f=f, std=4.0)
    check_dense(mods, seed, 70, 40, 37, relu, True, True, f=f, std=4.0)


@pytest.mark.parametrize("rows,din,dout", [(1, 40, 24), (300, 200, 70)])
@pytest.mark.parametrize("relu", [False, True])
def test_words_of_any_size(mods, seed, rows, din, dout, relu):
    """Plain words over the whole ring: sums wrap, results are what the protocol makes of them on both sides."""
    o, g = pair(mods, seed)
    rng = np.random.default_rng(rows)
    x, W, b = (rng.integers(0, (1 << 64) - 1, size=s, dtype=np.uint64) for s in (rows * din, din * dout, dout))
    (xo, xg), (Wo, Wg), (bo, bg) = ((o.share(a), g.share_a(a)) for a in (x, W, b))
    layer = g.dense_create(Wg, din, dout, b=bg)
    same(g.dense_forward(layer, xg, rows, relu=relu), o.dense_forward(xo, Wo, rows, din, dout, b=bo, relu=relu)[0])
    layer.close(); g.close()


def test_no_rows_and_in_place_residual(mods, seed):
    o, g = pair(mods, seed)
    rng = np.random.default_rng(0)
    W, r = pl.fixed(rng, 16, 1.0, 6, 10), pl.fixed(rng, 16, 1.0, 3, 10)
    x = pl.fixed(rng, 16, 1.0, 3, 6)
    (Wo, Wg), (ro, rg), (xo, xg) = (shared(o, g, a) for a in (W, r, x))
    layer = g.dense_create(Wg, 6, 10)
    empty = o.share(np.zeros(0, dtype=np.uint64)), g.share_a(np.zeros(0, dtype=np.uint64))
    assert g.dense_forward(layer, empty[1], 0, relu=True).n == 0
    o.dense_forward(empty[0], Wo, 0, 6, 10, relu=True)
    yo, _ = o.dense_forward(xo, Wo, 3, 6, 10, residual=ro)
    from paper_2305_00645_amd import gtree
    gtree._chk(g.L.gt_dense_forward(g.ctx, layer.h, gtree._ref(xg), 3, 0, gtree._ref(rg), gtree._ref(rg), None), "gt_dense_forward")
    same(rg, yo)
    same_stats(o, g)
    layer.close(); g.close()


def check_backward(mods, seed, rows, din, dout, gated, f=16, want=(True, True, True)):
    o, g = pair(mods, seed, tau=f)
    rng = np.random.default_rng(rows * 7 + din + dout)
    x, W, dy = pl.fixed(rng, f, 1.0, rows, din), pl.fixed(rng, f, 1.0, din, dout), pl.fixed(rng, f, 0.1, rows, dout)
    gate = rng.integers(0, 2, size=(rows, dout)).astype(object) if gated else None
    (xo, xg), (Wo, Wg), (do, dg), (go, gg) = (shared(o, g, a) for a in (x, W, dy, gate))
    layer = g.dense_create(Wg, din, dout)
    for call in range(2):
        print("backward", rows, din, dout, gated, call, flush=True)
        for name, a, b in zip(("dx", "dW", "db"), g.dense_backward(layer, xg, dg, rows, gate=gg, want=want),
                              o.dense_backward(xo, Wo, do, rows, din, dout, gate=go, want=want)):
            assert (a is None) == (b is None)
            if a is not None:
                same(a, b, name)
        same_stats(o, g)
    layer.close(); g.close()


@pytest.mark.parametrize("rows,din,dout", [(1, 1, 1), (1, 50, 70), (5, 33, 20), (16, 64, 17), (40, 3, 129), (129, 70, 65), (267, 22, 16), (300, 64, 33)])
@pytest.mark.parametrize("gated", [False, True])
def test_dense_backward(mods, seed, rows, din, dout, gated):
    check_backward(mods, seed, rows, din, dout, gated)


@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True), (True, False, True)])
def test_dense_backward_parts(mods, seed, want):
    check_backward(mods, seed, 9, 20, 30, True, want=want)


def check_moe(mods, seed, rows, d, ff, E, top, bias, res, f=16, calls=2, most=None, std=0.7):
    o, g = pair(mods, seed, tau=f)
    rng = np.random.default_rng(rows * 3 + E + d)
    x, Wr, W1, W2 = (pl.fixed(rng, f, std, *s) for s in ((rows, d), (d, E), (E, d, ff), (E, ff, d)))
    br, b1, b2 = (pl.fixed(rng, f, 0.5, *s) if bias else None for s in ((E,), (E, ff), (E, d)))
    r = pl.fixed(rng, f, 1.0, rows, d) if res else None
    both = [shared(o, g, a) for a in (x, Wr, W1, W2, br, b1, b2, r)]
    so, sg = [t[0] for t in both], [t[1] for t in both]
    moe = g.moe_create(sg[1], sg[2], sg[3], d, ff, E, top, most or rows, br=sg[4], b1=sg[5], b2=sg[6])
    for call in range(calls):
        print("moe", rows, d, ff, E, top, call, flush=True)
        yo = o.moe_forward(*so[:4], rows, d, ff, E, top, br=so[4], b1=so[5], b2=so[6], residual=so[7])
        yg = g.moe_forward(moe, sg[0], rows, residual=sg[7])
        same(yg, yo, "y")
        same_stats(o, g)
    assert np.array_equal(g.rec(yg), pl.words(pl.moe(x, Wr, W1, W2, f, top, br, b1, b2, r)))
    moe.close(); g.close()


@pytest.mark.parametrize("rows,d,ff,E,top", [(1, 1, 1, 1, 1), (1, 64, 64, 8, 1), (1, 17, 33, 2, 2), (5, 65, 130, 5, 2), (3, 20, 16, 16, 3), (16, 24, 40, 8, 2),
                                             (20, 30, 18, 4, 4), (2, 8, 8, 64, 2), (70, 9, 11, 3, 1)])
@pytest.mark.parametrize("bias,res", [(True, False), (False, True)])
def test_moe(mods, seed, rows, d, ff, E, top, bias, res):
    check_moe(mods, seed, rows, d, ff, E, top, bias, res)


@pytest.mark.parametrize("f", [3, 10, 20])
def test_moe_fraction_widths(mods, seed, f):
    check_moe(mods, seed, 3, 12, 10, 4, 2, True, True, f=f, most=8)


def test_new_weights_in_place(mods, seed):
    o, g = pair(mods, seed)
    rng = np.random.default_rng(4)
    x, b = pl.fixed(rng, 16, 1.0, 70, 20), pl.fixed(rng, 16, 1.0, 9)
    (xo, xg), (bo, bg) = shared(o, g, x), shared(o, g, b)
    layer = None
    for _ in range(2):
        Wo, Wg = shared(o, g, pl.fixed(rng, 16, 1.0, 20, 9))
        if layer is None:
            layer = g.dense_create(Wg, 20, 9, b=bg)
        else:
            g.dense_set(layer, Wg, b=bg)
        for rows in (2, 70):
            xs = np.ascontiguousarray(xo[:, :rows * 20])
            same(g.dense_forward(layer, xg, rows), o.dense_forward(xs, Wo, rows, 20, 9, b=bo)[0])
            dy = shared(o, g, pl.fixed(rng, 16, 0.1, rows, 9))
            for a, w in zip(g.dense_backward(layer, xg, dy[1], rows), o.dense_backward(xs, Wo, dy[0], rows, 20, 9)):
                same(a, w)
    layer.close(); g.close()


def test_another_stream_and_planes_of_odd_alignment(mods, seed):
    """Work on the context's own stream; planes that start 8 but not 16 bytes aligned."""
    import torch
    Oracle, gtree = mods
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        o, g = Oracle(seed), gtree.GTree(seed, stream=st)
        rng = np.random.default_rng(6)
        for rows in (3, 90):
            x, W = pl.fixed(rng, 16, 1.0, rows, 21), pl.fixed(rng, 16, 0.3, 21, 13)
            (xo, xg), (Wo, Wg) = shared(o, g, x), shared(o, g, W)

            def odd(s):
                t = torch.empty((3, 2, s.n + 3 - s.n % 2), dtype=torch.int64, device="cuda")[:, :, 1:s.n + 1]
                t.copy_(s.t)
                return gtree.Shares(s.n, t=t)

            layer = g.dense_create(odd(Wg), 21, 13)
            same(g.dense_forward(layer, odd(xg), rows, relu=True), o.dense_forward(xo, Wo, rows, 21, 13, relu=True)[0])
            layer.close()
        st.synchronize()
        g.close()


def test_refusals(mods, seed):
    _, gtree = mods
    g = gtree.GTree(seed)
    rng = np.random.default_rng(1)
    s = lambda n: g.share_a(rng.integers(0, 1 << 20, size=n).astype(np.uint64))  # noqa: E731
    W, x, y = s(12), s(8), s(6)
    layer, plain = g.dense_create(W, 4, 3, b=s(3)), g.dense_create(W, 4, 3)
    moe = g.moe_create(s(8), s(24), s(24), 4, 3, 2, 1, 2)
    ref, L, E = gtree._ref, g.L, gtree.GT_EINVAL
    import ctypes as C
    h = C.c_void_p()
    bad = [
        L.gt_dense_create(g.ctx, ref(W), None, 0, 3, C.byref(h)), L.gt_dense_create(g.ctx, ref(W), None, 4, 4, C.byref(h)),
        L.gt_dense_create(g.ctx, ref(W), ref(s(2)), 4, 3, C.byref(h)), L.gt_dense_create(g.ctx, None, None, 4, 3, C.byref(h)),
        L.gt_dense_create(g.ctx, ref(W), None, (1 << 20) + 1, 1, C.byref(h)),
        L.gt_dense_set(g.ctx, layer.h, ref(W), None), L.gt_dense_set(g.ctx, plain.h, ref(W), ref(s(3))), L.gt_dense_set(g.ctx, layer.h, ref(s(11)), ref(s(3))),
        L.gt_dense_forward(g.ctx, layer.h, ref(x), 3, 0, None, ref(y), None), L.gt_dense_forward(g.ctx, layer.h, ref(x), 2, 2, None, ref(y), None),
        L.gt_dense_forward(g.ctx, layer.h, ref(x), 2, 0, None, ref(s(5)), None), L.gt_dense_forward(g.ctx, layer.h, ref(x), 2, 0, ref(s(5)), ref(y), None),
        L.gt_dense_forward(g.ctx, layer.h, ref(x), 2, 0, None, ref(y), ref(s(6))), L.gt_dense_forward(g.ctx, layer.h, None, 2, 0, None, ref(y), None),
        L.gt_dense_backward(g.ctx, layer.h, None, None, ref(y), 2, None, ref(s(12)), None),
        L.gt_dense_backward(g.ctx, layer.h, ref(x), ref(s(5)), ref(y), 2, ref(s(8)), None, None),
        L.gt_dense_backward(g.ctx, layer.h, ref(x), None, ref(y), 2, ref(s(7)), None, None),
        L.gt_dense_backward(g.ctx, layer.h, ref(x), None, ref(y), 2, None, ref(s(11)), None),
        L.gt_dense_backward(g.ctx, layer.h, ref(x), None, ref(y), 2, None, None, ref(s(2))),
        L.gt_moe_create(g.ctx, ref(s(8)), None, ref(s(24)), None, ref(s(24)), None, 4, 3, 2, 3, 2, C.byref(h)),
        L.gt_moe_create(g.ctx, ref(s(8)), None, ref(s(24)), None, ref(s(24)), None, 4, 3, 0, 0, 2, C.byref(h)),
        L.gt_moe_create(g.ctx, ref(s(8)), None, ref(s(23)), None, ref(s(24)), None, 4, 3, 2, 1, 2, C.byref(h)),
        L.gt_moe_create(g.ctx, ref(s(260)), None, ref(s(780)), None, ref(s(780)), None, 4, 3, 65, 1, 2, C.byref(h)),
        L.gt_moe_forward(g.ctx, moe.h, ref(s(12)), 3, None, ref(s(12))), L.gt_moe_forward(g.ctx, moe.h, ref(s(7)), 2, None, ref(s(8))),
        L.gt_moe_forward(g.ctx, moe.h, ref(s(8)), 2, ref(s(7)), ref(s(8))),
    ]
    assert bad == [E] * len(bad), bad
    assert not h.value
    op, xs, ys = g.op_counter(), s(12), s(9)             # a refused call takes no operation id
    assert L.gt_dense_forward(g.ctx, layer.h, ref(xs), 4, 0, None, ref(ys), None) == E and g.op_counter() == op + 2
    for t in (layer, plain, moe):
        t.close()
    g.close()
