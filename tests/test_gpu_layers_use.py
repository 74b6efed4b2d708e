"""The layers used together, and recorded into a graph."""
import importlib.util
import os

import numpy as np
import pytest

import plain_layers as pl
from test_gpu_layers import shared
from test_gpu_parity import mods, pair, same  # noqa: F401

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "layers.py")
    spec = importlib.util.spec_from_file_location("layers_example", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_trains_as_its_plain_form_does(mods, seed):
    """Three steps of the example's network against the same steps in integers, weights and losses equal."""
    _, gtree = mods
    f, ex = 16, example()
    g = gtree.GTree(seed, tau=f)
    rng = np.random.default_rng(11)
    X, T = (pl.signed(g.rec(s)) for s in ex.data(g, rng))
    rate = 0.5 / ex.ROWS
    W = [pl.signed(g.rec(g.share_a(g.fixed(rng.normal(size=s) * s[0] ** -0.5).reshape(-1)))).reshape(s) for s in ((ex.COLS, ex.HIDDEN), (ex.HIDDEN, 1))]
    b = [np.array([0] * s.shape[1], dtype=object) for s in W]
    X, T = X.reshape(ex.ROWS, ex.COLS), T.reshape(ex.ROWS, 1)
    eye = [np.array(np.round(-rate * np.eye(s.shape[1]) * 2 ** f).astype(np.int64), dtype=object) for s in W]
    net, _, losses = ex.train(g, 3)
    for step in range(3):
        h, gate = pl.forward(X, W[0], f, b[0], True)
        y, _ = pl.forward(h, W[1], f, b[1])
        dy = y - T
        assert abs(losses[step] - 0.5 * float(np.mean((dy.astype(np.float64) / 2 ** f) ** 2))) <= 1e-9 * max(1.0, losses[step])
        dh, dW1, db1 = pl.backward(h, W[1], dy, f)
        _, dW0, db0 = pl.backward(X, W[0], dh, f, gate)
        for i, (dW, db) in enumerate(((dW0, db0), (dW1, db1))):
            W[i], _ = pl.forward(dW, eye[i], f, None, False, W[i])
            step_b, _ = pl.forward(db[None, :], eye[i], f, None, False, b[i][None, :])
            b[i] = step_b[0]
    for i in range(2):
        assert np.array_equal(g.rec(net.W[i]), pl.words(W[i])) and np.array_equal(g.rec(net.b[i]), pl.words(b[i]))
    net.close(); g.close()


def test_example_learns(mods, seed):
    _, gtree = mods
    g = gtree.GTree(seed, tau=16)
    net, _, losses = example().train(g, 40)
    assert losses[-1] < 0.5 * losses[0], (losses[0], losses[-1])
    net.close(); g.close()


@pytest.mark.parametrize("rows,din,dout", [(3, 40, 70), (500, 600, 130)])
def test_layers_in_a_graph(mods, seed, rows, din, dout):
    """Forward, backward and a mixture in a captured graph: every replay gives the eager results of the same operation ids, with eager work between."""
    import torch
    Oracle, gtree = mods
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        o, g = Oracle(seed), gtree.GTree(seed, stream=st)
        rng = np.random.default_rng(3)
        x, W, dy = pl.fixed(rng, 16, 1.0, rows, din), pl.fixed(rng, 16, 0.2, din, dout), pl.fixed(rng, 16, 0.1, rows, dout)
        (_, xg), (_, Wg), (_, dg) = (shared(o, g, a) for a in (x, W, dy))
        E, ff, few = 3, 20, min(rows, 4)
        m = [shared(o, g, pl.fixed(rng, 16, 0.3, *s))[1] for s in ((din, E), (E, din, ff), (E, ff, din))]
        layer, moe = g.dense_create(Wg, din, dout), g.moe_create(*m, din, ff, E, 2, few)
        xs = gtree.Shares(few * din, t=xg.t[:, :, :few * din].contiguous())

        def work():
            y, gate = g.dense_forward(layer, xg, rows, relu=True, want_gate=True)
            return [y, gate, *g.dense_backward(layer, xg, dg, rows, gate=gate), g.moe_forward(moe, xs, few)]

        work()                                            # workspaces grow here
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            got = work()
        words = []
        for replay in range(3):
            for t in got:
                t.t.zero_()
            graph.replay()
            st.synchronize()
            words.append([t.t.clone() for t in got])
            eager = work()                                # other operation ids: other shares of the same values
            st.synchronize()
            for a, b in zip(got, eager):
                assert np.array_equal(g.rec(a), g.rec(b))
        for later in words[1:]:
            assert all(torch.equal(a, b) for a, b in zip(words[0], later))
        st.synchronize()
        layer.close(); moe.close(); g.close()
