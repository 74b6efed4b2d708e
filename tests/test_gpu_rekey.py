"""New keys on the GPU, and captured calls replayed on new inputs: every replay under keys of its own, against the oracle bit for bit."""
import numpy as np
import pytest

import plain_layers as pl
from test_gpu_layers import shared
from test_gpu_parity import mods, pair, same, same_stats  # noqa: F401

pytestmark = pytest.mark.gpu


def test_calls_before_and_after(mods, seed):
    o, g = pair(mods, seed)
    rng = np.random.default_rng(1)
    x, y = (rng.integers(0, 1 << 40, size=333).astype(np.uint64) for _ in range(2))
    for _ in range(3):
        (xo, xg), (yo, yg) = ((o.share(a), g.share_a(a)) for a in (x, y))
        same(xg, xo)
        same(g.mult(xg, yg), o.mult(xo, yo))
        o.rekey(); g.rekey()
        same(g.oaa(xg, yg), o.oaa(xo, yo))
        assert g.op_counter() == o.op_counter()
        same_stats(o, g)
    g.close()


@pytest.mark.parametrize("rows,din,dout", [(3, 40, 70), (260, 70, 65)])
def test_replays_on_new_inputs(mods, seed, rows, din, dout):
    import torch
    Oracle, gtree = mods
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        o, g = Oracle(seed), gtree.GTree(seed, stream=st)
        rng = np.random.default_rng(rows)
        (Wo, Wg), (bo, bg) = (shared(o, g, pl.fixed(rng, 16, 0.3, *s)) for s in ((din, dout), (dout,)))
        (xo, xg), (do, dg) = (shared(o, g, pl.fixed(rng, 16, 1.0, *s)) for s in ((rows, din), (rows, dout)))
        layer = g.dense_create(Wg, din, dout, b=bg)

        def work():
            y, gate = g.dense_forward(layer, xg, rows, relu=True, want_gate=True)
            return [y, gate, *g.dense_backward(layer, xg, dg, rows, gate=gate)]

        def oracle():
            y, gate = o.dense_forward(xo, Wo, rows, din, dout, b=bo, relu=True)
            return [y, gate, *o.dense_backward(xo, Wo, do, rows, din, dout, gate=gate)]

        for a, b in zip(work(), oracle()):                # eager first: the workspace grows
            same(a, b)
        op = g.op_counter()
        graph = torch.cuda.CUDAGraph()
        st.synchronize()
        with torch.cuda.graph(graph, stream=st):
            g.rekey()
            got = work()
        later, last = g.op_counter(), None
        o.set_op(later)
        for replay in range(3):
            x, d = pl.fixed(rng, 16, 1.0, rows, din), pl.fixed(rng, 16, 0.1, rows, dout)
            (xo, xn), (do, dn) = shared(o, g, x), shared(o, g, d)   # eager, under the newest keys
            same(xn, xo)
            now = o.op_counter()
            xg.t.copy_(xn.t); dg.t.copy_(dn.t)
            graph.replay()
            st.synchronize()
            o.rekey()
            o.set_op(op)
            want = oracle()
            assert o.op_counter() == later
            for a, b in zip(got, want):
                same(a, b)
            o.set_op(now)
            y = got[0].t.clone()
            assert last is None or not torch.equal(y, last)
            last = y
            assert g.op_counter() == now
        st.synchronize()
        layer.close(); g.close()
