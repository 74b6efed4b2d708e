"""A captured layer next to larger eager calls, which outgrow the workspace that its graph holds; a captured call whose workspace would have to grow."""
import numpy as np
import pytest

import plain_layers as pl
from test_gpu_layers import shared
from test_gpu_parity import mods, pair, same  # noqa: F401

pytestmark = pytest.mark.gpu


def test_larger_calls_between_replays(mods, seed):
    import torch
    Oracle, gtree = mods
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        o, g = Oracle(seed), gtree.GTree(seed, stream=st)
        rng = np.random.default_rng(2)
        few, many, din, dout = 250, 700, 140, 130
        x, W, dy = pl.fixed(rng, 16, 1.0, many, din), pl.fixed(rng, 16, 0.2, din, dout), pl.fixed(rng, 16, 0.1, many, dout)
        (_, xg), (_, Wg), (_, dg) = (shared(o, g, a) for a in (x, W, dy))
        layer = g.dense_create(Wg, din, dout)

        def work(rows):
            y, gate = g.dense_forward(layer, xg, rows, relu=True, want_gate=True)
            return [y, gate, *g.dense_backward(layer, xg, dg, rows, gate=gate), g.dense_forward(layer, xg, 3)]

        work(few)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        y, gate, refused = g.new(many * dout), g.new(many * dout), []
        with torch.cuda.graph(graph, stream=st):
            op = g.op_counter()
            refused.append(g.L.gt_dense_forward(g.ctx, layer.h, gtree._ref(xg), many, 1, None, gtree._ref(y), gtree._ref(gate)))
            refused.append(g.op_counter() - op)
            got = work(few)
        assert refused == [gtree.GT_ESTATE, 0]
        graph.replay()
        st.synchronize()
        want = [t.t.clone() for t in got]
        for a, b in zip(got, work(few)):
            assert np.array_equal(g.rec(a), g.rec(b))
        for rows in (many, few):
            work(rows)                                    # the workspaces of products and gradients grow
            g.oaa_literal(g.share_a(np.arange(50, dtype=np.uint64)), g.share_a(np.arange(4000, dtype=np.uint64)))    # ... and the one of parts
            spare = [torch.full((1 << 22,), 7, dtype=torch.int64, device="cuda") for _ in range(8)]    # what was free is written
            st.synchronize()
            for t in got:
                t.t.zero_()
            graph.replay()
            st.synchronize()
            assert all(torch.equal(a.t, b) for a, b in zip(got, want))
            del spare
        layer.close(); g.close()
