"""The gated layer and linear attention on the GPU against the CPU oracle: every share plane bit for bit, rounds and bytes; refusals; a block of them, captured
into a graph too."""
import numpy as np
import pytest

import plain_block as pb
import plain_layers as pl
from test_block import lin_inputs
from test_gpu_layers import shared
from test_gpu_parity import mods, pair, same, same_stats  # noqa: F401

pytestmark = pytest.mark.gpu

DECAYS = [4096, 3900, 0, 2048, 4095, 1]


def contexts(mods, seed, f, small):
    if not small:
        return pair(mods, seed, tau=f)
    Oracle, gtree = mods
    return Oracle(seed, tau=f), gtree.GTree(seed, tau=f, flags=gtree.GT_FLAG_SMALL_WORKSPACE)


def check_gated(mods, seed, rows, din, ff, relu, bias, keep, f=16, calls=2, small=False):
    o, g = contexts(mods, seed, f, small)
    rng = np.random.default_rng(rows * 1009 + din * 31 + ff)
    x, Wg, Wu = pl.fixed(rng, f, 1.0, rows, din), pl.fixed(rng, f, din ** -0.5, din, ff), pl.fixed(rng, f, din ** -0.5, din, ff)
    bg, bu = (pl.fixed(rng, f, 1.0, ff) if bias else None for _ in range(2))
    (xo, xg), (go, gg), (uo, ug), (bo, bgg), (co, cg) = (shared(o, g, a) for a in (x, Wg, Wu, bg, bu))
    layer = g.gated_create(gg, ug, din, ff, bg=bgg, bu=cg)
    for call in range(calls):
        print("gated", rows, din, ff, relu, bias, keep, f, call, flush=True)
        want = o.gated_forward(xo, go, uo, rows, din, ff, bg=bo, bu=co, relu=relu)
        got = g.gated_forward(layer, xg, rows, relu=relu, keep=keep)
        same(got[0] if keep else got, want[0], "h")
        if keep:
            for name, a, b in zip(("g", "u", "gate"), got[1], want[1:]):
                assert (a is None) == (b is None)
                if a is not None:
                    same(a, b, name)
        same_stats(o, g)
    if rows:
        plain = pb.gated(x[:4], Wg, Wu, f, bg, bu, relu)[0]
        assert np.array_equal(g.rec(got[0] if keep else got)[:plain.size], pl.words(plain))
    layer.close(); g.close()


# few rows; more than 192 rows; odd widths, below 8, at the borders of 64; many parts; residues, one tile and two a wavefront (see tests/block_shapes.py)
GATED = [(1, 1, 1), (1, 64, 128), (1, 300, 7), (2, 65, 33), (7, 31, 64), (8, 64, 65), (16, 130, 9), (33, 294, 257), (100, 22, 16), (193, 70, 24), (193, 70, 25),
         (267, 22, 3), (300, 200, 127), (1000, 50, 130), (400, 300, 301), (700, 150, 260), (1000, 294, 257)]


@pytest.mark.parametrize("rows,din,ff", GATED)
@pytest.mark.parametrize("relu,bias,keep", [(True, True, False), (False, False, True), (True, False, True)])
def test_gated_forward(mods, seed, rows, din, ff, relu, bias, keep):
    check_gated(mods, seed, rows, din, ff, relu, bias, keep)


@pytest.mark.parametrize("f", [1, 9, 20])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("rows", [5, 300])
def test_gated_fraction_widths(mods, seed, f, relu, rows):
    check_gated(mods, seed, rows, 90, 37, relu, True, True, f=f, calls=1)


@pytest.mark.parametrize("rows,din,ff", [(600, 130, 300), (300, 8300, 70)])
def test_gated_small_workspace(mods, seed, rows, din, ff):
    check_gated(mods, seed, rows, din, ff, True, True, True, small=True)


def test_gated_no_rows(mods, seed):
    check_gated(mods, seed, 0, 5, 6, True, True, True)


def test_gated_set(mods, seed):
    """New weights in place: the outputs are those of a new layer."""
    o, g = pair(mods, seed)
    rng = np.random.default_rng(1)
    sets = [[shared(o, g, pl.fixed(rng, 16, 0.5, *s)) for s in ((9, 70), (9, 70), (70,), (70,))] for _ in range(2)]
    xo, xg = shared(o, g, pl.fixed(rng, 16, 1.0, 4, 9))
    layer = g.gated_create(sets[0][0][1], sets[0][1][1], 9, 70, bg=sets[0][2][1], bu=sets[0][3][1])
    for Wg, Wu, bg, bu in (sets[0], sets[1]):
        g.gated_set(layer, Wg[1], Wu[1], bg=bg[1], bu=bu[1])
        same(g.gated_forward(layer, xg, 4), o.gated_forward(xo, Wg[0], Wu[0], 4, 9, 70, bg=bg[0], bu=bu[0])[0])
    layer.close(); g.close()


def check_gated_back(mods, seed, rows, din, ff, relu, f=16, want=(True, True, True), small=False):
    o, g = contexts(mods, seed, f, small)
    rng = np.random.default_rng(rows * 7 + din + ff)
    x, Wg, Wu = pl.fixed(rng, f, 1.0, rows, din), pl.fixed(rng, f, 1.0, din, ff), pl.fixed(rng, f, 1.0, din, ff)
    dh, u, a = pl.fixed(rng, f, 0.1, rows, ff), pl.fixed(rng, f, 1.0, rows, ff), pl.fixed(rng, f, 1.0, rows, ff)
    s = rng.integers(0, 2, size=(rows, ff)).astype(object) if relu else None
    (xo, xg), (go, gg), (uo, ug), (do, dg), (ao, ag), (vo, vg), (so, sg) = (shared(o, g, t) for t in (x, Wg, Wu, dh, a, u, s))
    layer = g.gated_create(gg, ug, din, ff)
    for call in range(2):
        print("gated back", rows, din, ff, relu, want, call, flush=True)
        for name, p, q in zip(("dx", "dWg", "dWu", "dbg", "dbu"), g.gated_backward(layer, xg, dg, rows, (ag, vg, sg), want=want),
                              o.gated_backward(xo, go, uo, do, rows, din, ff, (ao, vo, so), want=want)):
            assert (p is None) == (q is None)
            if p is not None:
                same(p, q, name)
        same_stats(o, g)
    layer.close(); g.close()


@pytest.mark.parametrize("rows,din,ff", [(0, 3, 4), (1, 1, 1), (1, 50, 70), (5, 33, 20), (16, 64, 17), (40, 3, 129), (129, 70, 65), (267, 22, 16), (300, 64, 33),
                                         (300, 300, 90), (600, 70, 90), (70, 1000, 1030), (140, 600, 500)])
@pytest.mark.parametrize("relu", [False, True])
def test_gated_backward(mods, seed, rows, din, ff, relu):
    check_gated_back(mods, seed, rows, din, ff, relu)


# few elements (k_gated_back_few) and at least 40 a SIMD (k_gated_back); see tests/test_block_shapes.py
BACK_WIDTHS = [(9, 20, 37), (700, 30, 61)]


@pytest.mark.parametrize("rows,din,ff", BACK_WIDTHS)
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("f", [1, 9, 20])
def test_gated_backward_fraction_widths(mods, seed, rows, din, ff, relu, f):
    check_gated_back(mods, seed, rows, din, ff, relu, f=f)


@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True), (True, False, True), (False, False, False)])
def test_gated_backward_parts(mods, seed, want):
    check_gated_back(mods, seed, 9, 20, 30, True, want=want)


def test_gated_backward_small_workspace(mods, seed):
    check_gated_back(mods, seed, 4500, 20, 30, True, small=True)


def check_lin(mods, seed, seqs, tokens, heads, dk, dv, f=16, fused=False, state=True, inplace=False, calls=2, small=False, decays=DECAYS):
    o, g = contexts(mods, seed, f, small)
    decay = (decays * heads)[:heads]
    q, k, v, S = lin_inputs(f, seqs, tokens, heads, dk, dv)
    n = seqs * tokens
    if fused:
        rows = np.concatenate([t.reshape(n, -1) for t in (q, k, v)], 1)
        ro, rg = shared(o, g, rows)
        parts = np.split(ro.reshape(3, n, -1), [heads * dk, 2 * heads * dk], axis=2)
        xo, xg = [np.ascontiguousarray(t).reshape(3, -1) for t in parts], (rg,)
    else:
        both = [shared(o, g, t) for t in (q, k, v)]
        xo, xg = [t[0] for t in both], [t[1] for t in both]
    So, Sg = shared(o, g, S) if state else (None, None)
    layer = g.linattn_create([w / 4096 for w in decay], dk, dv)
    for call in range(calls):
        print("linattn", seqs, tokens, heads, dk, dv, f, fused, state, inplace, call, flush=True)
        yo, So = o.linattn_forward(*xo, So, decay, seqs, tokens, dk, dv)
        y, Sg = g.linattn_forward(layer, *xg, seqs=seqs, tokens=tokens, state=Sg, inplace=inplace)
        same(y, yo, "o")
        same(Sg, So, "state")
        same_stats(o, g)
        if call == 0:
            want, last = pb.linattn(q[:1], k[:1], v[:1], S[:1] if state else S[:1] * 0, decay, f)
            assert np.array_equal(g.rec(y)[:want.size], pl.words(want)) and np.array_equal(g.rec(Sg)[:last.size], pl.words(last))
    layer.close(); g.close()


LIN = [(1, 1, 1, 1, 1), (1, 1, 4, 64, 64), (5, 1, 3, 20, 77), (2, 1, 2, 130, 9), (1, 2, 1, 3, 2), (3, 7, 2, 16, 8), (2, 31, 2, 5, 12), (1, 32, 1, 64, 16), (1, 33, 1, 8, 65),
       (2, 63, 1, 40, 30), (1, 64, 2, 64, 64), (3, 77, 5, 33, 65), (1, 129, 2, 65, 130), (2, 200, 1, 9, 24), (1, 1, 1, 256, 256), (1, 70, 1, 200, 250), (3, 1, 16, 64, 64), (1, 65, 16, 64, 64), (1, 300, 16, 16, 40), (2, 320, 8, 4, 4)]


@pytest.mark.parametrize("seqs,tokens,heads,dk,dv", LIN)
@pytest.mark.parametrize("fused,state,inplace", [(False, True, False), (True, False, False), (True, True, True)])
def test_linattn(mods, seed, seqs, tokens, heads, dk, dv, fused, state, inplace):
    check_lin(mods, seed, seqs, tokens, heads, dk, dv, fused=fused, state=state, inplace=inplace)


@pytest.mark.parametrize("f", [1, 8, 13, 20])
@pytest.mark.parametrize("tokens", [1, 90])
def test_linattn_fraction_widths(mods, seed, f, tokens):
    check_lin(mods, seed, 2, tokens, 2, 20, 18, f=f)


@pytest.mark.parametrize("tokens", [1, 64])
def test_linattn_many_heads(mods, seed, tokens):
    check_lin(mods, seed, 2, tokens, 256, 3, 5, calls=1, decays=[(h * 16) % 4097 for h in range(256)])


@pytest.mark.parametrize("seqs,tokens,heads", [(1, 150, 6), (3, 65, 7)])
def test_linattn_passes(mods, seed, seqs, tokens, heads):
    """More than a small workspace holds: passes over chunks, and over heads."""
    check_lin(mods, seed, seqs, tokens, heads, 256, 250, small=True, inplace=True)


# several chunks a pass and passes behind them (2, 2 and 1 chunks, 2 and 2), a short last chunk; passes over heads, a chunk each (see tests/test_block_shapes.py)
PASSES = [(16, 300, 16, 8, 9), (5, 200, 16, 64, 50), (3, 65, 7, 256, 250)]


@pytest.mark.parametrize("seqs,tokens,heads,dk,dv", PASSES)
@pytest.mark.parametrize("state,inplace", [(True, True), (True, False), (False, False)])
def test_linattn_state_from_pass_to_pass(mods, seed, seqs, tokens, heads, dk, dv, state, inplace):
    """The first pass takes the given state or zeros, the later ones what the one before has left."""
    check_lin(mods, seed, seqs, tokens, heads, dk, dv, state=state, inplace=inplace, calls=1, small=True)


@pytest.mark.parametrize("tokens", [1, 70])
def test_linattn_words_of_any_size(mods, seed, tokens):
    """Words over the whole ring: sums wrap, results are what the protocol makes of them on both sides."""
    o, g = pair(mods, seed)
    rng = np.random.default_rng(tokens)
    parts = [rng.integers(0, (1 << 64) - 1, size=n, dtype=np.uint64) for n in (tokens * 24, tokens * 24, tokens * 20, 240)]
    both = [(o.share(a), g.share_a(a)) for a in parts]
    layer = g.linattn_create([0.9, 1.0], 12, 10)
    yo, So = o.linattn_forward(*[t[0] for t in both], [3686, 4096], 1, tokens, 12, 10)
    y, S = g.linattn_forward(layer, *[t[1] for t in both[:3]], tokens=tokens, state=both[3][1])
    same(y, yo); same(S, So)
    layer.close(); g.close()


def test_linattn_no_tokens(mods, seed):
    o, g = pair(mods, seed)
    S = pl.fixed(np.random.default_rng(0), 16, 1.0, 2, 3, 4, 5)
    So, Sg = shared(o, g, S)
    layer = g.linattn_create([0.5] * 3, 4, 5)
    e = g.share_a(np.zeros(0, dtype=np.uint64))
    none = o.share(np.zeros(0, dtype=np.uint64))
    for given in (Sg, None):
        wo, ws = o.linattn_forward(none, none, none, So if given is not None else None, [2048] * 3, 2, 0, 4, 5)
        y, got = g.linattn_forward(layer, e, e, e, seqs=2, tokens=0, state=given)
        assert y.n == 0
        same(got, ws)
    y, got = g.linattn_forward(layer, e, e, e, seqs=2, tokens=0, state=Sg, inplace=True)
    o.linattn_forward(none, none, none, So, [2048] * 3, 2, 0, 4, 5)
    same(got, So)
    same_stats(o, g)
    layer.close(); g.close()


def test_behind_the_outputs(mods, seed):
    """Words behind the last row, the last state and the last gradient stay as they were."""
    import torch
    _, gtree = mods
    g = gtree.GTree(seed)
    rng = np.random.default_rng(4)

    def guarded(n):
        t = torch.full((3, 2, n + 64), 77, dtype=torch.int64, device="cuda")
        return t, gtree.Shares(n, "cuda", t)

    layer, rows, din, ff = g.linattn_create([0.7, 0.9], 5, 9), 3, 6, 11
    made, real = [], g._out
    g._out = lambda n: made.append(guarded(n)) or made[-1][1]
    x = [gtree.Shares(n, "cuda", torch.randint(0, 99, (3, 2, n), device="cuda")) for n in (3 * 70 * 10, 3 * 70 * 10, 3 * 70 * 18)]
    g.linattn_forward(layer, *x, seqs=3, tokens=70)
    w = [real(n) for n in (din * ff, din * ff, rows * din, rows * ff)]
    for t in w:
        t.t.random_(0, 99)
    gl = g.gated_create(w[0], w[1], din, ff)
    _, kept = g.gated_forward(gl, w[2], rows, keep=True)
    g.gated_backward(gl, w[2], w[3], rows, kept)
    assert len(made) == 11
    for t, s in made:
        assert bool((t[:, :, s.n:] == 77).all())
    layer.close(); gl.close(); g.close()


class Block:
    """Attention and gated layer as they are used together: a projection to queries, keys and values, attention, its projection beside the residual, the
    gated layer, its projection beside the residual."""

    def __init__(self, o, g, d, heads, dk, dv, ff, seed=0):
        rng = np.random.default_rng(seed)
        self.o, self.g, self.dims = o, g, (d, heads, dk, dv, ff)
        shapes = dict(qkv=(d, heads * (2 * dk + dv)), out=(heads * dv, d), gate=(d, ff), up=(d, ff), down=(ff, d))
        self.w = {k: shared(o, g, pl.fixed(rng, 16, 0.6 * s[0] ** -0.5, *s)) for k, s in shapes.items()}
        self.decay = (DECAYS * heads)[:heads]
        self.layer = {k: g.dense_create(self.w[k][1], *shapes[k]) for k in ("qkv", "out", "down")}
        self.gated = g.gated_create(self.w["gate"][1], self.w["up"][1], d, ff)
        self.attention = g.linattn_create([t / 4096 for t in self.decay], dk, dv)

    def here(self, x, state, seqs, tokens, inplace=False):
        g, n = self.g, seqs * tokens
        y, state = g.linattn_forward(self.attention, g.dense_forward(self.layer["qkv"], x, n), seqs=seqs, tokens=tokens, state=state, inplace=inplace)
        x = g.dense_forward(self.layer["out"], y, n, residual=x)
        return g.dense_forward(self.layer["down"], g.gated_forward(self.gated, x, n), n, residual=x), state

    def oracle(self, x, state, seqs, tokens):
        o, n, (d, heads, dk, dv, ff) = self.o, seqs * tokens, self.dims
        w = {k: v[0] for k, v in self.w.items()}
        rows = o.dense_forward(x, w["qkv"], n, d, heads * (2 * dk + dv))[0].reshape(3, n, -1)
        q, k, v = (np.ascontiguousarray(t).reshape(3, -1) for t in np.split(rows, [heads * dk, 2 * heads * dk], axis=2))
        y, state = o.linattn_forward(q, k, v, state, self.decay, seqs, tokens, dk, dv)
        x = o.dense_forward(y, w["out"], n, heads * dv, d, residual=x)[0]
        h = o.gated_forward(x, w["gate"], w["up"], n, d, ff)[0]
        return o.dense_forward(h, w["down"], n, ff, d, residual=x)[0], state


def test_block_prompt_and_tokens(mods, seed):
    """A prompt, then single tokens on its state."""
    o, g = pair(mods, seed)
    b = Block(o, g, 24, 3, 8, 10, 40)
    rng = np.random.default_rng(9)
    xo, xg = shared(o, g, pl.fixed(rng, 16, 1.0, 2 * 70, 24))
    yo, So = b.oracle(xo, None, 2, 70)
    yg, Sg = b.here(xg, None, 2, 70)
    same(yg, yo); same(Sg, So)
    for _ in range(3):
        xo, xg = shared(o, g, pl.fixed(rng, 16, 1.0, 2, 24))
        yo, So = b.oracle(xo, So, 2, 1)
        yg, Sg = b.here(xg, Sg, 2, 1, inplace=True)
        same(yg, yo); same(Sg, So)
    same_stats(o, g)
    g.close()


def test_block_in_a_graph(mods, seed):
    """Single tokens by a captured graph that carries its state from replay to replay, a larger eager call between them, against eager calls: values, not shares (every
    replay has keys of its own)."""
    import torch
    Oracle, gtree = mods
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        o, g = Oracle(seed), gtree.GTree(seed, stream=st)
        b = Block(o, g, 24, 3, 8, 10, 40)
        rng = np.random.default_rng(3)
        steps = [shared(o, g, pl.fixed(rng, 16, 1.0, 2, 24))[1] for _ in range(4)]
        x, S, zero = g.new(2 * 24), g.new(2 * 3 * 80), g.new(2 * 3 * 80)
        b.here(x, S, 2, 1)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            g.rekey()
            y, _ = b.here(x, S, 2, 1, inplace=True)
        S.t.zero_()
        state = zero
        for i, step in enumerate(steps):
            x.t.copy_(step.t)
            graph.replay()
            st.synchronize()
            got, kept = g.rec(y), g.rec(S)
            want, state = b.here(step, state, 2, 1)
            assert np.array_equal(got, g.rec(want)) and np.array_equal(kept, g.rec(state)), i
            big = shared(o, g, pl.fixed(rng, 16, 1.0, 2 * 70, 24))[1]
            b.here(big, None, 2, 70)                                         # the workspaces grow
            st.synchronize()
        g.close()


def test_refused_under_capture(mods, seed):
    """Calls that would have to allocate: refused, without a trace."""
    import torch
    _, gtree = mods
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        g = gtree.GTree(seed, stream=st)
        layer, gl = g.linattn_create([0.5], 4, 4), g.gated_create(g.new(4 * 9), g.new(4 * 9), 4, 9)
        q, S, y, h = g.new(12), g.new(16), g.new(8), g.new(9)
        st.synchronize()
        graph, got = torch.cuda.CUDAGraph(), []
        with torch.cuda.graph(graph, stream=st):
            op = g.op_counter()
            r = gtree._ref
            got.append(g.L.gt_linattn_forward(g.ctx, layer.h, r(q), r(q), r(q), 0, 1, 2, None, r(S), r(y)))
            got.append(g.L.gt_gated_forward(g.ctx, gl.h, r(q), 1, 1, r(h), None, None, None))
            got.append(g.L.gt_gated_backward(g.ctx, gl.h, None, r(h), r(h), r(h), r(h), 1, r(q), None, None, None, None))
            got.append(g.op_counter() - op)
            g.rekey()
        assert got == [gtree.GT_ESTATE] * 3 + [0]
        g.linattn_forward(layer, q, q, q)
        st.synchronize()
        g.close()


def test_another_stream_and_planes_of_odd_alignment(mods, seed):
    """Work on the context's own stream; planes that start 8 but not 16 bytes aligned; q, k and v as parts of rows of an odd length; q and k the same words."""
    import torch
    Oracle, gtree = mods
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        o, g = Oracle(seed), gtree.GTree(seed, stream=st)
        rng = np.random.default_rng(6)

        def odd(s):
            t = torch.empty((3, 2, s.n + 3 - s.n % 2), dtype=torch.int64, device="cuda")[:, :, 1:s.n + 1]
            t.copy_(s.t)
            return gtree.Shares(s.n, t=t)

        for rows in (3, 300):
            x, Wg, Wu, dh = (shared(o, g, pl.fixed(rng, 16, 0.5, *s)) for s in ((rows, 21), (21, 113), (21, 113), (rows, 113)))
            layer = g.gated_create(odd(Wg[1]), odd(Wu[1]), 21, 113)
            want = o.gated_forward(x[0], Wg[0], Wu[0], rows, 21, 113)
            h, kept = g.gated_forward(layer, odd(x[1]), rows, keep=True)
            same(h, want[0])
            got = g.gated_backward(layer, odd(x[1]), odd(dh[1]), rows, tuple(odd(t) for t in kept))
            for a, b in zip(got, o.gated_backward(x[0], Wg[0], Wu[0], dh[0], rows, 21, 113, want[1:])):
                same(a, b)
            layer.close()
        for tokens in (1, 64, 67):
            q, v = (shared(o, g, pl.fixed(rng, 16, 0.5, *s)) for s in ((tokens, 2 * 33), (tokens, 2 * 31)))
            S = shared(o, g, pl.fixed(rng, 16, 0.5, 2, 33, 31))
            layer = g.linattn_create([0.7, 1.0], 33, 31)
            yo, So = o.linattn_forward(q[0], q[0], v[0], S[0], [2867, 4096], 1, tokens, 33, 31)
            y, Sg = g.linattn_forward(layer, odd(q[1]), odd(q[1]), odd(v[1]), tokens=tokens, state=odd(S[1]))
            same(y, yo); same(Sg, So)
            n, ld = tokens, 2 * 33 * 2 + 2 * 31
            rows = np.concatenate([t.reshape(3, n, -1) for t in (q[0], q[0], v[0])], 2).reshape(3, -1)
            t = torch.from_numpy(np.stack([rows, np.roll(rows, -1, 0)], 1).view(np.int64)).cuda()
            yo, So = o.linattn_forward(q[0], q[0], v[0], So, [2867, 4096], 1, tokens, 33, 31)
            y, Sg = g.linattn_forward(layer, odd(gtree.Shares(n * ld, t=t)), tokens=tokens, state=Sg, inplace=True)
            same(y, yo); same(Sg, So)
            layer.close()
        st.synchronize()
        g.close()


def test_two_graphs_of_one_context(mods, seed):
    """Two captured graphs share the context's workspaces: replayed in turns, with eager calls between them, each gives the eager values."""
    import torch
    _, gtree = mods
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        g = gtree.GTree(seed, stream=st)
        rng = np.random.default_rng(8)
        s = lambda *shape: g.share_a(pl.words(pl.fixed(rng, 16, 0.5, *shape)))  # noqa: E731
        rows, din, ff = 250, 30, 70
        layer, att = g.gated_create(s(din, ff), s(din, ff), din, ff), g.linattn_create([0.9, 0.5], 10, 15)
        x, dh, qkv, S = s(rows, din), s(rows, ff), s(rows, 2 * 35), s(2, 10, 15)

        def first():
            h, kept = g.gated_forward(layer, x, rows, keep=True)
            return [h, *kept, *g.gated_backward(layer, x, dh, rows, kept)]

        def second():
            return list(g.linattn_forward(att, qkv, seqs=1, tokens=rows, state=S))

        want = [[g.rec(t) for t in f()] for f in (first, second)]
        graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
        for graph, f in zip(graphs, (first, second)):
            with torch.cuda.graph(graph, stream=st):
                g.rekey()
                outs.append(f())
        for turn in range(3):
            for i in (0, 1, 1, 0):
                for t in outs[i]:
                    t.t.zero_()
                graphs[i].replay()
                st.synchronize()
                for a, b in zip(outs[i], want[i]):
                    assert np.array_equal(g.rec(a), b), (turn, i)
            first() if turn else second()
        g.close()


def test_offsets_past_32_bits(mods, seed):
    """Planes of more than 4 GiB, several passes: with decays of zero and zero states the last tokens' values are those of a call on them alone."""
    import torch
    _, gtree = mods
    g = gtree.GTree(seed)
    tokens, heads, d, last = 1 << 17, 33, 128, 128
    n = tokens * heads * d
    assert n * 8 > 1 << 32
    own = torch.randint(-(1 << 16), 1 << 16, (3, n), device="cuda")
    t = torch.empty((3, 2, n), dtype=torch.int64, device="cuda")
    for p in range(3):
        t[p, 0], t[p, 1] = own[p], own[(p + 1) % 3]
    del own
    x = gtree.Shares(n, t=t)
    layer = g.linattn_create([0.0] * heads, d, d)
    o, S = g.linattn_forward(layer, x, x, x, tokens=tokens)
    tail = gtree.Shares(last * heads * d, t=t[:, :, n - last * heads * d:].contiguous())
    want, state = g.linattn_forward(layer, tail, tail, tail, tokens=last)
    got = gtree.Shares(tail.n, t=o.t[:, :, n - tail.n:].contiguous())
    assert np.array_equal(g.rec(got), g.rec(want)) and np.array_equal(g.rec(S), g.rec(state))
    layer.close(); g.close()
