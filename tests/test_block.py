"""The protocols of the gated layer and of linear attention (oracle) against Python integers, against the formulas in real numbers, at the sizes and
values where they can go wrong, and their message counts."""
import numpy as np
import pytest

import plain_block as pb
import plain_layers as pl
from oracle import Oracle


def shared(o, *arrays):
    return [None if a is None else o.share(pl.words(a)) for a in arrays]


def gated_inputs(f, rows, din, ff, bias, seed=0):
    rng = np.random.default_rng(seed + 31 * rows + din + ff)
    x, Wg, Wu = pl.fixed(rng, f, 1.0, rows, din), pl.fixed(rng, f, 1.0, din, ff), pl.fixed(rng, f, 1.0, din, ff)
    return (x, Wg, Wu) + ((pl.fixed(rng, f, 1.0, ff), pl.fixed(rng, f, 1.0, ff)) if bias else (None, None))


@pytest.mark.parametrize("rows,din,ff", [(1, 1, 1), (1, 7, 9), (3, 1, 5), (2, 33, 17), (9, 5, 8), (0, 4, 3)])
@pytest.mark.parametrize("relu,bias", [(False, False), (True, True), (True, False)])
@pytest.mark.parametrize("f", [1, 12, 20])
def test_gated_forward(seed, rows, din, ff, relu, bias, f):
    x, Wg, Wu, bg, bu = gated_inputs(f, rows, din, ff, bias)
    o = Oracle(seed, tau=f)
    X, G, U, b, c = shared(o, x, Wg, Wu, bg, bu)
    before, rounds = o.wire_bits(), o.stats()[0]
    op = o.op_counter()
    got = o.gated_forward(X, G, U, rows, din, ff, bg=b, bu=c, relu=relu)
    want = pb.gated(x, Wg, Wu, f, bg, bu, relu)
    for a, w in zip(got, want[:4 if relu else 3]):
        assert np.array_equal(o.rec(a), pl.words(w))
    assert o.op_counter() == op + 3 and o.stats()[0] == rounds + (14 if relu else 12)
    bits, n = o.wire_bits() - before, rows * ff
    # three openings to both others, trees and conversions, with ReLU the wider tree, the sign's conversion and the product
    assert bits[0][1] == n * (3 * 65 + (1 if relu else 0)) and bits[0][2] == n * (3 * 94 + (95 if relu else 0))


@pytest.mark.parametrize("rows,din,ff", [(1, 1, 1), (5, 7, 9), (2, 33, 17), (9, 5, 8), (0, 4, 3)])
@pytest.mark.parametrize("relu", [False, True])
def test_gated_backward(seed, rows, din, ff, relu):
    f = 12
    x, Wg, Wu, _, _ = gated_inputs(f, rows, din, ff, False)
    rng = np.random.default_rng(rows)
    dh = pl.fixed(rng, f, 0.5, rows, ff)
    _, g, u, s = pb.gated(x, Wg, Wu, f, relu=relu)
    s = s if relu else None
    o = Oracle(seed, tau=f)
    X, G, U, D, gs, us, ss = shared(o, x, Wg, Wu, dh, g, u, s)
    op, rounds = o.op_counter(), o.stats()[0]
    got = o.gated_backward(X, G, U, D, rows, din, ff, (gs, us, ss))
    for a, w in zip(got, pb.gated_back(x, Wg, Wu, dh, g, u, s, f)):
        assert np.array_equal(o.rec(a), pl.words(w))
    assert o.op_counter() == op + 5 and o.stats()[0] == rounds + (7 if relu else 6) + 18


@pytest.mark.parametrize("f", [1, 9, 20])
@pytest.mark.parametrize("relu", [False, True])
def test_gated_backward_fraction_widths(seed, f, relu):
    rows, din, ff = 5, 7, 9
    x, Wg, Wu, _, _ = gated_inputs(f, rows, din, ff, False)
    dh = pl.fixed(np.random.default_rng(f), f, 0.5, rows, ff)
    _, g, u, s = pb.gated(x, Wg, Wu, f, relu=relu)
    s = s if relu else None
    o = Oracle(seed, tau=f)
    X, G, U, D, gs, us, ss = shared(o, x, Wg, Wu, dh, g, u, s)
    for a, w in zip(o.gated_backward(X, G, U, D, rows, din, ff, (gs, us, ss)), pb.gated_back(x, Wg, Wu, dh, g, u, s, f)):
        assert np.array_equal(o.rec(a), pl.words(w))


def test_gated_gradients_against_differences(seed):
    """Gradients of sum(h c) against central differences of the real function.  A value of the backward pass is rounded by at most half a word per
    completion: with two factors of at most M in absolute value and K terms it is off by K M / 2 + 1 words; the differences of a bilinear function are exact but for
    rounding in double precision, away from ReLU's corner."""
    f, rows, din, ff = 16, 4, 5, 6
    x, Wg, Wu, bg, bu = gated_inputs(f, rows, din, ff, True, seed=3)
    rng = np.random.default_rng(5)
    c = pl.fixed(rng, f, 1.0, rows, ff)
    _, g, u, s = pb.gated(x, Wg, Wu, f, bg, bu)
    real = [np.asarray(a, dtype=np.float64) / 2.0 ** f for a in (x, Wg, Wu, bg, bu, c)]

    def loss(x, Wg, Wu, bg, bu):
        return float((np.maximum(x @ Wg + bg, 0) * (x @ Wu + bu) * real[5]).sum())

    assert np.abs(real[0] @ real[1] + real[3]).min() > 1e-3               # no value within a step of the corner
    o = Oracle(seed, tau=f)
    X, G, U, D, gs, us, ss = shared(o, x, Wg, Wu, c, g, u, s)
    got = o.gated_backward(X, G, U, D, rows, din, ff, (gs, us, ss))
    most = max(np.abs(a).max() for a in real)
    # dg and du are off by half a word each and by that of g and u times c; sums of at most 2 ff or rows of them times a factor of at most `most`; one more rounding
    off = (max(2 * ff, rows) * (0.5 + 0.5 * most) * most + 1) / 2.0 ** f + 1e-9
    for i, a in zip((0, 1, 2, 3, 4), got):
        value = (o.rec(a).astype(np.int64) / 2.0 ** f).reshape(real[i].shape)
        for at in np.ndindex(real[i].shape):
            step = [t.copy() for t in real[:5]]
            h = 1e-4
            step[i][at] += h
            up = loss(*step)
            step[i][at] -= 2 * h
            assert abs((up - loss(*step)) / (2 * h) - value[at]) <= off + 1e-6, (i, at)


LIN = [(1, 1, 1, 1, 1), (1, 1, 3, 5, 9), (2, 1, 2, 8, 16), (1, 2, 1, 3, 2), (2, 63, 1, 4, 3), (1, 64, 2, 2, 5), (1, 65, 1, 3, 9), (2, 130, 2, 2, 1)]


def lin_inputs(f, seqs, tokens, heads, dk, dv, seed=0):
    rng = np.random.default_rng(seed + tokens * 17 + dk + dv)
    return (pl.fixed(rng, f, 1.0, seqs, tokens, heads, dk), pl.fixed(rng, f, 1.0, seqs, tokens, heads, dk), pl.fixed(rng, f, 1.0, seqs, tokens, heads, dv),
            pl.fixed(rng, f, 1.0, seqs, heads, dk, dv))


DECAYS = [4096, 0, 3900, 1, 4095]


@pytest.mark.parametrize("seqs,tokens,heads,dk,dv", LIN)
@pytest.mark.parametrize("f", [1, 13, 20])
def test_linear_attention(seed, seqs, tokens, heads, dk, dv, f):
    q, k, v, S = lin_inputs(f, seqs, tokens, heads, dk, dv)
    for first in range(0, 5, heads):
        decay = (DECAYS[first:] + DECAYS)[:heads]
        o = Oracle(seed, tau=f)
        sh = shared(o, q, k, v, S)
        op, rounds, before = o.op_counter(), o.stats()[0], o.wire_bits()
        out, state = o.linattn_forward(*sh, decay, seqs, tokens, dk, dv)
        want, last = pb.linattn(q, k, v, S, decay, f)
        assert np.array_equal(o.rec(out), pl.words(want)) and np.array_equal(o.rec(state), pl.words(last))
        chunks = (tokens + 63) // 64
        n = seqs * heads * (sum(c * (c + 1) // 2 for c in [64] * (tokens // 64) + [tokens % 64]) + chunks * dk * dv + tokens * dv)
        bits = o.wire_bits() - before
        assert o.op_counter() == op + 3 and o.stats()[0] == rounds + 6 * max(2, chunks)
        assert bits[0][1] == 65 * n and bits[0][2] == 94 * n


def test_no_tokens(seed):
    S = lin_inputs(16, 2, 1, 1, 3, 4)[3]
    o = Oracle(seed, tau=16)
    empty, state = np.zeros((3, 0), dtype=np.uint64), shared(o, S)[0]
    out, got = o.linattn_forward(empty, empty, empty, state, [4000], 2, 0, 3, 4)
    assert out.size == 0 and np.array_equal(got, state) and o.stats()[0] == 0


def test_chunks_are_the_recurrence(seed):
    """A prompt in one call and token by token, against the recurrence in real numbers.  In words: a state is rounded by half a word a token (or chunk), which later tokens see
    at most decayed: at most T / 2; its decay is exact token by token, and off by at most 2^-13 in a chunk's power; an output adds dk of these times |q|."""
    f, T, dk, dv, w = 16, 100, 6, 5, 4000
    q, k, v, S = lin_inputs(f, 1, T, 1, dk, dv)
    o = Oracle(seed, tau=f)
    sh = shared(o, q, k, v, S)
    whole, last = o.linattn_forward(*sh, [w], 1, T, dk, dv)
    state, rows = sh[3], []
    for t in range(T):
        one = shared(o, q[:, t:t + 1], k[:, t:t + 1], v[:, t:t + 1])
        y, state = o.linattn_forward(*one, state, [w], 1, 1, dk, dv)
        rows.append(o.rec(y).astype(np.int64))
    Q, K, V, R = (np.asarray(a[0, ...], dtype=np.float64) / 2.0 ** f for a in (q, k, v, S))
    R, want, biggest, reach = R[0], [], 0.0, 0.0
    for t in range(T):
        R = (w / 4096) * R + np.outer(K[t, 0], V[t, 0])
        want.append(Q[t, 0] @ R)
        biggest = max(biggest, np.abs(R).max())
        reach = max(reach, np.abs(Q[t, 0]).sum())
    one = T / 2 / 2.0 ** f
    # a chunk's exponents are off by 2^-13 each: of the state before, and of up to 64 terms k v and scores q k
    terms = np.abs(K).max() * np.abs(V).max()
    many = (2 * biggest + 64 * terms) * 2.0 ** -13 * 2 + 4 / 2.0 ** f
    score = 64 * (np.abs(Q).max() * np.abs(K).max() * dk * 2.0 ** -13 + 2.0 ** -17) * np.abs(V).max()
    for got, off in ((o.rec(state), one), (o.rec(last), many)):
        assert np.abs(got.astype(np.int64).reshape(dk, dv) / 2.0 ** f - R).max() <= off
    want = np.array(want)
    # (a token's own score is rounded by half a word, times |v|)
    assert np.abs(np.array(rows) / 2.0 ** f - want).max() <= reach * one + (np.abs(V).max() + 1) / 2.0 ** f
    assert np.abs(o.rec(whole).astype(np.int64).reshape(T, dv) / 2.0 ** f - want).max() <= reach * many + score + 2.0 ** -f


@pytest.mark.parametrize("f", [8, 16, 20])
@pytest.mark.parametrize("w", [0, 2048, 3900, 4095, 4096])
@pytest.mark.parametrize("size", [1, 64])
def test_how_far_a_prompt_is_from_the_recurrence(seed, f, w, size):
    """Against the recurrence in real numbers, term by term.  A power of the decay is off by at most d = 2^-13 (12 fraction bits, from 46, whose own roundings add less than
    2^-40), of a single token by nothing; every completion by r = 2^-(f+1).  So with e the state's error, P_ij = q_i k_j in real numbers:
      an output by    sum_j (d |P_ij| + r) |v_j| + sum |q_i| (d (|S| + e) + D[i+1] e) + r
      a state by      d (|S| + e) + D[c] e + sum_j d |k_j v_j| + r
    and the sums in double precision by less than 2^-40 of theirs."""
    T, dk, dv = 128, 6, 4
    q, k, v, S = lin_inputs(f, 1, T, 1, dk, dv, seed=w)
    o = Oracle(seed, tau=f)
    shares = shared(o, q, k, v, S)
    if size == 1:
        state, rows = shares[3], []
        for t in range(T):
            y, state = o.linattn_forward(*shared(o, q[:, t], k[:, t], v[:, t]), state, [w], 1, 1, dk, dv)
            rows.append(o.rec(y))
        got = np.concatenate(rows)
    else:
        y, state = o.linattn_forward(*shares, [w], 1, T, dk, dv)
        got = o.rec(y)
    Q, K, V = (np.asarray(a[0, :, 0], dtype=np.float64) / 2.0 ** f for a in (q, k, v))
    R, e, decay, r = np.asarray(S[0, 0], dtype=np.float64) / 2.0 ** f, np.zeros((dk, dv)), w / 4096, 2.0 ** -(f + 1)
    d = 0.0 if size == 1 else 2.0 ** -13 + 2.0 ** -40
    want, off = np.zeros((T, dv)), np.zeros((T, dv))
    for t0 in range(0, T, size):
        qc, kc, vc = Q[t0:t0 + size], K[t0:t0 + size], V[t0:t0 + size]
        n = np.arange(size)
        low = np.tri(size)
        P, D = qc @ kc.T, decay ** (n + 1.0)[:, None]
        want[t0:t0 + size] = (P * low * decay ** np.maximum(n[:, None] - n, 0)) @ vc + D * (qc @ R)
        off[t0:t0 + size] = ((d * np.abs(P) + r) * low) @ np.abs(vc) + d * (np.abs(qc) @ (np.abs(R) + e)) + D * (np.abs(qc) @ e) + r
        e = d * (np.abs(R) + e) + decay ** size * e + d * (np.abs(kc).T @ np.abs(vc)) + r
        R = decay ** size * R + (kc * decay ** (size - 1.0 - n)[:, None]).T @ vc
    slack = 2.0 ** -40 * (np.abs(want).max() + np.abs(R).max() + dk * T)
    assert (np.abs(got.astype(np.int64).reshape(T, dv) / 2.0 ** f - want) <= off + slack).all()
    assert (np.abs(o.rec(state).astype(np.int64).reshape(dk, dv) / 2.0 ** f - R) <= e + slack).all()
