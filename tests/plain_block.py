"""The gated layer and linear attention in Python integers: what the shares of their results have to stand for."""
import numpy as np

from plain_layers import scaled

CHUNK, DECAY = 64, 12


def gated(x, Wg, Wu, f, bg=None, bu=None, relu=True):
    """(h, g, u, s) of object matrices; g after the activation."""
    g = scaled(x.dot(Wg) + (0 if bg is None else bg * (1 << f)), f)
    u = scaled(x.dot(Wu) + (0 if bu is None else bu * (1 << f)), f)
    s = np.array([int(t >= 0) for t in g.reshape(-1)], dtype=object).reshape(g.shape)
    if relu:
        g = g * s
    return scaled(g * u, f), g, u, s


def gated_back(x, Wg, Wu, dh, g, u, s, f):
    """(dx, dWg, dWu, dbg, dbu); s None: no activation."""
    dg, du = scaled(dh * u, f) * (1 if s is None else s), scaled(dh * g, f)
    return scaled(dg.dot(Wg.T) + du.dot(Wu.T), f), scaled(x.T.dot(dg), f), scaled(x.T.dot(du), f), dg.sum(0), du.sum(0)


def powers(w):
    """decay^n, n <= 64, with 12 fraction bits, rounded from 46."""
    E, out = 1 << 46, []
    for _ in range(CHUNK + 1):
        out.append((E + (1 << 33)) >> 34)
        E = (E * int(w) + (1 << 11)) >> 12
    return out


def linattn(q, k, v, S, decay, f):
    """(o, state): q, k seqs x tokens x heads x dk, v ... x dv, S seqs x heads x dk x dv, object arrays."""
    seqs, T, H, dk = q.shape
    o, S, s = np.zeros(v.shape, dtype=object), S.copy(), f + DECAY
    for b in range(seqs):
        for h in range(H):
            D = powers(decay[h])
            for t in range(0, T, CHUNK):
                qc, kc, vc = q[b, t:t + CHUNK, h], k[b, t:t + CHUNK, h], v[b, t:t + CHUNK, h]
                n = len(qc)
                gap = [[D[i - j] if j <= i else 0 for j in range(n)] for i in range(n)]
                P = scaled(qc.dot(kc.T) * np.array(gap, dtype=object), s) * np.tri(n, dtype=int).astype(object)
                before = np.array(D[1:n + 1], dtype=object)[:, None]
                o[b, t:t + CHUNK, h] = scaled(P.dot(vc) * (1 << DECAY) + qc.dot(S[b, h]) * before, s)
                age = np.array(D[:n][::-1], dtype=object)[:, None]
                S[b, h] = scaled(S[b, h] * D[n] * (1 << f) + (kc * age).T.dot(vc), s)
    return o, S
