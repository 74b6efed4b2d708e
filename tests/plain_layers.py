"""Layers in Python integers: what the shares of a layer's results have to stand for (no shares, no rounding but the definition's)."""
import numpy as np

M64 = (1 << 64) - 1


def signed(a):
    """uint64 words -> Python integers in [-2^63, 2^63)."""
    return np.asarray(a, dtype=np.uint64).astype(np.int64).astype(object)


def words(a):
    """Integers -> uint64 words modulo 2^64."""
    return np.array([int(v) & M64 for v in np.asarray(a, dtype=object).reshape(-1)], dtype=np.uint64)


def scaled(v, f):
    """floor((v + 2^(f-1)) / 2^f) of an object array."""
    return np.array([(int(x) + (1 << (f - 1))) >> f for x in v.reshape(-1)], dtype=object).reshape(v.shape)


def forward(x, W, f, b=None, relu=False, res=None):
    """(y, gate) of object matrices."""
    v = x.dot(W)
    if b is not None:
        v = v + b * (1 << f)
    y = scaled(v, f)
    gate = np.array([int(t >= 0) for t in y.reshape(-1)], dtype=object).reshape(y.shape)
    if relu:
        y = y * gate
    return (y if res is None else y + res), gate


def backward(x, W, dy, f, gate=None):
    dz = dy if gate is None else dy * gate
    return scaled(dz.dot(W.T), f), scaled(x.T.dot(dz), f), dz.sum(0)


def moe(x, Wr, W1, W2, f, top, br=None, b1=None, b2=None, res=None):
    """Wr d x E, W1 E x d x ff, W2 E x ff x d."""
    s, _ = forward(x, Wr, f, br, True)
    E = Wr.shape[1]
    y = np.zeros(x.shape, dtype=object)
    for t in range(x.shape[0]):
        total = np.zeros(x.shape[1], dtype=object)
        for a in sorted(range(E), key=lambda a: (-s[t, a], a))[:top]:
            g = (int(s[t, a]) << f) // (1 + int(s[t].sum()))
            h, _ = forward(x[t:t + 1], W1[a], f, None if b1 is None else b1[a], True)
            total = total + scaled(h * g, f).dot(W2[a])[0] + (0 if b2 is None else b2[a] * g)
        y[t] = scaled(total, f)
    return y if res is None else y + res


def fixed(rng, f, std, *shape):
    """Normal fixed-point values as an object array."""
    return np.round(rng.normal(0.0, std * 2.0 ** f, size=shape)).astype(np.int64).astype(object)
