"""Layers of a small network on 2-out-of-3 shares over Z_2^64, as measurable cases: the matrix product with bias, activation and
residual in its epilogue (forward, and its backward pass), and a mixture-of-experts layer for a few tokens.

Everything is fixed point with tau fraction bits and exact: an output value is floor((v + 2^(tau-1)) / 2^tau) of the integer sum v.  Shares in,
shares out: every party multiplies the components that it holds, sums are opened under a mask, bits come back as daBits, all randomness is
a function of the keys, the operation id and the element.  So outputs are whole numbers, the shares themselves (six planes, a party's own and next component)
and the values that they stand for, and have to be equal.  A state counts its operation ids, as a context does.

The plain form follows the protocol on the components with torch's elementwise operations and products in 64 bits (a ring product is six exact products of
22-bit digits); a comparison's bit, which the protocol finds by a tree of ANDs on shares, is taken from the opened and the dealer's word.

Sizes: 294 columns are those of the discretised census table, 22 and 267 those of the heart data of this repository's workloads; the others are generic.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
# keys: three pairwise ones, the dealer's, the owner's, four words each
KEYS = [[(0x9E3779B97F4A7C15 * (4 * k + i + 1)) & ((1 << 64) - 1) for i in range(4)] for k in range(5)]


def listed():
    F, B, M = "forward", "backward", "moe"
    return [
        # one token through a small layer: launches and rounds count
        dict(name="dense-token", kind=F, rows=1, din=64, dout=64, relu=True, bias=True, residual=True, gate=False, tau=16),
        # one token through a wide layer: the weights' bytes count
        dict(name="dense-token-wide", kind=F, rows=1, din=1024, dout=4096, relu=True, bias=True, residual=False, gate=False, tau=16),
        # a handful of census rows, odd sizes, fewer fraction bits, no activation
        dict(name="dense-ragged", kind=F, rows=33, din=294, dout=257, relu=False, bias=True, residual=True, gate=False, tau=13),
        # a batch of a training step: the activation's bits are kept for the backward pass
        dict(name="dense-batch", kind=F, rows=1000, din=294, dout=512, relu=True, bias=True, residual=False, gate=True, tau=16),
        # the second product of a block on a long prompt
        dict(name="dense-residual", kind=F, rows=2048, din=1024, dout=1024, relu=False, bias=False, residual=True, gate=False, tau=16),
        # the first product of a block on a long prompt: the largest
        dict(name="dense-long", kind=F, rows=2048, din=1024, dout=4096, relu=True, bias=True, residual=False, gate=False, tau=16),
        # a training step's gradients on the heart table
        dict(name="grad-small", kind=B, rows=267, din=22, dout=16, relu=True, tau=16),
        # ... on census rows with an odd width
        dict(name="grad-census", kind=B, rows=1000, din=294, dout=257, relu=True, tau=16),
        # ... of a large layer
        dict(name="grad-large", kind=B, rows=2048, din=1024, dout=1024, relu=False, tau=16),
        # one token through eight experts: serving
        dict(name="moe-token", kind=M, rows=1, d=256, ff=1024, experts=8, top=1, bias=True, residual=True, tau=16),
        # a few tokens, odd sizes, two of five experts
        dict(name="moe-ragged", kind=M, rows=5, d=65, ff=130, experts=5, top=2, bias=True, residual=False, tau=14),
        # a few tokens through two of sixteen larger experts
        dict(name="moe-large", kind=M, rows=8, d=512, ff=2048, experts=16, top=2, bias=False, residual=True, tau=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(("forward", "forward", "backward", "moe"))
        tau, flip = rng.randint(8, 20), lambda: rng.random() < 0.5  # noqa: E731
        if kind == "forward":
            c = dict(kind=kind, rows=_log(rng, 1, 2048), din=_log(rng, 1, 2048), dout=_log(rng, 1, 4096), relu=flip(), bias=flip(), residual=flip(),
                     gate=False, tau=tau)
            c["gate"] = c["relu"] and flip()
        elif kind == "backward":
            c = dict(kind=kind, rows=_log(rng, 1, 2048), din=_log(rng, 1, 1024), dout=_log(rng, 1, 1024), relu=flip(), tau=tau)
        else:
            experts = rng.randint(1, 16)
            c = dict(kind=kind, rows=_log(rng, 1, 16), d=_log(rng, 16, 512), ff=_log(rng, 16, 2048), experts=experts,
                     top=rng.randint(1, min(3, experts)), bias=flip(), residual=flip(), tau=tau)
        if _cost(c) <= most:
            return c


# ---- inputs ------------------------------------------------------------------------------
def _values(c, seed):
    """Fixed-point inputs on the GPU from the seed alone, as a dict of int64 tensors."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (seed + 1) + 29)

    def fixed(std, *shape):
        return torch.round(torch.randn(shape, generator=g, device=DEV, dtype=torch.float64) * (std * 2.0 ** c["tau"])).to(torch.int64)

    n = c["rows"]
    if c["kind"] == "moe":
        d, ff, E = c["d"], c["ff"], c["experts"]
        v = dict(x=fixed(1.0, n, d), Wr=fixed(d ** -0.5, d, E), W1=fixed(d ** -0.5, E, d, ff), W2=fixed(ff ** -0.5, E, ff, d))
        if c["bias"]:
            v.update(br=fixed(0.1, E), b1=fixed(0.1, E, ff), b2=fixed(0.1, E, d))
        if c["residual"]:
            v["res"] = fixed(1.0, n, d)
        return v
    din, dout = c["din"], c["dout"]
    v = dict(x=fixed(1.0, n, din), W=fixed(din ** -0.5, din, dout))
    if c["kind"] == "backward":
        v["dy"] = fixed(0.1, n, dout)
        if c["relu"]:
            v["gate"] = torch.randint(0, 2, (n, dout), generator=g, device=DEV, dtype=torch.int64)
        return v
    if c["bias"]:
        v["b"] = fixed(0.1, dout)
    if c["residual"]:
        v["res"] = fixed(1.0, n, dout)
    return v


def _split(v, seed):
    """Components of fresh sharings, [3, ...] each: two uniform words, the third completes the sum."""
    g = torch.Generator(device=DEV)
    g.manual_seed(7000003 * (seed + 1) + 31)
    lo, hi = -(1 << 63), (1 << 63) - 1

    def one(t):
        a, b = (torch.randint(lo, hi, t.shape, generator=g, device=DEV, dtype=torch.int64) for _ in range(2))
        return torch.stack([a, b, t - a - b])

    return {k: one(t) for k, t in v.items()}


def _planes(comp):
    """Six planes [3, 2, n] of components [3, ...]: a party's own and its next one."""
    q = comp.reshape(3, -1)
    return torch.stack([q, q.roll(-1, 0)], 1).contiguous()


def prepare(c, seed):
    """Shared inputs and, of the framework, the context and the layer: what a program keeps."""
    comp = _split(_values(c, seed), seed)
    if not own:
        return dict(c=c, op=0, **comp)
    from paper_2305_00645_amd import gtree
    s = dict(c=c, g=gtree.GTree(KEYS, tau=c["tau"], device=DEV))
    for k, t in comp.items():
        s[k] = gtree.Shares(t[0].numel(), DEV, _planes(t))
    if c["kind"] == "moe":
        s["layer"] = s["g"].moe_create(s["Wr"], s["W1"], s["W2"], c["d"], c["ff"], c["experts"], c["top"], c["rows"],
                                       br=s.get("br"), b1=s.get("b1"), b2=s.get("b2"))
    else:
        s["layer"] = s["g"].dense_create(s["W"], c["din"], c["dout"], b=s.get("b"))
    torch.cuda.synchronize()
    return s


# ---- a pass -------------------------------------------------------------------------------
def run(s):
    c = s["c"]
    if not own:
        return {"moe": _plain_moe, "forward": _plain_forward, "backward": _plain_backward}[c["kind"]](s, c)
    g = s["g"]

    def out(**shares):
        r = {}
        for k, z in shares.items():
            r[k], r[k + "_shares"] = g.reconstruct_a(z), z.t
        return r

    if c["kind"] == "moe":
        return out(y=g.moe_forward(s["layer"], s["x"], c["rows"], residual=s.get("res")))
    if c["kind"] == "forward":
        if c["gate"]:
            y, gate = g.dense_forward(s["layer"], s["x"], c["rows"], relu=c["relu"], residual=s.get("res"), want_gate=True)
            return out(y=y, gate=gate)
        return out(y=g.dense_forward(s["layer"], s["x"], c["rows"], relu=c["relu"], residual=s.get("res")))
    dx, dW, db = g.dense_backward(s["layer"], s["x"], s["dy"], c["rows"], gate=s.get("gate"))
    return out(dx=dx, dW=dW, db=db)


# ---- the plain form ------------------------------------------------------------------------
def _rot(x, r):
    return (x << r) | ((x >> (32 - r)) & ((1 << r) - 1))


def _quarters(a, b, c, d):
    a = a + b
    d = _rot(d ^ a, 16)
    c = c + d
    b = _rot(b ^ c, 12)
    a = a + b
    d = _rot(d ^ a, 8)
    c = c + d
    b = _rot(b ^ c, 7)
    return a, b, c, d


def _signed(x, bits):
    x &= (1 << bits) - 1
    return x - (1 << bits) if x >> (bits - 1) else x


def _prf(key, blk, op, stream):
    """Words [n, 8] of the blocks blk [n] under a key: the ChaCha block function with eight rounds."""
    n = blk.numel()
    words = [0x61707865, 0x3320646E, 0x79622D32, 0x6B206574] + [(KEYS[key][i] >> s) & 0xFFFFFFFF for i in range(4) for s in (0, 32)]
    const = torch.tensor([_signed(w, 32) for w in words], dtype=torch.int32, device=DEV).view(3, 4, 1)
    low = ((blk << 32) >> 32).to(torch.int32)
    tail = torch.stack([low, (blk >> 32).to(torch.int32), torch.full_like(low, op), torch.full_like(low, stream)])
    a0, b0, c0 = (const[i].expand(4, n) for i in range(3))
    a, b, c, d = a0, b0, c0, tail
    for _ in range(4):
        a, b, c, d = _quarters(a, b, c, d)
        a, b, c, d = _quarters(a, b.roll(-1, 0), c.roll(-2, 0), d.roll(-3, 0))
        b, c, d = b.roll(1, 0), c.roll(2, 0), d.roll(3, 0)
    x = torch.cat([a + a0, b + b0, c + c0, d + tail]).to(torch.int64)
    return ((x[0::2] & 0xFFFFFFFF) | (x[1::2] << 32)).t()


def _zero(op, stream, n):
    """Arithmetic zero sharing of elements 0..n-1, [3, n]."""
    blk = torch.arange((n + 7) // 8, device=DEV)
    w = torch.stack([_prf(k, blk, op, stream).reshape(-1)[:n] for k in range(3)])
    return w - w.roll(-1, 0)


def _complete(a, b, total):
    return torch.stack([a, b, total - a - b])


def _public(x):
    return torch.stack([x, torch.zeros_like(x), torch.zeros_like(x)])


def _from_bit(bit, beta, share):
    """Arithmetic sharing of a bit from a daBit (beta and its sharing): the opened bit is bit xor beta."""
    f = bit ^ beta
    return torch.where(f.bool(), _public(torch.ones_like(bit)) - share, share)


def _dabit(op, n):
    D = _prf(3, torch.arange(n, device=DEV), op, 0)
    beta = D[:, 5] & 1
    return beta, _complete(D[:, 6], D[:, 7], beta)


def _local(x, y):
    """A party's part of an elementwise product: x_p y_p + x_{p+1} y_p + x_p y_{p+1}."""
    return x * (y + y.roll(-1, 0)) + x.roll(-1, 0) * y


def _mult(x, y, op, n):
    return _local(x, y) + _zero(op, 0, n).view(x.shape)


def _digits(x):
    """x = d0 + d1 2^22 + d2 2^44 modulo 2^64, digits in [-2^21, 2^21]."""
    r, got = x, []
    for _ in range(2):
        d = ((r + (1 << 21)) & ((1 << 22) - 1)) - (1 << 21)
        got.append(d.double())
        r = (r - d) >> 22
    return got + [(((r + (1 << 19)) & ((1 << 20) - 1)) - (1 << 19)).double()]


def _ring_product(a, b):
    """a [m, k] times b [k, n] modulo 2^64: exact products of digits in 64-bit floating point, 1024 terms at a time."""
    out = 0
    for k in range(0, a.shape[1], 1024):
        x, y = _digits(a[:, k:k + 1024]), _digits(b[k:k + 1024])
        low = (x[0] @ y[0]).to(torch.int64)
        mid = (x[0] @ y[1]).to(torch.int64) + (x[1] @ y[0]).to(torch.int64)
        top = (x[0] @ y[2]).to(torch.int64) + (x[1] @ y[1]).to(torch.int64) + (x[2] @ y[0]).to(torch.int64)
        out = out + low + (mid << 22) + (top << 44)
    return out


def _products(x, w):
    """The three parties' parts [3, m, n] of a matrix product of shared matrices [3, m, k] and [3, k, n]."""
    return torch.stack([_ring_product(torch.cat([x[p], x[(p + 1) % 3]], 1), torch.cat([w[p] + w[(p + 1) % 3], w[p]], 0)) for p in range(3)])


def _finish(z, op, f, relu=False):
    """Parts z [3, ...] of sums v to sharings of floor((v + 2^(f-1)) / 2^f), ReLU's bit taken from the same opened word."""
    shape = z.shape
    z = z.reshape(3, -1)
    n = z.shape[1]
    e = torch.arange(n, device=DEV)
    D, G = _prf(3, e, op, 0), _prf(3, e, op, 5)
    r, beta = D[:, 0], D[:, 5] & 1
    off = (1 << (f + 31)) if relu else (1 << 62)
    m = z + _zero(op, 0, n) + _complete(D[:, 1], D[:, 2], r)
    c = m.sum(0) + ((1 << (f - 1)) + off)
    low, high = (1 << f) - 1, (1 << (64 - f)) - 1
    borrow = _from_bit(((c & low) < (r & low)).to(torch.int64), beta, _complete(D[:, 6], D[:, 7], beta))
    shifted = _complete(G[:, 0], G[:, 1], (r >> f) & high)
    top = _complete(G[:, 2], G[:, 3], (r >> 63) & 1)
    y = torch.where(c < 0, 0, top << (64 - f)) - shifted - borrow + _public(((c >> f) & high) - (off >> f))
    if not relu:
        return y.view(shape), None
    beta = G[:, 6] & 1
    s = _from_bit(((c - r) >> (f + 31)) & 1, beta, _complete(G[:, 4], G[:, 5], beta))
    return (_local(s, y) + _zero(op, 3, n)).view(shape), s.view(shape)


def _out(**comp):
    r = {}
    for k, z in comp.items():
        r[k], r[k + "_shares"] = z.sum(0).reshape(-1), _planes(z)
    return r


def _take(s, count=1):
    s["op"] += count
    return s["op"] - count


def _plain_dense(s, x, w, b, f, relu, res):
    z = _products(x, w)
    if b is not None:
        z = z + (b << f)[:, None, :]
    y, gate = _finish(z, _take(s), f, relu)
    return (y if res is None else y + res), gate


def _plain_forward(s, c):
    y, gate = _plain_dense(s, s["x"], s["W"], s.get("b"), c["tau"], c["relu"], s.get("res"))
    return _out(y=y, gate=gate) if c["gate"] else _out(y=y)


def _plain_backward(s, c):
    dz, f = s["dy"], c["tau"]
    if "gate" in s:
        dz = _mult(s["gate"], dz, _take(s), dz[0].numel())
    dx, _ = _finish(_products(dz, s["W"].transpose(1, 2).contiguous()), _take(s), f)
    dW, _ = _finish(_products(s["x"].transpose(1, 2).contiguous(), dz), _take(s), f)
    return _out(dx=dx, dW=dW, db=dz.sum(1))


def _plain_moe(s, c):
    n, d, ff, E, k, f = c["rows"], c["d"], c["ff"], c["experts"], c["top"], c["tau"]
    scores, _ = _plain_dense(s, s["x"], s["Wr"], s.get("br"), f, True, None)
    v = scores.sum(0)                                                     # [n, E]
    _take(s)                                                              # the comparisons: their bits only count ranks
    a, b = v[:, :, None], v[:, None, :]
    idx = torch.arange(E, device=DEV)
    rank = ((b > a) | ((b == a) & (idx[None, None, :] < idx[None, :, None]))).sum(2)
    hot = (rank[:, None, :] == torch.arange(k, device=DEV)[None, :, None]).to(torch.int64)   # [n, k, E]
    beta, share = _dabit(_take(s), n * k * E)
    o = _from_bit(hot.reshape(-1), beta, share).view(3, n, k, E)
    _take(s)                                                              # the chosen scores
    quo = torch.div((hot * v[:, None, :]).sum(2) << f, 1 + v.sum(1, keepdim=True), rounding_mode="floor").reshape(-1)
    g = torch.zeros(3, n * k, dtype=torch.int64, device=DEV)
    for t in range(f + 1):
        g = 2 * g + _from_bit((quo >> (f - t)) & 1, *_dabit(_take(s), n * k))
    g = g.view(3, n, k)
    xe = _mult(o[..., None].expand(3, n, k, E, d), s["x"][:, :, None, None, :].expand(3, n, k, E, d), _take(s), n * k * E * d)
    rows, W1 = xe.reshape(3, n * k, E * d), s["W1"].reshape(3, E * d, ff)
    if "b1" in s:
        rows, W1 = torch.cat([rows, (o << f).reshape(3, n * k, E)], 2), torch.cat([W1, s["b1"]], 1)
    h, _ = _finish(_products(rows, W1), _take(s), f, True)
    hg, _ = _finish(_local(g.reshape(3, n * k, 1).expand(3, n * k, ff).contiguous(), h), _take(s), f)
    parts = [_local(o[..., None].expand(3, n, k, E, ff), hg.view(3, n, k, 1, ff).expand(3, n, k, E, ff)).sum(2).view(3, n, E * ff),
             _local(o, g[..., None].expand(3, n, k, E)).sum(2)]
    he = torch.cat(parts, 2)
    he = he + _zero(_take(s), 0, he[0].numel()).view(he.shape)
    W2 = s["W2"].reshape(3, E * ff, d)
    if "b2" in s:
        W2 = torch.cat([W2, s["b2"]], 1)
    else:
        he = he[:, :, :E * ff]
    y, _ = _finish(_products(he, W2), _take(s), f)
    return _out(y=y if "res" not in s else y + s["res"])


# ---- values in 64 bits ------------------------------------------------------------------------
def exact(c, seed):
    """The values by integers on the host: products of whole numbers below 2^53, floors by shifts."""
    v, f = {k: t.cpu().numpy() for k, t in _values(c, seed).items()}, c["tau"]

    def product(a, b):
        assert float(np.abs(a).max()) * float(np.abs(b).max()) * a.shape[-1] < 2.0 ** 62
        z = a.astype(np.float64) @ b.astype(np.float64)
        assert np.abs(z).max(initial=0) < 2.0 ** 53
        return z.astype(np.int64)

    def scaled(z):
        return (z + (1 << (f - 1))) >> f

    if c["kind"] == "backward":
        dz = v["dy"] * v.get("gate", 1)
        return dict(dx=scaled(product(dz, v["W"].T)).ravel(), dW=scaled(product(v["x"].T, dz)).ravel(), db=dz.sum(0), dx_shares=None, dW_shares=None,
                    db_shares=None)
    if c["kind"] == "forward":
        y = scaled(product(v["x"], v["W"]) + (v["b"] << f if "b" in v else 0))
        r = dict(y=((np.maximum(y, 0) if c["relu"] else y) + v.get("res", 0)).ravel(), y_shares=None)
        if c["gate"]:
            r.update(gate=(y >= 0).astype(np.int64).ravel(), gate_shares=None)
        return r
    zero = np.int64(0)
    score = np.maximum(scaled(product(v["x"], v["Wr"]) + (v["br"] << f if "br" in v else zero)), 0)
    y = np.zeros((c["rows"], c["d"]), np.int64)
    for t in range(c["rows"]):
        order = sorted(range(c["experts"]), key=lambda a: (-int(score[t, a]), a))
        total = np.zeros(c["d"], np.int64)
        for a in order[:c["top"]]:
            gate = (int(score[t, a]) << f) // (1 + int(score[t].sum()))
            h = np.maximum(scaled(product(v["x"][t:t + 1], v["W1"][a]) + (v["b1"][a] << f if "b1" in v else zero)), 0)
            total = total + product(scaled(gate * h), v["W2"][a])[0] + (gate * v["b2"][a] if "b2" in v else zero)
        y[t] = scaled(total)
    return dict(y=(y + v.get("res", 0)).ravel(), y_shares=None)


# ---- what a pass cannot do without --------------------------------------------------------------
# Words: an input's three components, an output's six planes and its values.  Operations: a ring product of 64-bit words takes 18 products of
# 8-bit residues (36 operations), each party makes two per term; a PRF block 400 operations.  A completed output takes two blocks of the dealer's and, for eight outputs,
# three keys' blocks of the zero sharing, of the tree's two masks and, with ReLU, of the product.
RING, BLOCK = 36.0, 400.0


def _finish_work(n, relu):
    return n * BLOCK * (2 + 3 * (4 if relu else 3) / 8.0)


def work(c):
    n = c["rows"]
    if c["kind"] == "moe":
        d, ff, E, k = c["d"], c["ff"], c["experts"], c["top"]
        weights = d * E + 2 * E * d * ff + (E + E * ff + E * d if c["bias"] else 0)
        words = 3 * (weights + n * d * (2 if c["residual"] else 1)) + 7 * n * d
        macs = n * d * E + n * k * E * d * ff + n * E * ff * d
        ops = 6 * RING * macs + _finish_work(n * E, True) + _finish_work(n * k * ff, True) + _finish_work(n * k * ff + n * d, False)
        ops += BLOCK * 3 / 8.0 * n * E * (k * d + ff)
        return dict(bytes=8.0 * words, flops=float(ops))
    din, dout = c["din"], c["dout"]
    if c["kind"] == "backward":
        words = 3 * (n * din + din * dout + n * dout * (2 if c["relu"] else 1)) + 7 * (n * din + din * dout + dout)
        ops = 6 * RING * 2 * n * din * dout + _finish_work(n * din + din * dout, False) + (n * dout * BLOCK * 3 / 8.0 if c["relu"] else 0)
        return dict(bytes=8.0 * words, flops=float(ops))
    words = 3 * (n * din + din * dout + (dout if c["bias"] else 0) + (n * dout if c["residual"] else 0)) + (14 if c["gate"] else 7) * n * dout
    return dict(bytes=8.0 * words, flops=float(6 * RING * n * din * dout + _finish_work(n * dout, c["relu"])))


def _cost(c):
    """Rough seconds of a pass, for bounding what draw() asks for."""
    w = work(c)
    return w["bytes"] / 3e12 + w["flops"] / 1e15
