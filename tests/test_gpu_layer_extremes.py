"""Layers on the words whose sums are the largest that limbs and residues have to tell apart, of both signs, against the CPU oracle bit for bit."""
import numpy as np
import pytest

from test_gpu_parity import mods, pair, same  # noqa: F401

pytestmark = pytest.mark.gpu

# all signed bytes -128, all 127
LOW, HIGH = 0x7f7f7f7f7f7f7f80, 0x7f7f7f7f7f7f7f7f
PAIRS = [(LOW, LOW, 1), (LOW, HIGH, -1), (HIGH, LOW, -1), (HIGH, HIGH, 1)]          # words, sign of their product
# rows, din, dout: the sums in the left and in the right factor; a whole chunk of terms, one more
RESIDUES = [(200, 4096, 300), (300, 4096, 200), (200, 4097, 300), (300, 4097, 200)]
GRADIENTS = [(4096, 40, 30), (4097, 30, 40)]
# few rows: a split of 64 steps and a second one
FEW = [(192, 4160, 704)]


def on_gpu(gtree, c):
    import torch
    t = torch.from_numpy(np.stack([c, np.roll(c, -1, 0)], 1).view(np.int64)).to("cuda")
    return gtree.Shares(c.shape[1], t=t.contiguous())


def parts(a, b, na, nb):
    """Components with which both of a party's two products a term are a b: (a, 0, 0) and (b, b, b) where the left factor's are added up, else mirrored."""
    one = np.zeros((3, na), dtype=np.uint64)
    one[0] = a
    return one, np.full((3, nb), b, dtype=np.uint64)


@pytest.mark.parametrize("rows,din,dout", RESIDUES + FEW)
@pytest.mark.parametrize("a,b,sign", PAIRS)
def test_dense_forward(mods, seed, rows, din, dout, a, b, sign):
    _, gtree = mods
    o, g = pair(mods, seed)
    for mirrored in (False, True):
        print("dense", rows, din, dout, hex(a), hex(b), mirrored, flush=True)
        x, w = parts(np.uint64(a), np.uint64(b), rows * din, din * dout) if not mirrored else parts(np.uint64(b), np.uint64(a), din * dout, rows * din)[::-1]
        layer = g.dense_create(on_gpu(gtree, w), din, dout)
        same(g.dense_forward(layer, on_gpu(gtree, x), rows), o.dense_forward(x, w, rows, din, dout)[0], "y")
        layer.close()
    g.close()


@pytest.mark.parametrize("rows,din,dout", GRADIENTS)
@pytest.mark.parametrize("a,b,sign", PAIRS)
def test_dense_backward(mods, seed, rows, din, dout, a, b, sign):
    _, gtree = mods
    o, g = pair(mods, seed)
    w = np.full((3, din * dout), b, dtype=np.uint64)
    layer = g.dense_create(on_gpu(gtree, w), din, dout)
    for mirrored in (False, True):
        print("backward", rows, din, dout, hex(a), hex(b), mirrored, flush=True)
        x, dy = parts(np.uint64(a), np.uint64(b), rows * din, rows * dout) if not mirrored else parts(np.uint64(b), np.uint64(a), rows * dout, rows * din)[::-1]
        for name, got, want in zip(("dx", "dW", "db"), g.dense_backward(layer, on_gpu(gtree, x), on_gpu(gtree, dy), rows), o.dense_backward(x, w, dy, rows, din, dout)):
            same(got, want, name)
    layer.close(); g.close()
