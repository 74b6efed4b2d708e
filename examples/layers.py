"""A small network on shares, trained and then used: python examples/layers.py [steps]

The data owner shares a table of binary columns and a target; a hidden layer with ReLU and a linear one are trained by gradient steps in which nothing but the
loss is revealed; then a mixture of experts answers single rows next to the trained layers.  Synthetic data of the shape of the heart table (267 rows, 22 columns)."""
import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2305_00645_amd import gtree, workloads as wl  # noqa: E402

ROWS, COLS, HIDDEN = 267, 22, 16


def minus(a, b):
    """Difference of shared vectors: local."""
    return gtree.Shares(a.n, t=a.t[:, :, :a.n] - b.t[:, :, :b.n])


class Network:
    """COLS -> HIDDEN, ReLU -> 1, weights as shares."""

    def __init__(self, g, rng, rate):
        self.g, self.sizes = g, ((COLS, HIDDEN), (HIDDEN, 1))
        self.W = [g.share_a(g.fixed(rng.normal(size=s) * s[0] ** -0.5).reshape(-1)) for s in self.sizes]
        self.b = [g.share_a(g.fixed(np.zeros(s[1]))) for s in self.sizes]
        self.layers = [g.dense_create(w, *s, b=b) for w, s, b in zip(self.W, self.sizes, self.b)]
        # a step's update w - rate * dw is a layer itself: the gradient times -rate times the identity, w as the residual
        self.update = [g.dense_create(g.share_a(g.fixed(-rate * np.eye(s[1])).reshape(-1)), s[1], s[1]) for s in self.sizes]

    def forward(self, x, rows):
        self.h, self.gate = self.g.dense_forward(self.layers[0], x, rows, relu=True, want_gate=True)
        return self.g.dense_forward(self.layers[1], self.h, rows)

    def step(self, x, target, rows):
        """One gradient step on half the mean squared error; returns the loss of the weights before it."""
        y = self.forward(x, rows)
        dy = minus(y, target)
        dh, dW1, db1 = self.g.dense_backward(self.layers[1], self.h, dy, rows)
        _, dW0, db0 = self.g.dense_backward(self.layers[0], x, dh, rows, gate=self.gate, want=(False, True, True))
        for i, (dW, db) in enumerate(((dW0, db0), (dW1, db1))):
            din, dout = self.sizes[i]
            self.W[i] = self.g.dense_forward(self.update[i], dW, din, residual=self.W[i])
            self.b[i] = self.g.dense_forward(self.update[i], db, 1, residual=self.b[i])
            self.g.dense_set(self.layers[i], self.W[i], b=self.b[i])
        return 0.5 * float((self.g.real(dy) ** 2).mean())

    def close(self):
        for t in self.layers + self.update:
            t.close()


def data(g, rng):
    X = (rng.random((ROWS, COLS)) < 0.4).astype(np.float64)
    target = np.maximum(X @ rng.normal(size=(COLS, 3)) - 0.5, 0) @ np.array([1.0, -0.7, 0.5])
    return g.share_a(g.fixed(X).reshape(-1)), g.share_a(g.fixed(target))


def train(g, steps, rate=0.5):
    rng = np.random.default_rng(11)
    x, target = data(g, rng)
    net = Network(g, rng, rate / ROWS)
    return net, x, [net.step(x, target, ROWS) for _ in range(steps)]


def main(steps):
    g = gtree.GTree(wl.PROTOCOL_SEED, tau=16)
    net, x, losses = train(g, steps)
    print("loss %.4f -> %.4f in %d steps, %d rounds" % (losses[0], losses[-1], steps, g.stats()[0]))
    rng = np.random.default_rng(12)
    E, ff = 4, 32
    Wr, W1, W2 = (g.share_a(g.fixed(rng.normal(size=s) * s[-2] ** -0.5).reshape(-1)) for s in ((COLS, E), (E, COLS, ff), (E, ff, COLS)))
    moe = g.moe_create(Wr, W1, W2, COLS, ff, E, 1, max_rows=8)
    one = gtree.Shares(COLS, t=x.t[:, :, :COLS].contiguous())            # a single row: the experts' answer on top of it, then the network's
    print("answer for the first row: %.4f" % float(g.real(net.forward(g.moe_forward(moe, one, 1, residual=one), 1))))
    moe.close()
    net.close()
    g.close()


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
