"""The gated layer and linear attention, on the host alone: refusals, graph capture, workspaces that cannot be allocated, launches within the limits."""
import ctypes as C

import pytest

from fake_hip import run
from paper_2305_00645_amd import gtree

SETUP = """
ctx = context(%d)
def gated(din, ff, bias=False):
    h = C.c_void_p()
    b = shares(ff) if bias else None
    assert L.gt_gated_create(ctx, shares(din * ff), b, shares(din * ff), b, din, ff, C.byref(h)) == 0
    return h
def attention(heads, dk, dv, w=4000):
    h = C.c_void_p()
    assert L.gt_linattn_create(ctx, (C.c_uint32 * heads)(*[w] * heads), heads, dk, dv, C.byref(h)) == 0
    return h
DIN, FF = 1000, 1000
layer, att = gated(DIN, FF), attention(16, 64, 64)
X, Y, W = 9000 * DIN, 9000 * FF, DIN * FF
def forward(rows, keep=True):
    k = [shares(Y)] * 3 if keep else [None] * 3
    return L.gt_gated_forward(ctx, layer, shares(X), rows, 1, shares(Y), *k)
def backward(rows):
    return L.gt_gated_backward(ctx, layer, shares(X), shares(Y), shares(Y), shares(Y), shares(Y), rows, shares(X), shares(W), shares(W), shares(FF), shares(FF))
def prompt(tokens):
    n = 9000 * 1024
    return L.gt_linattn_forward(ctx, att, shares(n), shares(n), shares(n), 0, 2, tokens, None, shares(2 * 16 * 4096), shares(n))
"""
CALLS = dict(forward=(3, 190, 700, 3000), backward=(3, 190, 700, 3000), prompt=(2, 70, 700, 4000))


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("small", [0, 4])
def test_a_workspace_too_small_under_capture(name, small):
    """Refused without a trace; when it is there, captured; larger calls free nothing that the graph holds."""
    run(SETUP % small + """
call, sizes = %s, %r
for size in sizes[:3]:
    before, n = counted(ctx), fake.fake_launches()
    fake.fake_capture(1)
    rc = call(size)
    fake.fake_capture(0)
    if rc:                                                # (a small workspace may be large enough already)
        assert rc == gtree.GT_ESTATE and counted(ctx) == before and fake.fake_launches() == n
    assert call(size) == 0
    fake.fake_capture(1)
    assert call(size) == 0
    fake.fake_capture(0)
    held, live = fake.fake_now(), fake.fake_newest()
    assert call(sizes[-1]) == 0
    assert fake.fake_now() >= held and fake.fake_live(live)
    ctx, layer, att = context(%d), gated(DIN, FF), attention(16, 64, 64)
assert fake.fake_bad() == 0
""" % (name, CALLS[name], small))


def test_a_single_token_needs_no_workspace():
    run(SETUP % 0 + """
n, before = 64 * 1024, fake.fake_tries()
fake.fake_capture(1)
for state in (None, shares(64 * 16 * 4096)):
    assert L.gt_linattn_forward(ctx, att, shares(n), shares(n), shares(n), 0, 64, 1, state, shares(64 * 16 * 4096), shares(n)) == 0
fake.fake_capture(0)
assert fake.fake_tries() == before and fake.fake_bad() == 0
""")


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("size", [0, 1, 3])
def test_no_memory_leaves_no_trace(name, size):
    run(SETUP % 0 + """
call, size = %s, %d
before = counted(ctx)
fake.fake_fail(-1)
assert call(size) == 0
needs, want = fake.fake_tries(), counted(ctx)
assert needs >= 1 and want[0] > before[0]
for at in range(needs):
    fake.fake_fail(-1)
    ctx = context(0)
    layer, att = gated(DIN, FF), attention(16, 64, 64)
    n = fake.fake_launches()
    fake.fake_fail(at)
    assert call(size) == gtree.GT_ENOMEM
    assert counted(ctx) == before and fake.fake_launches() == n
    fake.fake_fail(-1)
    assert call(size) == 0 and counted(ctx) == want
assert fake.fake_bad() == 0
""" % (name, CALLS[name][size]))


def test_layers_without_memory_and_everything_freed():
    run(SETUP % 0 + """
assert L.gt_gated_destroy(layer) == 0 and L.gt_linattn_destroy(att) == 0 and L.gt_ctx_destroy(ctx) == 0
assert fake.fake_now() == 0
ctx = context(0)
start = fake.fake_now()
h = C.c_void_p()
for at in range(2):
    fake.fake_fail(at)
    assert L.gt_gated_create(ctx, shares(70), shares(7), shares(70), shares(7), 10, 7, C.byref(h)) == gtree.GT_ENOMEM
    assert fake.fake_now() == start
fake.fake_fail(0)
assert L.gt_linattn_create(ctx, (C.c_uint32 * 2)(1, 2), 2, 3, 4, C.byref(h)) == gtree.GT_ENOMEM
fake.fake_fail(-1)
assert fake.fake_now() == start and not h.value and fake.fake_bad() == 0
layer, att = gated(100, 70, True), attention(3, 5, 6)
assert L.gt_gated_forward(ctx, layer, shares(30000), 300, 0, shares(21000), shares(21000), shares(21000), None) == 0
assert L.gt_gated_backward(ctx, layer, None, shares(21000), shares(21000), None, shares(21000), 300, shares(30000), None, None, shares(70), shares(70)) == 0
assert L.gt_linattn_forward(ctx, att, shares(1500), shares(1500), shares(1800), 0, 1, 100, None, shares(90), shares(1800)) == 0
assert L.gt_gated_destroy(layer) == 0 and L.gt_linattn_destroy(att) == 0 and L.gt_ctx_destroy(ctx) == 0
assert fake.fake_now() == 0
""")


def test_the_largest_calls():
    """Sizes at their limits: launches and workspaces within theirs."""
    run(SETUP % 0 + """
M = gtree_max = 1 << 20
big = shares(1 << 50)
for din, ff in ((1, M // 2), (M, 1), (1, 1)):
    l = gated(din, ff)
    fake.fake_largest()
    assert L.gt_gated_forward(ctx, l, big, M, 1, big, big, big, big) == 0
    assert L.gt_gated_backward(ctx, l, big, big, big, big, big, 4096, big, big, big, big, big) == 0
    assert fake.fake_bad() == 0, (din, ff)
assert L.gt_gated_backward(ctx, gated(1, 4096), big, big, big, big, big, M, big, None, None, big, big) == 0
assert fake.fake_bad() == 0
for heads, dk, dv, seqs, tokens in ((256, 256, 256, 16, M // 16), (1, 1, 1, M, 1), (1, 256, 256, M // 16, 1), (256, 1, 1, 4096, 256), (1, 256, 256, 1, M), (16, 1, 256, M // 16, 16)):
    a = attention(heads, dk, dv)
    fake.fake_largest()
    for state in (None, big):
        assert L.gt_linattn_forward(ctx, a, big, big, big, 0, seqs, tokens, state, big, big) == 0, (heads, dk, dv, seqs, tokens)
    assert fake.fake_largest() <= (1 << 31) + 10**7 and fake.fake_bad() == 0, (heads, dk, dv, seqs, tokens)
assert fake.fake_bad() == 0
""")


def test_small_workspace_of_attention():
    run(SETUP % 4 + """
for heads, dk, dv in ((16, 64, 64), (256, 8, 8), (2, 256, 256)):
    a = attention(heads, dk, dv)
    fake.fake_largest()
    big = shares(1 << 50)
    assert L.gt_linattn_forward(ctx, a, big, big, big, 0, 1, 1 << 16, None, big, big) == 0
    assert fake.fake_largest() <= 1 << 26
""")


def test_refusals():
    run(SETUP % 0 + """
E, before, n = gtree.GT_EINVAL, counted(ctx), fake.fake_launches()
h, s = C.c_void_p(), shares
make = lambda *a: L.gt_gated_create(ctx, *a, C.byref(h))
assert make(None, None, s(6), None, 2, 3) == E and make(s(6), None, None, None, 2, 3) == E and make(s(5), None, s(6), None, 2, 3) == E
assert make(s(6), s(3), s(6), None, 2, 3) == E and make(s(6), None, s(6), s(3), 2, 3) == E and make(s(6), s(2), s(6), s(3), 2, 3) == E
assert make(s(0), None, s(0), None, 0, 3) == E and make(s(0), None, s(0), None, 2, 0) == E
assert make(s(1 << 21), None, s(1 << 21), None, 1, (1 << 19) + 1) == E and L.gt_gated_create(ctx, s(6), None, s(6), None, 2, 3, None) == E
assert L.gt_gated_set(ctx, layer, s(W), s(FF), s(W), s(FF)) == E and L.gt_gated_set(ctx, layer, s(W), None, s(W - 1), None) == E
f = lambda rows, act, *a: L.gt_gated_forward(ctx, layer, s(X), rows, act, *a)
assert f(2, 2, s(Y), None, None, None) == E and f((1 << 20) + 1, 1, s(Y), None, None, None) == E and f(2, 1, s(2 * FF - 1), None, None, None) == E
assert f(2, 1, s(Y), s(Y), None, None) == E and f(2, 1, s(Y), s(Y), s(Y), None) == E and f(2, 0, s(Y), s(Y), s(Y), s(Y)) == E
assert f(2, 1, s(Y), None, None, s(Y)) == E and f(2, 1, s(Y), s(Y), s(Y), s(7)) == E and f(9001, 1, s(9001 * FF), None, None, None) == E
b = lambda rows, x, g, u, gate, dh, *o: L.gt_gated_backward(ctx, layer, x, g, u, gate, dh, rows, *o)
k = [s(Y)] * 4
assert b(2, None, *k, None, s(W), s(W), None, None) == E                       # x is needed for dWg, dWu
assert b(2, s(X), *k, None, s(W), None, None, None) == E and b(2, s(X), *k, None, None, None, s(FF), None) == E
assert b(2, s(X), None, *k[1:], s(X), None, None, None, None) == E and b(2, s(X), *k[:3], None, s(X), None, None, None, None) == E
assert b(2, s(X), *k, s(2 * DIN - 1), None, None, None, None) == E and b((1 << 20) + 1, s(X), *k, s(X), None, None, None, None) == E
w = lambda *v: (C.c_uint32 * len(v))(*v)
make = lambda d, heads, dk, dv: L.gt_linattn_create(ctx, d, heads, dk, dv, C.byref(h))
assert make(None, 1, 1, 1) == E and make(w(1), 0, 1, 1) == E and make(w(1), 1, 0, 1) == E and make(w(1), 1, 1, 0) == E and make(w(4097), 1, 1, 1) == E
assert make(w(1), 1, 257, 1) == E and make(w(1), 1, 1, 257) == E and make(w(*[1] * 257), 257, 1, 1) == E
N, S = 1024, 16 * 4096
a = lambda q, k, v, ld, seqs, t, i, o, y: L.gt_linattn_forward(ctx, att, q, k, v, ld, seqs, t, i, o, y)
assert a(s(N - 1), s(N), s(N), 0, 1, 1, None, s(S), s(N)) == E and a(s(N), s(N), s(N), 0, 1, 1, None, s(S - 1), s(N)) == E
assert a(s(N), s(N), s(N), 0, 1, 1, s(S - 1), s(S), s(N)) == E and a(s(N), s(N), s(N), 0, 1, 1, None, None, s(N)) == E
assert a(s(N), s(N), s(N), 0, 1, 1, None, s(S), s(N - 1)) == E and a(s(N), s(N), s(N), N - 1, 1, 1, None, s(S), s(N)) == E
assert a(s(2 * N), s(2 * N), s(2 * N), N + 1, 1, 2, None, s(S), s(2 * N)) == E   # the second row does not fit
big = s(1 << 50)
assert a(big, big, big, 0, (1 << 16) + 1, 1, None, big, big) == E and a(big, big, big, 0, 1, (1 << 20) + 1, None, big, big) == E
assert a(big, big, big, 0, 1 << 16, 17, None, big, big) == E and a(big, big, big, (1 << 22) + 1, 1, 1, None, big, big) == E
for rc in (L.gt_gated_forward(None, layer, s(X), 1, 1, s(Y), None, None, None), L.gt_gated_forward(ctx, None, s(X), 1, 1, s(Y), None, None, None),
           L.gt_linattn_forward(ctx, None, s(N), s(N), s(N), 0, 1, 1, None, s(S), s(N)), L.gt_gated_destroy(None), L.gt_linattn_destroy(None),
           L.gt_gated_set(ctx, None, s(W), None, s(W), None)):
    assert rc == E
assert counted(ctx) == before and fake.fake_launches() == n and not h.value
""")


def test_refusals_without_a_gpu():
    L, h = gtree.load(), C.c_void_p()
    assert L.gt_gated_create(None, None, None, None, None, 1, 1, C.byref(h)) == gtree.GT_EINVAL
    assert L.gt_linattn_create(None, None, 1, 1, 1, C.byref(h)) == gtree.GT_EINVAL
    assert not h.value


def test_decays_outside_their_range():
    """A decay's word has 32 bits at the library's border: one that does not fit must not arrive there as another."""
    run(SETUP % 0 + """
import math
g = object.__new__(gtree.GTree)
g.L, g.ctx = L, ctx
before, n = counted(ctx), fake.fake_launches()
for w in (2.0 ** 20, 2.0 ** 20 + 0.5, -2.0 ** 20, 1e300, -0.001, 1.001, 2, math.nan, math.inf, -math.inf):
    for decay in ([w], [0.5, w], [w, 0.5]):
        try:
            g.linattn_create(decay, 4, 4)
        except gtree.GtError as e:
            assert e.code == gtree.GT_EINVAL, (w, e.code)
        else:
            raise AssertionError(w)
assert counted(ctx) == before and fake.fake_launches() == n
for decay in ([0, 1], [0.0, 1.0], [0.25], np.array([0.5, 1.0])):
    g.linattn_create(decay, 4, 4).close()
""")


def test_a_decay_below_one_that_rounds_to_one():
    """A head that forgets slowly must not become one that never does: its state would grow without bound."""
    run(SETUP % 0 + """
g = object.__new__(gtree.GTree)
g.L, g.ctx = L, ctx
n = fake.fake_launches()
for w in (4095.5 / 4096, 0.9999, 1 - 2.0 ** -20, 1 - 2.0 ** -53):
    for decay in ([w], [1.0, w]):
        try:
            g.linattn_create(decay, 4, 4)
        except gtree.GtError as e:
            assert e.code == gtree.GT_EINVAL, (w, e.code)
        else:
            raise AssertionError(w)
assert fake.fake_launches() == n
for w in (1.0, 4095 / 4096, 4095.49 / 4096, 2.0 ** -14, 0.0):
    g.linattn_create([w], 4, 4).close()
""")
