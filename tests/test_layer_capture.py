"""Layers under graph capture, on the host alone: nothing that a capture forbids, and no workspace freed that a graph may hold."""
import pytest

from fake_hip import run

CALLS = ["lambda rows: L.gt_dense_forward(ctx, layer, shares(X), rows, 1, None, shares(Y), None)",
         "lambda rows: L.gt_dense_backward(ctx, layer, shares(X), shares(Y), shares(Y), rows, shares(X), shares(W), shares(2000))",
         "lambda rows: L.gt_moe_forward(ctx, mixture, shares(X), rows, None, shares(X))"]
SETUP = """
X, Y, W = 9000 * 1000, 9000 * 2000, 1000 * 2000
ctx = context()
layer, mixture = dense(ctx, 1000, 2000), moe(ctx, 300, 600, 4, 2, 3000)
call = %s
def captured(rows):
    fake.fake_capture(1)
    rc = call(rows)
    fake.fake_capture(0)
    return rc
"""


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("rows", [3, 700])
def test_a_workspace_too_small_is_refused(call, rows):
    run(SETUP % call + """
before, n = counted(ctx), fake.fake_launches()
assert captured(%d) == gtree.GT_ESTATE
assert counted(ctx) == before and fake.fake_launches() == n and fake.fake_bad() == 0
assert call(%d) == 0
op = L.gt_op_counter(ctx)
assert captured(%d) == 0 and L.gt_op_counter(ctx) == 2 * op and fake.fake_bad() == 0
""" % (rows, rows, rows))


@pytest.mark.parametrize("call", CALLS)
def test_larger_calls_free_nothing_that_a_graph_holds(call):
    """Larger layers, and array accesses, which share a workspace with them, after a capture."""
    run(SETUP % call + """
start = fake.fake_now()
assert call(3) == 0
held = fake.fake_now()
assert captured(3) == 0
frees = []
for rows in (20, 190, 700, 3000):
    before, live = fake.fake_now(), fake.fake_newest()
    assert call(rows) == 0
    assert fake.fake_now() >= before and fake.fake_live(live)
before = fake.fake_now()
assert L.gt_oaa_literal(ctx, shares(100000), 100000, shares(300), 300, shares(300)) == 0
assert L.gt_oaa(ctx, shares(4000), 4000, shares(9 * 10**6), 9 * 10**6, shares(9 * 10**6)) == 0
assert fake.fake_now() >= before
assert L.gt_dense_destroy(layer) == 0 and L.gt_moe_destroy(mixture) == 0 and L.gt_ctx_destroy(ctx) == 0
assert fake.fake_now() == 0 and fake.fake_bad() == 0
""")


def test_without_a_capture_nothing_is_held():
    run(SETUP % CALLS[1] + """
assert call(700) == 0
once = fake.fake_now()
other = context()
l2 = dense(other, 1000, 2000)
assert L.gt_dense_backward(other, l2, shares(X), shares(Y), shares(Y), 3, shares(X), shares(W), None) == 0
before = fake.fake_now()
assert L.gt_dense_backward(other, l2, shares(X), shares(Y), shares(Y), 3000, shares(X), shares(W), None) == 0
fake.fake_peak()
live = fake.fake_newest()
assert L.gt_dense_backward(other, l2, shares(X), shares(Y), shares(Y), 9000, shares(X), shares(W), None) == 0
assert not fake.fake_live(live)
""")
