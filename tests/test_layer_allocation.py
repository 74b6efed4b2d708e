"""Layers whose workspace cannot be allocated: GT_ENOMEM before anything is counted or launched, and the next call runs as if there had been none."""
import pytest

from fake_hip import run

CALLS = dict(
    few="lambda: L.gt_dense_forward(ctx, layer, shares(X), 4, 1, None, shares(Y), None)",
    rows_ahead="lambda: L.gt_dense_forward(ctx, layer, shares(X), 180, 0, None, shares(Y), None)",
    residues="lambda: L.gt_dense_forward(ctx, layer, shares(X), 3000, 1, None, shares(Y), shares(Y))",
    gradients="lambda: L.gt_dense_backward(ctx, layer, shares(X), shares(Y), shares(Y), 3000, shares(X), shares(W), shares(2000))",
    gradients_few="lambda: L.gt_dense_backward(ctx, layer, shares(X), shares(Y), shares(Y), 20, shares(X), shares(W), None)",
    gradients_small="lambda: L.gt_dense_backward(ctx, layer, shares(X), shares(Y), shares(Y), 9000, shares(X), shares(W), None)",
    mixture_few="lambda: L.gt_moe_forward(ctx, mixture, shares(X), 3, None, shares(X))",
    mixture_many="lambda: L.gt_moe_forward(ctx, mixture, shares(X), 700, None, shares(X))",
)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_a_refused_call_leaves_no_trace(name):
    out = run("""
small = "small" in %r
def make():
    ctx = context(4 if small else 0)
    return ctx, dense(ctx, 1000, 2000), moe(ctx, 300, 600, 4, 2, 700)
X, Y, W = 9000 * 1000, 9000 * 2000, 1000 * 2000
def call():
    return (%s)()
ctx, layer, mixture = make()
fake.fake_fail(-1)
before = counted(ctx)
assert call() == 0
needs, want = fake.fake_tries(), counted(ctx)
assert needs >= 1 and want[0] > before[0]
fake.fake_fail(0)
assert call() == 0                                    # the workspace is there now
assert fake.fake_tries() == 0
for at in range(needs):
    fake.fake_fail(-1)
    ctx, layer, mixture = make()
    n = fake.fake_launches()
    fake.fake_fail(at)
    assert call() == gtree.GT_ENOMEM
    assert counted(ctx) == before, (at, counted(ctx), before)
    assert fake.fake_launches() == n
    fake.fake_fail(-1)
    assert call() == 0 and counted(ctx) == want
assert fake.fake_bad() == 0
print(needs)
""" % (name, CALLS[name]))
    assert int(out) >= 1


def test_everything_is_freed():
    run("""
start = fake.fake_now()
ctx = context()
layer, mixture = dense(ctx, 100, 200), moe(ctx, 30, 60, 4, 2, 70)
assert L.gt_dense_forward(ctx, layer, shares(300 * 100), 300, 1, None, shares(300 * 200), None) == 0
assert L.gt_dense_backward(ctx, layer, shares(30000), shares(60000), shares(60000), 300, shares(30000), shares(20000), None) == 0
assert L.gt_moe_forward(ctx, mixture, shares(2100), 70, None, shares(2100)) == 0
assert L.gt_dense_destroy(layer) == 0 and L.gt_moe_destroy(mixture) == 0 and L.gt_ctx_destroy(ctx) == 0
assert fake.fake_now() == start and fake.fake_bad() == 0
""")
