"""Array accesses whose workspace cannot grow (no memory, graph capture): refused with nothing counted or launched, on a HIP runtime of bookkeeping alone."""
import pytest

from fake_hip import run

CALLS = dict(oaa="L.gt_oaa(ctx, shares(4000), 4000, shares(5000), 5000, shares(5000))", oaa_literal="L.gt_oaa_literal(ctx, shares(400), 400, shares(50), 50, shares(50))")


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("how", ["memory", "capture"])
def test_a_refused_access_leaves_no_trace(name, how):
    run("""
ctx = context()
call = lambda: %s
before, n, capture = counted(ctx), fake.fake_launches(), %d
fake.fake_fail(-1 if capture else 0)
fake.fake_capture(capture)
assert call() == (gtree.GT_ESTATE if capture else gtree.GT_ENOMEM)
fake.fake_capture(0)
assert counted(ctx) == before and fake.fake_launches() == n and fake.fake_bad() == 0
fake.fake_fail(-1)
assert call() == 0 and fake.fake_tries() == 1 and L.gt_op_counter(ctx) == 1
fake.fake_capture(capture)
assert call() == 0 and L.gt_op_counter(ctx) == 2 and fake.fake_tries() == 1 and fake.fake_bad() == 0
""" % (CALLS[name], how == "capture"))
