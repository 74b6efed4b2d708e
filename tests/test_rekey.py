"""Keys and their successors (gt_rekey): the definition on the oracle, and refusals that need no GPU."""
import numpy as np

from oracle import Oracle, orc
from paper_2305_00645_amd import gtree


def successor(key):
    """Four 64-bit words of a key -> those of the next one."""
    words = [w >> s & 0xFFFFFFFF for w in (int(k) for k in key) for s in (0, 32)]
    out = [int(x) for x in orc.chacha_block(words, 0, 0, 0, 0xFFFFFFFF, 8)]
    return [out[2 * i] | out[2 * i + 1] << 32 for i in range(4)]


def test_every_key_is_replaced_by_its_successor(seed):
    o, keys = Oracle(seed), [list(k) for k in seed]
    for _ in range(3):
        o.rekey()
        keys = [successor(k) for k in keys]
        fresh = Oracle(keys)
        for k in range(5):
            assert o.prf_word(k, 3, 1, 77) == fresh.prf_word(k, 3, 1, 77)
    assert o.op_counter() == 0


def test_same_ids_under_new_keys(seed):
    """The same call with the same id: other shares of the same values, messages counted as before."""
    o = Oracle(seed)
    x = np.arange(40, dtype=np.uint64) << np.uint64(9)
    a, b = o.share(x), o.share(x + np.uint64(5))
    op, got = o.op_counter(), []
    for again in range(2):
        o.set_op(op)
        got.append(o.mult(a, b))
        o.rekey()
    assert np.array_equal(o.rec(got[0]), o.rec(got[1])) and not (got[0] == got[1]).any()


def test_refuses_no_context():
    assert gtree.load().gt_rekey(None) == gtree.GT_EINVAL
