"""The workspace of products by residues: bounded over all sizes that a layer may have, every chunk and column covered."""
import itertools

import pytest

import test_gpu_layer_workspace as gw
from layer_plans import plan, workspace
from layer_shapes import few

SIDES = [1, 22, 64, 257, 1000, 4095, 4096, 4097, 8192, 11585, 16384, 16385, 32768, 40000, 48842, 1 << 18, 1 << 20]


@pytest.mark.parametrize("small,most", [(False, 17e9), (True, 128 << 20)])
def test_residues_do_not_grow_with_any_side(small, most):
    got = max((workspace(M, N, K, small), M, N, K) for M, N, K in itertools.product(SIDES, SIDES, SIDES + [1 << 26]))
    assert got[0] <= most, got


@pytest.mark.parametrize("small", [False, True])
def test_plans_cover_the_product(small):
    for M, N, K in itertools.product(SIDES, SIDES, [0] + SIDES):
        p, chunks = plan(M, N, K, small), (K + 4095) // 4096
        assert p.rows >= 128 and p.rows % 128 == 0 and (p.cols >= N or p.cols % 256 == 0) and p.cols >= 1
        assert p.keep <= chunks and (p.keep >= 1 or K == 0)
        assert p.whole == (p.cols >= N and p.keep == chunks)
        assert min(M, p.rows) * N <= 128 * (1 << 20)                # words of a pass: 24 bytes each


def test_calls_keep_what_fits():
    """Sizes whose residues fit are not cut further than the rows of a pass were: one chunk, or all of them."""
    for M, N, K in ((2048, 4096, 1024), (16384, 8192, 4096), (1000, 257, 294), (294, 257, 48842), (1024, 1024, 1 << 18)):
        p = plan(M, N, K)
        assert p.whole and p.rows >= M
    assert plan(16384, 8192, 8192) == (8192, 8192, 2, True)               # fewer rows rather than a joining launch
    assert not plan(16384, 8192, 20000).whole and not plan(1024, 1024, 1 << 20).whole and plan(1024, 1024, 1 << 20).keep == 128


def test_calls_take_the_variants_that_they_name():
    kinds = set()
    for rows, din, dout in gw.FORWARD:
        assert not few(rows, dout, din)
        p = plan(rows, dout, din, True)
        assert p.rows < rows
        kinds.add((p.cols < dout, (din + 4095) // 4096 > p.keep, p.keep))
    assert kinds == {(True, False, 1), (False, True, 1), (False, True, 4), (True, True, 1), (False, False, 2)}, kinds
    assert any(not plan(din, dout, rows, True).whole for rows, din, dout in gw.BACKWARD)
    assert any(plan(din, dout, rows, True).whole for rows, din, dout in gw.BACKWARD)
