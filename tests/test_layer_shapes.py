"""The layers' rules: every output is covered once, sums stay in their words, and the GPU tests' calls take every variant."""
import pytest

import test_gpu_layers as gl
import test_gpu_layers_variants as gv
from layer_shapes import apart, few, few_split, fin, left, parts_pairs, rmm, rows_of_pass

SIZES = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 192, 193, 255, 257, 600, 1000, 4097, 30000, 1 << 20]


@pytest.mark.parametrize("n", [1, 39, 40, 41, 79, 3072 * 40, 3072 * 40 + 1, 2 * 3072 * 40, 2 * 3072 * 40 + 39, 512000, 1 << 23, (1 << 27) + (1 << 20)])
def test_completion_covers_every_tile(n):
    per, nbig, waves = fin(n)
    tiles = (n + 39) // 40
    assert 1 <= per <= 4 and nbig * per + (waves - nbig) == tiles and waves >= nbig and waves < 1 << 31


def test_products_cover_every_output():
    for M in SIZES:
        for N in SIZES:
            wm, wn, ntm, ntn = rmm(M, N)
            assert 64 * wm * ntm >= M > 64 * wm * (ntm - 1) and 64 * wn * ntn >= N > 64 * wn * (ntn - 1)
            assert rows_of_pass(N) % 128 == 0
            for K in SIZES:
                rows, ntile, ngrp, nsplit, per = few_split(M, N, K)
                steps = (K + 63) // 64
                assert rows * ntile >= M and 64 * ngrp >= N and nsplit * per >= steps > (nsplit - 1) * per
                assert per <= 64                     # int32 sums of limbs, 2^19 a step, times two where rows fill a tile


def kinds(sizes):
    return {few(M, N, K) for M, K, N in sizes}


def test_calls_take_the_variants_that_they_name():
    assert kinds(gl.SIZES) == {True}
    assert kinds(gv.RESIDUES) == {False} and kinds(gv.FEW_MANY) == {True}
    assert {parts_pairs(M * N) for M, K, N in gv.FEW_MANY} == {True} and {parts_pairs(M * N) for M, K, N in gl.SIZES} == {False}
    assert {rmm(M, N)[:2] for M, K, N in gv.RESIDUES} == {(1, 1), (2, 2), (4, 2)}
    assert {fin(M * N)[0] for M, K, N in gv.RESIDUES} == {1, 2, 4}
    assert any(M > rows_of_pass(N) for M, K, N in gv.RESIDUES) and any(K > 4096 for M, K, N in gv.RESIDUES)
    assert {few_split(M, N, K)[0] for M, K, N in gl.SIZES} == {8, 16}
    assert [few(M, N, K) for M, K, N in gv.LARGEST] == [True, True, True, False, False]
    assert {left(M, N, K) for M, K, N in gv.LEFT} == {True} and kinds(gv.LEFT) == {True} and {left(M, N, K) for M, K, N in gl.SIZES} == {False}
    assert all(left(rows, din, dout) for rows, din, dout in gv.LEFT_BACKWARD)
    assert all(left(rows * k, ff, E * (d + 1)) and few(rows, d, E * (ff + 1)) for rows, d, ff, E, k in gv.LEFT_MIXTURES)
    assert {apart(*s) for s in gv.BACKWARD} == {False, True}
    for rows, d, ff, E, k in gv.MIXTURES:
        assert not (few(rows * k, ff, E * (d + 1)) and few(rows, d, E * (ff + 1)))


def test_rule_at_its_borders():
    assert few(192, 4096, 1024) and not few(193, 4096, 1024)
    assert few(16 * 1024, 64, 64) and not few(16 * 1024 + 1, 64, 64)
    assert not few(1, 1, 1 << 25)
    assert apart(64, 512, 256) and not apart(65, 512, 256) and not apart(64, 512, 255)
