"""Rules of the gated layer and of linear attention: every tile is taken once, workspaces are bounded, and the GPU tests' calls take every variant."""
import random

import pytest

import block_shapes as bs
import layer_shapes as ls
from test_gpu_block import BACK_WIDTHS, GATED, LIN, PASSES


def pad8(n):
    return (n + 7) // 8 * 8


def tiles(n):
    return (n + 39) // 40


def test_every_tile_once():
    rng = random.Random(0)
    for _ in range(2000):
        t = int(2 ** rng.uniform(0, 28))
        p = bs.per(t)
        assert 1 <= p <= 16 and p * ((t + p - 1) // p) >= t
        per, nbig, waves = bs.gated(40 * t)
        assert per in (1, 2) and nbig * per + (waves - nbig) == t and nbig <= waves


def test_workspace_is_bounded():
    rng = random.Random(1)
    for small in (False, True):
        for _ in range(2000):
            nbh, nc, dk, dv = (int(2 ** rng.uniform(0, b)) for b in (20, 14, 8, 8))
            h, c = bs.lin_pass(nbh, nc, dk, dv, small)
            each = 24 * (2 * 2080 + 2 * pad8(dk * dv) + 64 * pad8(dv))
            assert 1 <= h <= nbh and 1 <= c <= nc and h * c * each <= (1 << 26 if small else 1 << 31)
            assert h == nbh or c == 1


@pytest.mark.parametrize("rows,n,want", [(1, 8192, True), (300, 40959, True), (300, 40960, False)])
def test_few_elements(rows, n, want):
    assert bs.few(n) == want


def test_the_gpu_tests_take_every_variant():
    seen = set()
    for rows, din, ff in GATED:
        n = rows * pad8(ff)
        seen.add("few" if ls.few(rows, 2 * ((ff + 63) // 64 * 64), din) and bs.few(n) else "parts" if ls.few(rows, 2 * ((ff + 63) // 64 * 64), din) else "residues %d" % bs.gated(n)[0])
    assert seen == {"few", "parts", "residues 1", "residues 2"}
    seen = set()
    for seqs, tokens, heads, dk, dv in LIN:
        bh, chunks = seqs * heads, (tokens + 63) // 64
        if tokens == 1:
            seen.add("token %d" % min(2, bs.per(bh * tiles(dk * dv))))
            continue
        seen.add("pairs" if bs.pairs(bh * tiles(dk * dv)) else "chains")
        last = tokens - 64 * (chunks - 1)
        seen.add("scores %d" % min(2, bs.per(bh * ((chunks - 1) * 52 + tiles(last * (last + 1) // 2)))))
        seen.add("outputs %d" % min(2, bs.per(bh * ((chunks - 1) * tiles(64 * pad8(dv)) + tiles(last * pad8(dv))))))
        seen.add("wide" if dk > 64 else "narrow")
        seen.add("whole" if dk % 64 == 0 and dv % 16 == 0 and tokens % 64 == 0 else "ragged")
    assert seen == {"token 1", "token 2", "pairs", "chains", "scores 1", "scores 2", "outputs 1", "outputs 2", "wide", "narrow", "whole", "ragged"}


def test_the_gpu_tests_take_every_kind_of_pass():
    seen = set()
    for seqs, tokens, heads, dk, dv in PASSES:
        nbh, nc = seqs * heads, (tokens + 63) // 64
        h, c = bs.lin_pass(nbh, nc, dk, dv, True)
        if h < nbh:
            seen.add("heads")
            seen.add("fewer heads last" if nbh % h else "equal heads")
        if c < nc:
            seen.add("chunks" if c > 1 else "a chunk")
            if c > 1:
                seen.add("fewer chunks last" if nc % c else "equal chunks")
        seen.add("short last chunk" if tokens % 64 else "full")
        seen.add("pairs" if bs.pairs(h * tiles(dk * dv)) else "chains")
    assert seen >= {"heads", "fewer heads last", "chunks", "a chunk", "fewer chunks last", "equal chunks", "short last chunk", "pairs", "chains"}


def test_gradients_of_every_width_by_both_kernels():
    assert [bs.few(rows * pad8(ff)) for rows, _, ff in BACK_WIDTHS] == [True, False]
