"""What the exactness of the layers' products rests on, in whole numbers: the moduli as the source has them, the largest sums, and that the GPU tests' words reach them."""
import math
import os
import re

import test_gpu_layer_extremes as gx
from layer_shapes import few, few_split
from shapes import CSRC

R = (256 ** 8 - 1) // 255


def source(name):
    return open(os.path.join(CSRC, name)).read()


MODULI = [int(v) for v in re.search(r"const int m\[RNS_N\] = \{([^}]*)\}", source("gt_layers.hpp")).group(1).split(",")]
TERMS = int(re.search(r"#define RNS_TERMS (\d+)", source("gt_shape.hpp")).group(1))
M = math.prod(MODULI)
LARGEST = 2 * TERMS * (128 * R) ** 2


def number(word):
    """What a word's signed bytes stand for."""
    digits, carry = [], 0
    for s in range(8):
        v = (word >> 8 * s & 255) + carry
        carry = int(v >= 128)
        digits.append(v - 256 * carry)
    return sum(d * 256 ** s for s, d in enumerate(digits)), digits


def join(S):
    """The definition's way from balanced residues to the sum: the rounded quotient as the kernels round it."""
    r = []
    for m in MODULI:
        v = S * pow(M // m, -1, m) % m
        r.append(v - m if 2 * v > m - 1 + m % 2 else v)
    q = sum(a * ((16384 + m // 2) // m) for a, m in zip(r, MODULI)) + (1 << 13) >> 14
    return sum(a * (M // m) for a, m in zip(r, MODULI)) - q * M


def test_moduli():
    assert len(MODULI) == 18 and max(MODULI) <= 256
    assert all(math.gcd(a, b) == 1 for i, a in enumerate(MODULI) for b in MODULI[:i])


def test_the_quotient_is_exact():
    """The quotient's error: every residue (at most 128) times half a unit of its factor; with it the largest sum stays on its side of a half."""
    error = 18 * 128
    assert LARGEST * (1 << 15) + error * M < M * (1 << 14)
    assert 3681 * M < 10000 * LARGEST < 3682 * M
    most = 2 * TERMS * 2 ** 14                            # int32 sums of residues, and their reduction in a float's 24 bits
    assert most == 2 ** 27 and (most >> 13) * 128 + 8191 < 2 ** 21.1
    for S in (0, 1, -1, LARGEST, -LARGEST, LARGEST - 1, LARGEST // 3, -LARGEST // 7):
        assert join(S) == S


def test_the_limb_sums_stay_in_their_words():
    """At most 64 steps of 64 terms: eight products of limbs a term, 2^23 a step, twice where both factors fill a tile."""
    assert 64 * 64 * 8 * 2 ** 14 * 2 == 2 ** 30


def test_the_words_of_the_gpu_tests_reach_the_bounds():
    low, high = number(gx.LOW), number(gx.HIGH)
    assert low == (-128 * R, [-128] * 8) and high == (127 * R, [127] * 8)
    for a, b, sign in gx.PAIRS:
        S = 2 * TERMS * number(a)[0] * number(b)[0]
        assert S * sign > 0.98 * LARGEST and join(S) == S
    assert all(not few(rows, dout, din) for rows, din, dout in gx.RESIDUES)
    assert {(rows <= dout, min(din, TERMS), din > TERMS) for rows, din, dout in gx.RESIDUES} == {(True, TERMS, False), (False, TERMS, False), (True, TERMS, True), (False, TERMS, True)}
    assert {rows for rows, _, _ in gx.GRADIENTS} >= {TERMS, TERMS + 1}
    for rows, din, dout in gx.FEW:
        assert few(rows, dout, din) and few_split(rows, dout, din)[3:] == (2, 64)
