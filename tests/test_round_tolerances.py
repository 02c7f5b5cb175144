"""The sharper tolerance of attention's products with v: what it allows, and that a coarser kernel would not keep to it (planted in plain arithmetic; no GPU).

The kernel multiplies exact codes by p times the scale of v.  A bf16 batch rounds that product to 16 bits once: u = 2^-8 of each term at most, u A in all
(A = sum p |v| / sum p).  An fp16 batch keeps it in two bf16 parts: the first is off by at most 2^-8 of it, which is the second, which is off by at most
2^-8 of that: 2^-16 A.  Neither rounds v = code * scale itself.  What else there is, for up to 64 positions whose scores are exact and within 16 of each
other: sums of 64 terms, numerator and denominator, 2^-18 each; exponents off by 2^-22 of their size, 2^-19; their exponentials, the joining of pieces and the
division 2^-20: 2^-16 A together.

Where a wave has tiles of its own (up to 32 rows of a sequence and key head) bf16 batches have two parts as well, and over a bf16 cache, whose p has no scale, up
to 64 rows; there the first part is cut, the second is up to 2^-7 of p, off by 2^-8 of itself, and 2^-20 of p too large: 2^-15 A + 2^-20 A.
"""
import numpy as np
import pytest

from oracle import round_oracle as RO
from round_util import HALF_STEP, rounded

PART = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -16}


def parts(dtype, kept, rows):
    """How far p (v_scale) may be off, relative to it."""
    if kept == dtype:
        return 2.0 ** -15 + 2.0 ** -20 if dtype == "bf16" and rows <= 64 else HALF_STEP[dtype]
    return PART["fp16" if rows <= 32 else dtype]


def allowed(dtype, o, A, part=None):
    """Tolerance of an output: its own rounding, that of p v_scale and the rest above, half of the smallest fp16 number."""
    return HALF_STEP[dtype] * np.abs(o) + ((PART[dtype] if part is None else part) + 2.0 ** -16) * A + 2.0 ** -25


def computed(p, codes, scale, dtype, way):
    """sum p v / sum p of one row with the roundings of `way`, rounded to the type."""
    w = p * scale
    half = lambda x, t="bf16": rounded(x, t)[1].astype(np.float64)  # noqa: E731
    if way == "parts":
        first = half(w)
        got = first + half(w - first) if dtype == "fp16" else first
        o = got @ codes
    elif way == "cut":
        first = (w.astype(np.float32).view(np.uint32) & 0xFFFF0000).view(np.float32).astype(np.float64)
        o = (first + half(w * (1 + 2.0 ** -20) - first)) @ codes
    elif way == "one part":
        o = half(w) @ codes
    elif way == "v rounded":
        o = half(p, dtype) @ half(codes * scale[:, None], dtype)
    return half(o / p.sum(), dtype)


def row(rng, n, kept):
    v = rng.standard_normal((n, 64)) * np.exp(0.5 * rng.standard_normal((n, 1)))
    c, s = RO.quantise(v, kept)
    return np.exp(rng.standard_normal(n) - 3.0), c.astype(np.float64), s.astype(np.float64)


@pytest.mark.parametrize("kept", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_the_tolerance_holds_for_the_kernel_s_roundings(dtype, kept):
    rng = np.random.default_rng(1)
    for n in (1, 2, 3, 10, 64):
        for _ in range(20):
            p, c, s = row(rng, n, kept)
            o, A = (p * s) @ c / p.sum(), (p * s) @ np.abs(c) / p.sum()
            assert np.all(np.abs(computed(p, c, s, dtype, "parts") - o) <= allowed(dtype, o, A))


@pytest.mark.parametrize("kept", ["int8", "e4m3"])
@pytest.mark.parametrize("way", ["one part", "v rounded"])
def test_coarser_products_do_not_keep_to_it_in_fp16(way, kept):
    rng = np.random.default_rng(2)
    outside = 0
    for _ in range(50):
        p, c, s = row(rng, 3, kept)
        o, A = (p * s) @ c / p.sum(), (p * s) @ np.abs(c) / p.sum()
        outside += int(np.any(np.abs(computed(p, c, s, "fp16", way) - o) > allowed("fp16", o, A)))
    assert outside >= 25


def test_a_cut_part_and_the_rest_keep_to_theirs():
    rng = np.random.default_rng(3)
    outside = 0
    for n in (1, 2, 3, 10, 64):
        for _ in range(20):
            p, _, _ = row(rng, n, "int8")
            v = rounded(rng.standard_normal((n, 64)), "bf16")[1].astype(np.float64)
            o, A, one = p @ v / p.sum(), p @ np.abs(v) / p.sum(), np.ones(n)
            assert np.all(np.abs(computed(p, v, one, "bf16", "cut") - o) <= allowed("bf16", o, A, parts("bf16", "bf16", 64)))
            outside += int(np.any(np.abs(computed(p, v, one, "bf16", "one part") - o) > allowed("bf16", o, A, parts("bf16", "bf16", 64))))
    assert outside >= 40
