"""Pins of oracle/round_oracle.py: values worked out by hand, and independent statements of the same definitions."""
import math

import numpy as np
import pytest

from oracle import round_oracle as RO


def test_e4m3_has_the_values_of_its_format():
    # all 127 non-negative values, from the format's definition, are their own nearest
    values = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8) if (e, m) != (8, 7)]
    assert len(values) == 127 and max(values) == 448
    assert np.array_equal(RO.e4m3_nearest(values), values)
    mid = [(a + b) / 2 for a, b in zip(values, values[1:])]
    even = [values[i] if i % 2 == 0 else values[i + 1] for i in range(len(mid))]     # the code is the index: ties to the even one
    assert np.array_equal(RO.e4m3_nearest(mid), even)
    assert np.array_equal(RO.e4m3_nearest([-x for x in mid]), [-x for x in even])


def test_codes_of_a_row():
    c, s = RO.quantise(np.array([[1.0, -2.0, 0.5, 0.0]]), "int8")
    assert s[0] == np.float32(2.0) / np.float32(127.0) and list(c[0]) == [64.0, -127.0, 32.0, 0.0]       # 63.5 and 31.75: ties to even, up
    c, s = RO.quantise(np.array([[1.0, -2.0, 0.5, 0.0]]), "e4m3")
    assert s[0] == np.float32(2.0) / np.float32(448.0) and list(c[0]) == [224.0, -448.0, 112.0, 0.0]
    c, s = RO.quantise(np.array([[0.0, 0.0], [1e-38, 1.0], [np.inf, 1.0], [np.nan, 1.0], [2.0 ** -101, 0.0]]), "int8")
    assert list(s[:2]) == [0.0, np.float32(1.0) / np.float32(127.0)] and np.isnan(s[2]) and np.isnan(s[3]) and s[4] == 0
    assert not c[[0, 2, 3, 4]].any()
    x = np.random.default_rng(0).standard_normal((50, 64)).astype(np.float32)
    c, s = RO.quantise(x, "int8")
    assert np.all(np.abs(c) <= 127) and np.all(np.abs(c * s[:, None] - x) <= s[:, None] * 0.5001)


def test_places_of_rows():
    table = np.array([[4, 1, 0], [2, 9, 3]])
    got = RO.places([0, 2, 5], [18, 34], table, 16, 5, 6)
    assert got == [(1, 0), (1, 1), None, (3, 0), (3, 1), "padding"]       # position 31 lies on page 9 of 5
    assert RO.place(-1, table[0], 16, 5) is None and RO.place(48, table[0], 16, 5) is None


def test_what_rows_see():
    assert RO.seen_by(0, 3, 5) == [0, 1, 2] and RO.seen_by(2, 3, 5) == [0, 1, 2, 3, 4]
    assert RO.seen_by(2, 3, 5, window=2) == [3, 4] and RO.seen_by(2, 3, 5, max_len=4) == [0, 1, 2, 3]
    assert RO.seen_by(1, 3, 5, bits=0b010) == [0, 1, 3] and RO.seen_by(1, 3, 3, bits=0) == []
    assert RO.seen_by(0, 4, 2) == []                                      # position -2


def test_attention_of_one_row():
    K, V = np.array([[1.0, 0.0], [0.0, 1.0]]), np.array([[2.0, -4.0], [6.0, 0.0]])
    o, lse, a, _ = RO.attend_row(np.array([math.log(3.0), 0.0]), K, V, 1.0)
    assert np.allclose(o, [3.0, -3.0]) and lse == pytest.approx(math.log(4.0)) and np.allclose(a, [3.0, 3.0])
    o, lse, _, _ = RO.attend_row(np.ones(2), K[:0], V[:0], 1.0)
    assert not o.any() and lse == -math.inf


def test_adjusted_logits_of_one_row():
    x, _ = RO.adjust_row([2.0, -2.0, 1.0, 0.5, 3.0], asked=[0, 1, 99], said=[2, 2, 4, -1], penalties=(2.0, 0.25, 0.125, 0.5), bias={3: 1.5, 2: -1.0, 77: 9.0},
                         allowed=np.array([1, 1, 1, 1, 0], dtype=bool))
    # 2/2; -2*2; 1/2 - (2*0.125 + 0.25) - 1; 0.5 + 1.5; masked; all over 0.5
    assert list(x) == [2.0, -8.0, -2.0, 4.0, -math.inf]
    x, _ = RO.adjust_row([1.0, 2.0], [], [], (1, 0, 0, 0.0), {}, None)
    assert list(x) == [1.0, 2.0]
