"""Pins of oracle/sparse_oracle.py: values worked out by hand, and independent statements of the same definitions."""
import math

import numpy as np
import pytest

from oracle import sparse_oracle as SO


def test_tables_by_hand():
    t = SO.Tables(3, 16, 6, 4, [5, 4, 3, 2, 1, 0])
    assert t.step([20, 0, 16], [20, 0, 1], 30) == ([0, 20, 20, 21], [20, 0, 16], [0, 0, 0], list(range(20)) + [2 * 16 + 15] + [-1] * 9, list(range(20)) + [15] + [-1] * 9)
    assert t.held == [[0, 1], [], [2]] and t.free == [5, 4, 3]
    # the first one ends, the second asks for four pages: two come back, last one first, and are the first to go out
    assert t.step([0, 50, 17], [0, 50, 1], 51) == ([0, 0, 50, 51], [0, 50, 17], [0, 0, 0], [0 * 16 + i for i in range(16)] + [16 + i for i in range(16)] +
                                                   [3 * 16 + i for i in range(16)] + [4 * 16, 4 * 16 + 1, 5 * 16], list(range(50)) + [16])
    assert t.held == [[], [0, 1, 3, 4], [2, 5]] and t.free == []
    # nothing left: the first goes empty-handed, and with it the third that asks; the second shrinks, one row does not fit
    assert t.step([1, 49, 40], [1, 4, 8], 3)[:3] == ([0, 0, 0, 0], [0, 45, 32], [1, 2, 1])
    t = SO.Tables(2, 16, 3, 2, [0, 1, 2])
    assert t.step([33, 16], [1, 1], 9)[2] == [1, 0] and t.held == [[], [2]]             # more than a table's width
    t.borrowed = [0, 1]
    t.step([0, 0], [0, 0], 1)
    assert t.free == [0, 1] and t.borrowed == [0, 0]                                    # somebody else's


def test_growing_and_shrinking_again_leaves_the_stack_as_it_was():
    rng = np.random.default_rng(0)
    t = SO.Tables(9, 16, 200, 20, rng.permutation(200))
    t.step(a := rng.integers(0, 200, 9), a * 0 + 1, 100)
    before = [list(h) for h in t.held], list(t.free)
    t.step(rng.integers(0, 200, 9), a * 0 + 1, 100)
    t.step(a, a * 0 + 1, 100)
    assert ([list(h) for h in t.held], t.free) == before


def test_turns():
    f = [2 * math.pi * float(x) for x in SO.rotary_turns(8, 10000.0)]
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001], rtol=1e-15)
    assert np.allclose([2 * math.pi * float(x) for x in SO.rotary_turns(8, 10000.0, "linear", 4.0)], np.array(f) / 4, rtol=1e-15)
    # the lowest frequency is divided by the factor, the highest stays
    g = [2 * math.pi * float(x) for x in SO.rotary_turns(8, 10000.0, "base", 4.0)]
    assert g[0] == 1.0 and np.isclose(g[-1], f[-1] / 4, rtol=1e-14)
    # 1000 positions: 159, 15.9, 1.59, 0.159 turns
    g = [2 * math.pi * float(x) for x in SO.rotary_turns(8, 10000.0, "bands", 8.0, 1000, 1.0, 4.0)]
    keep = (1000 * 0.01 / (2 * math.pi) - 1) / 3
    assert np.allclose(g, [1.0, 0.1, 0.01 * (keep + (1 - keep) / 8), 0.001 / 8], rtol=1e-14)
    # 4 turns at index 4 log10(1000 / 8 pi) / 4 = 1.6, 1 turn at 2.2: from 1 to 3
    g = [2 * math.pi * float(x) for x in SO.rotary_turns(8, 10000.0, "ramp", 8.0, 1000, 1.0, 4.0)]
    assert np.allclose(g, [1.0, 0.1, 0.01 * (0.5 + 0.5 / 8), 0.001 / 8], rtol=1e-14)


@pytest.mark.parametrize("interleaved", [False, True])
def test_turning(interleaved):
    rng = np.random.default_rng(1)
    x = rng.standard_normal(12)
    steps = [int(t * (1 << 64)) for t in SO.rotary_turns(8, 100.0)]
    y, size = SO.turned(x, [3, 5, -7, 1000003], steps, interleaved, 1.5)
    for i, pos in enumerate([3, 5, -7, 1000003]):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + 4)
        z = complex(x[a], x[b]) * 1.5 * np.exp(1j * pos * 100.0 ** (-i / 4))
        assert abs(complex(y[a], y[b]) - z) < 1e-9 and size[a] == size[b] == pytest.approx(1.5 * (abs(x[a]) + abs(x[b])))
    assert np.array_equal(y[8:], x[8:])
    back, _ = SO.turned(y, [-3, -5, 7, -1000003], steps, interleaved, 1 / 1.5)
    assert np.allclose(back, x, atol=1e-12)


def test_scores_bound_the_products_and_choices_go_by_them():
    rng = np.random.default_rng(2)
    k, q = rng.standard_normal((9, 16, 32)).astype(np.float32), rng.standard_normal((3, 32)).astype(np.float32)
    made = [SO.summarise(x) for x in k]
    z = SO.scores(q, np.stack([m[0] for m in made]), np.array([m[1] for m in made]))
    # a code is off by half a step of each scale: D (1/254) (|largest| + |q|) and so on, well below 3 %
    assert np.all(z >= (k @ q.T).max((1, 2)) - 0.03 * np.abs(k).max() * np.abs(q).max() * 32)
    exists = [True] * 9
    z = np.array([9.0, 1.0, np.nan, 3.0, 3.0, 2.0, np.nan, 0.0, 5.0], dtype=np.float32)
    assert SO.choose(z, exists, 9, 5, 1, 1) == [0, 2, 3, 6, 8] and SO.choose(z, exists, 9, 4, 0, 1) == [0, 2, 6, 8]
    assert SO.choose(z, [False] * 2 + [True] * 7, 8, 9, 1, 0) == [0, 2, 3, 4, 5, 6, 7] and SO.choose(z, exists, 2, 9, 1, 4) == [0, 1]
    c, s = SO.summarise(np.array([[1.0, -2.0], [0.5, 3.0]]))
    assert c.tolist() == [[42, 127], [21, -85]] and s == np.float32(3.0) / np.float32(127.0)
    assert np.isnan(SO.summarise(np.array([[1.0, np.inf]]))[1])
