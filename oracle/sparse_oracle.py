"""CPU oracle of page tables, rotary positions, and attention over selected pages.

Written from the definitions in include/covspec.h: one sequence, one page, one row at a time; integers are Python's, angles exact fractions of a turn,
the rest fp64, but for the codes of a summary and the scores, whose definition is fp32 arithmetic with each operation rounded on its own.
"""
from __future__ import annotations

import math
from decimal import Decimal, getcontext

import numpy as np

from oracle import round_oracle as RO

getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


class Tables:
    """The state of covspec_pages_step: what each sequence holds, and the stack of free pages."""

    def __init__(self, n_seq, page_size, n_pages, max_pages, free):
        self.page_size, self.n_pages, self.max_pages = page_size, n_pages, max_pages
        self.held, self.borrowed, self.free = [[] for _ in range(n_seq)], [0] * n_seq, list(free)

    def step(self, want, rows, n_tokens):
        """(start, length, outcome, slots, positions)."""
        S, page = len(self.held), self.page_size
        want = [max(int(w), 0) for w in want]
        rows = [min(max(int(r), 0), w) for r, w in zip(rows, want)]
        need = [-(-w // page) for w in want]
        back = []
        for s in range(S):
            if need[s] <= self.max_pages and len(self.held[s]) > need[s]:
                back += self.held[s][max(need[s], self.borrowed[s]):]
                self.held[s] = self.held[s][:need[s]]
        self.free = (self.free + back[::-1])[:self.n_pages]
        outcome, stopped = [0] * S, False
        for s in range(S):
            if need[s] > self.max_pages:
                outcome[s] = 1
                continue
            asks = need[s] - len(self.held[s])
            if asks > 0:
                stopped = stopped or asks > len(self.free)
                if stopped:
                    outcome[s] = 1
                else:
                    self.held[s] = self.held[s] + [self.free.pop() for _ in range(asks)]
        self.borrowed = [min(b, len(h)) for b, h in zip(self.borrowed, self.held)]
        used, start, length, slots, positions = 0, [0], [], [], []
        upto = 0                                        # rows asked for, with those left out
        for s in range(S):
            n = rows[s] if outcome[s] == 0 else 0
            upto += n
            if n > 0 and upto > n_tokens:
                outcome[s] = 2
            if outcome[s]:
                n = 0
                length.append(min(want[s] - rows[s], len(self.held[s]) * page))
            else:
                length.append(want[s])
            for j in range(want[s] - n, want[s]):
                at = self.held[s][j // page]
                slots.append(at * page + j % page if 0 <= at < self.n_pages else -1)
                positions.append(j)
            used += n
            start.append(used)
        pad = n_tokens - used
        return start, length, outcome, slots + [-1] * pad, positions + [-1] * pad


def rotary_turns(R, base, kind="plain", factor=1.0, original=0, low=0.0, high=0.0):
    """Turns from one position to the next, pair by pair, to 60 digits."""
    base, factor = Decimal(base), Decimal(factor)
    if kind == "base":
        base = base * factor ** (Decimal(R) / Decimal(R - 2))
    out = []
    for i in range(R // 2):
        f = base ** (Decimal(-2 * i) / Decimal(R))
        keep = Decimal(1)
        if kind == "linear":
            f = f / factor
        if kind == "bands":
            keep = (Decimal(original) * f / (2 * PI) - Decimal(low)) / (Decimal(high) - Decimal(low))
        if kind == "ramp":
            at = lambda turns: R * (Decimal(original) / (Decimal(turns) * 2 * PI)).ln() / (2 * base.ln())       # noqa: E731
            a = max(math.floor(at(high)), 0)
            b = min(math.ceil(at(low)), R - 1)
            keep = 1 - Decimal(i - a) / max(Decimal(b - a), Decimal("0.001"))
        if kind in ("bands", "ramp"):
            keep = min(max(keep, Decimal(0)), Decimal(1))
            f = f * (keep + (1 - keep) / factor)
        out.append(f / (2 * PI))
    return out


def cos_sin(pos, step):
    """Of pos * step 2^-64 turns, step a whole number: the turn's fraction is exact, around the nearest quarter in fp64."""
    u = (int(pos) * int(step)) % (1 << 64)
    quarter = (u + (1 << 61)) >> 62
    x = (u - (quarter << 62)) * (2.0 * math.pi / 2.0 ** 64)
    c, s = math.cos(x), math.sin(x)
    return [(c, s), (-s, c), (-c, -s), (s, -c)][quarter % 4]


def turned(x, positions, steps, interleaved, magnitude=1.0):
    """A row [D] with its pair i at positions[i]; and, element by element, the magnitude its roundings go by."""
    y, size = np.array(x, dtype=np.float64), np.zeros(len(x))
    h = len(steps)
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        c, s = cos_sin(positions[i], steps[i])
        y[a], y[b] = magnitude * (x[a] * c - x[b] * s), magnitude * (x[b] * c + x[a] * s)
        size[a] = size[b] = abs(magnitude) * (abs(x[a]) + abs(x[b]))
    return y, size


def summarise(k):
    """Codes [2, D] and the scale of the keys [n, D] (fp32) of a page."""
    k = np.asarray(k, dtype=np.float32)
    if not np.isfinite(k).all():
        return np.zeros((2, k.shape[1]), dtype=np.int8), np.float32(np.nan)
    both = np.stack([k.max(0), k.min(0)])
    c, s = RO.quantise(both.reshape(1, -1), "int8")
    return c.reshape(both.shape).astype(np.int8), s[0]


def scores(q, summary, scale):
    """fp32 scores of blocks [nb, 2, D] (with scales [nb]) for the query heads [G, D] of a row: the largest over the heads, NaN if one is."""
    c, s = RO.quantise(q, "int8")
    c = c.astype(np.int64)
    m = summary.astype(np.int64)
    best = None
    for h in range(len(c)):
        dot = (np.maximum(c[h], 0) * m[:, 0] + np.minimum(c[h], 0) * m[:, 1]).sum(1)
        with np.errstate(invalid="ignore", over="ignore"):
            z = (dot.astype(np.float32) * scale.astype(np.float32)).astype(np.float32) * np.float32(s[h])
        best = z if best is None else np.maximum(best, z)            # NaN wins
    return best


def choose(z, exists, nb, top, first, recent):
    """Blocks taken of 0 .. nb - 1 by the scores z, ascending."""
    forced = [b for b in range(nb) if b < first or b >= nb - recent]
    others = [b for b in range(nb) if first <= b < nb - recent and exists[b]]
    nan = sorted(b for b in others if np.isnan(z[b]))
    rest = sorted((b for b in others if not np.isnan(z[b])), key=lambda b: (-float(z[b]), b))
    return sorted(forced + (nan + rest)[:max(0, top - len(forced))])
