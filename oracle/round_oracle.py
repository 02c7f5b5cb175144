"""CPU oracle of what surrounds the verification of a drafted segment: paged cache, attention over it, adjustments of logits.

Written from the definitions in include/covspec.h, in fp64 but for the codes of the cache, whose definition is fp32 arithmetic with each operation
rounded on its own.  One row, one position, one word at a time where that costs nothing.
"""
from __future__ import annotations

import math

import numpy as np

Q = {"int8": np.float32(127.0), "e4m3": np.float32(448.0)}
TINY = np.float32(2.0 ** -100)


def e4m3_nearest(y):
    """Values of 4 exponent bits (bias 7) and 3 of significand next to y (|y| <= 448), ties to even: steps of 2^(e - 3), e >= -6."""
    y = np.asarray(y, dtype=np.float64)
    a = np.abs(y)
    e = np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -30))), -6.0)
    step = 2.0 ** (e - 3)
    return np.copysign(np.rint(a / step) * step, y)        # np.rint: ties to even


def quantise(x, kept):
    """Codes (as the values they stand for) and scales of rows [..., D] of fp32 values."""
    x = np.asarray(x, dtype=np.float32)
    top = np.max(np.abs(x), axis=-1)                       # NaN where one is in the row
    finite = np.isfinite(top)
    use = finite & (top >= TINY)
    safe = np.where(use, top, np.float32(1.0)).astype(np.float32)
    scale = np.where(finite, np.where(use, safe / Q[kept], np.float32(0.0)), np.float32(np.nan)).astype(np.float32)
    inv = (np.float32(1.0) / safe).astype(np.float32) * Q[kept]
    with np.errstate(invalid="ignore"):
        y = np.where(use[..., None], x * inv[..., None], np.float32(0.0)).astype(np.float32)
    y = np.clip(y, -Q[kept], Q[kept])
    return (np.rint(y) if kept == "int8" else e4m3_nearest(y)).astype(np.float32), scale


def places(start, length, pages, page_size, n_pages, n_tokens):
    """For every row: (page, place), None where its position does not exist, "padding" for a row of no sequence."""
    out = ["padding"] * n_tokens
    for s in range(len(length)):
        n = start[s + 1] - start[s]
        for i in range(n):
            out[start[s] + i] = place(length[s] - n + i, pages[s], page_size, n_pages)
    return out


def place(pos, table, page_size, n_pages):
    if pos < 0 or pos // page_size >= len(table):
        return None
    page = int(table[pos // page_size])
    return (page, pos % page_size) if 0 <= page < n_pages else None


def seen_by(i, n, length, window=0, bits=None, max_len=None):
    """Positions that row i of a chunk of n sees of a sequence of `length` tokens."""
    old = length - n
    if bits is not None:
        j = [j for j in range(0, max(old, 0))] + [old + b for b in range(min(n, 64)) if bits >> b & 1]
    else:
        pos = old + i
        j = list(range(max(0, pos + 1 - window) if window else 0, pos + 1))
    return [x for x in j if x >= 0 and (max_len is None or x < max_len)]


def attend_row(q, K, V, scale):
    """One row over the keys and values it sees, fp64: (o, lse, sum p |v| / sum p, largest sum |q k| scale)."""
    D = q.shape[0]
    if len(K) == 0:
        return np.zeros(D), -math.inf, np.zeros(D), 0.0
    z = (K @ q) * scale
    m = z.max()
    p = np.exp(z - m)
    total = p.sum()
    return (p @ V) / total, m + math.log(total), (p @ np.abs(V)) / total, float((np.abs(K) @ np.abs(q)).max() * abs(scale))


def adjust_row(z, asked, said, penalties, bias, allowed):
    """One position: z [V] fp64, words of the prompt and said since, (r, c, f, T), {word: bias}, bool [V] or None.
    Returns the logits and, word by word, the magnitude that their roundings go by."""
    r, c, f, T = (float(x) for x in penalties)
    V = len(z)
    n = np.bincount([w for w in said if 0 <= w < V], minlength=V).astype(np.float64)
    any_ = (np.bincount([w for w in asked if 0 <= w < V], minlength=V) + n) > 0
    x = np.array(z, dtype=np.float64)
    x = np.where(any_, np.where(x > 0, x / r, x * r), x)
    less = f * n + c * (n > 0)
    b = np.zeros(V)
    for w, v in bias.items():
        if 0 <= w < V:
            b[w] = v
    t = 1.0 / T if T > 0 else 1.0
    size = (np.abs(x) + np.abs(f) * n + np.abs(c) * (n > 0) + np.abs(b)) * t
    x = (x - less + b) * t
    if allowed is not None:
        x = np.where(allowed, x, -math.inf)
    return x, size
