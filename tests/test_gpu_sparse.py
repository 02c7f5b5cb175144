"""GPU parity of covspec_block_summary and covspec_sparse_attend with oracle/sparse_oracle.py.  Summaries and the choice of blocks are defined in exact integers and
single fp32 operations, so they are compared as they are.

Tolerance of an output, with u = half a step of the 16-bit type, A = sum p |v| / sum p and S = the largest sum |q k| scale of the row:
  u |o|           the output's own rounding
  w A             p's rounding for its product with v: w = 2^-11 in fp16 over an fp16 cache; else p (times v's scale) goes in as two bf16 parts, each of 8 bits: 2^-16
  e A, e = 2 (D + 64) 2^-24 S + 2^-19
                  scores off by the fp32 sums move every p by that much, numerator and denominator; fp32 exponentials, sums over the positions and
                  the joining of pieces: 2^-19
  2^-25 sum |v|   fp16 over an fp16 cache: p below 2^-14 has fixed steps of 2^-24
  2^-25           the same for the output itself
The log-sum: 2 (D + 64) 2^-24 S + 2^-20 (1 + |lse|)."""
import math

import numpy as np
import pytest

from oracle import round_oracle as RO
from oracle import sparse_oracle as SO
from round_util import HALF_STEP, Batch, pool_of, rounded, torch_dtype

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "bf16"), ("bf16", "int8"), ("bf16", "e4m3"), ("fp16", "fp16"), ("fp16", "int8"), ("fp16", "e4m3")]


def k32_of(pool):
    """The keys of a pool as the definition of a summary has them: fp32 values, code * scale rounded once."""
    v = pool[0].float().numpy()
    return v if pool[1] is None else (v * pool[1].numpy()[..., None]).astype(np.float32)


def summaries(b, k32, H, D, garbage=7):
    """All pages' summaries over what their sequences hold of them; pages of no sequence hold garbage."""
    codes = np.full((b.n_pages, H, 2, D), garbage, dtype=np.int8)
    scale = np.full((b.n_pages, H), 1e30, dtype=np.float32)
    for s in range(b.S):
        for blk in range(-(-max(b.length[s], 0) // b.page)):
            at = RO.place(blk * b.page, b.pages[s], b.page, b.n_pages)
            if at is not None:
                for h in range(H):
                    codes[at[0], h], scale[at[0], h] = SO.summarise(k32[at[0], h, :min(b.page, b.length[s] - blk * b.page)])
    return codes, scale


def make(rng, b, heads, H, D, dtype, kept):
    x = rng.standard_normal((b.n_pages, H, b.page, D)) + 0.8 * rng.standard_normal((b.n_pages, H, 1, D))
    x[..., 3::29] *= 4.0
    v = rng.standard_normal((b.n_pages, H, b.page, D)) * np.exp(0.5 * rng.standard_normal((b.n_pages, H, b.page, 1)))
    q, q32 = rounded(rng.standard_normal((b.T, heads, D)), dtype)
    return pool_of(x, kept, dtype), pool_of(v, kept, dtype), q, q32


def upload(k, v):
    return tuple(None if t is None else t.cuda() for t in (k[0], v[0], k[1], v[1]))


def row_end(b, s, i, tree, cap):
    n = b.new[s]
    return max(0, min(b.length[s] - n + (min(n, 64) if tree else i + 1), cap))


def wanted_blocks(b, codes, scale, q32, heads, H, top, first, recent, tree, cap):
    G, out = heads // H, np.full((b.T, H, top), -2)
    for s in range(b.S):
        for i in range(b.new[s]):
            t, nb = int(b.start[s]) + i, -(-row_end(b, s, i, tree, cap) // b.page)
            ids = [int(b.pages[s][x]) for x in range(nb)]
            exists = [0 <= x < b.n_pages for x in ids]
            safe = [x if ok else 0 for x, ok in zip(ids, exists)]
            for g in range(H):
                z = SO.scores(q32[t, g * G:(g + 1) * G], codes[safe, g], scale[safe, g]) if nb else []
                c = SO.choose(z, exists, nb, top, first, recent)
                out[t, g] = c + [-1] * (top - len(c))
    return out


def check_rows(b, blocks, heads, H, D, dtype, kept, k64, v64, q32, out, lse, scale, visible, cap, rows=None):
    G, u = heads // H, HALF_STEP[dtype]
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    plain = dtype == "fp16" and kept == "fp16"
    for s in range(b.S):
        n, length = b.new[s], b.length[s]
        for i in range(n):
            t = int(b.start[s]) + i
            if rows is not None and t not in rows:
                continue
            seen = set(RO.seen_by(i, n, length, 0, None if visible is None else int(visible[t]) & ((1 << 64) - 1), cap))
            for g in range(H):
                listed = [x for x in blocks[t, g] if x >= 0]
                js = [j for x in listed for j in range(x * b.page, (x + 1) * b.page) if j in seen]
                at = [p for p in (RO.place(j, b.pages[s], b.page, b.n_pages) for j in js) if p is not None]
                pg, of = np.array([p[0] for p in at], dtype=int), np.array([p[1] for p in at], dtype=int)
                K, V = k64[pg, g, of].reshape(-1, D), v64[pg, g, of].reshape(-1, D)
                for h in range(g * G, (g + 1) * G):
                    o, e, A, size = RO.attend_row(q32[t, h].astype(np.float64), K, V, scale)
                    rel = 2 * (D + 64) * 2.0 ** -24 * size
                    tol = u * np.abs(o) + (2.0 ** (-11 if plain else -16) + rel + 2.0 ** -19) * A + 2.0 ** -25
                    if plain and len(at):
                        tol = tol + 2.0 ** -25 * np.abs(V).sum(0)
                    where = "sequence %d row %d head %d (%d seen)" % (s, i, h, len(at))
                    err = np.abs(out[t, h] - o) - tol
                    assert np.all(err <= 0), "%s: off by %g beyond the tolerance" % (where, err.max())
                    if len(at) == 0:
                        assert lse[t, h] == -math.inf and not out[t, h].any(), where
                    else:
                        assert abs(lse[t, h] - e) <= rel + 2.0 ** -20 * (1 + abs(e)), where


def run(b, heads, H, D, dtype, kept, top, first=1, recent=1, seed=0, visible=None, max_len=None, rows=None):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(seed)
    k, v, q, q32 = make(rng, b, heads, H, D, dtype, kept)
    codes, scale = summaries(b, k32_of(k), H, D)
    cap = min(max_len or max(max(b.length), 1), b.width * b.page)
    p = C.SparseParams(C.AttendParams(b.params(H, D, dtype, kept), heads, cap, D ** -0.5), top, first, recent)
    out = torch.full((b.T, heads, D), 7.0, dtype=torch_dtype(dtype), device="cuda")
    blocks = torch.full((b.T, H, top), -2, dtype=torch.int32, device="cuda")
    vis = None if visible is None else torch.from_numpy(np.asarray(visible, dtype=np.int64)).cuda()
    ws = torch.full((C.sparse_workspace_size(p) + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse, got = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), (torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda()), visible=vis, out=out,
                                    want_lse=True, blocks_out=blocks, workspace=ws)
    torch.cuda.synchronize()
    want = wanted_blocks(b, codes, scale, q32, heads, H, top, first, recent, visible is not None, cap)
    np.testing.assert_array_equal(got.cpu().numpy(), want)
    check_rows(b, want, heads, H, D, dtype, kept, k[2], v[2], q32, out, lse, D ** -0.5, visible, cap, rows)
    assert bool((out[int(b.start[-1]):] == 7.0).all())
    return got


# ---------------------------------------------------------------- summaries
@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("D,H,page,new,length", [(64, 3, 16, [5, 0, 1, 40, 3], [5, 30, 77, 131, 2]), (96, 2, 32, [100, 1], [230, 64]), (128, 8, 64, [300, 7, 1], [300, 129, 1]),
                                                 (128, 1, 1024, [1, 2], [1500, 1025]), (64, 2, 256, [700, 1], [900, 257]), (128, 2, 16, [1] * 70, list(range(1, 71)))])
def test_summaries_equal_the_oracle(dtype, kept, D, H, page, new, length):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(D + page)
    b = Batch(rng, new, length, page, pad=2)
    b.pages[-1, -1] = b.n_pages if len(new) == 3 else b.pages[-1, -1]
    k = pool_of(rng.standard_normal((b.n_pages, H, page, D)) * np.exp(rng.standard_normal((b.n_pages, H, 1, 1))), kept, dtype)
    if kept != dtype:
        k[1][b.pages[0, 0], 0, 0] = float("nan")            # a row that held an infinity
    elif page < 64:
        k[0][b.pages[0, 0], 0, 1, 3], k[0][b.pages[1, 0], 1, 0, :] = -float("inf"), 0.0
    p = b.params(H, D, dtype, kept)
    summary = (torch.full((b.n_pages, H, 2, D), 7, dtype=torch.int8, device="cuda"), torch.full((b.n_pages, H), 1e30, device="cuda"))
    C.block_summary(p, *b.device(), upload(k, k), summary)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        k32 = k32_of((k[0], k[1]))
    want = np.full((b.n_pages, H, 2, D), 7, dtype=np.int8), np.full((b.n_pages, H), 1e30, dtype=np.float32)
    for s in range(b.S):
        for blk in sorted({(b.length[s] - b.new[s] + i) // page for i in range(b.new[s]) if b.length[s] - b.new[s] + i >= 0}):
            at = RO.place(blk * page, b.pages[s], page, b.n_pages)
            if at is not None:
                for h in range(H):
                    want[0][at[0], h], want[1][at[0], h] = SO.summarise(k32[at[0], h, :min(page, b.length[s] - blk * page)])
    np.testing.assert_array_equal(summary[0].cpu().numpy(), want[0])
    np.testing.assert_array_equal(summary[1].cpu().numpy(), want[1])


def test_summaries_of_many_sequences():
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(6)
    new = [int(n) for n in rng.integers(0, 4, 300)] + [3000]
    b = Batch(rng, new, [n + int(rng.integers(0, 40)) for n in new], 16)
    k = pool_of(rng.standard_normal((b.n_pages, 1, 16, 64)), "bf16", "bf16")
    codes, scale = summaries(b, k32_of(k), 1, 64)
    for cut in (300, 301):                                  # by rows, and with a prompt behind them by pages
        sub = Batch.__new__(Batch)
        sub.__dict__.update(b.__dict__, new=new[:cut], length=b.length[:cut], S=cut, pages=b.pages[:cut], start=b.start[:cut + 1], T=int(b.start[cut]))
        summary = C.block_alloc(sub.params(1, 64, "bf16", "bf16"))
        C.block_summary(sub.params(1, 64, "bf16", "bf16"), *sub.device(), upload(k, k), summary)
        torch.cuda.synchronize()
        for s in range(cut):
            old = sub.length[s] - new[s]
            for blk in range(old // 16, -(-sub.length[s] // 16)) if new[s] else ():
                pg = sub.pages[s, blk]
                assert np.array_equal(summary[0][pg].cpu().numpy(), codes[pg]) and float(summary[1][pg]) == scale[pg, 0], (s, blk)


# ---------------------------------------------------------------- the choice and the attention over it
@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("D,page,heads,H", [(64, 16, 8, 2), (96, 32, 3, 3), (128, 64, 16, 2), (128, 16, 5, 1)])
def test_single_tokens(dtype, kept, D, page, heads, H):
    rng = np.random.default_rng(1)
    run(Batch(rng, [1] * 7, [1, 2, 63, 64, 65, 700, 1333], page, pad=2), heads, H, D, dtype, kept, top=6, first=1, recent=2)


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("heads,H,D,page,top", [(6, 6, 64, 64, 3), (16, 2, 128, 32, 9), (17, 1, 96, 16, 20), (40, 1, 64, 16, 8), (64, 1, 128, 128, 4), (12, 4, 128, 256, 2)])
def test_drafted_segments(dtype, kept, heads, H, D, page, top):
    rng = np.random.default_rng(2)
    run(Batch(rng, [8, 5, 0, 1, 9, 3], [300, 5, 40, 129, 64, 1000], page, pad=1), heads, H, D, dtype, kept, top, first=0, recent=1)


@pytest.mark.parametrize("dtype,kept", [("bf16", "bf16"), ("fp16", "e4m3"), ("fp16", "int8")])
@pytest.mark.parametrize("new,top,recent", [(8, 12, 3), (64, 6, 1), (70, 8, 2)])
def test_trees(dtype, kept, new, top, recent):
    rng = np.random.default_rng(new)
    b = Batch(rng, [new, 3, new], [500, 3, 333], 16)
    bits = []
    for n in b.new:
        seen = []
        for i in range(n):
            seen.append(((seen[int(rng.integers(0, min(i, 64)))] if i else 0) | 1 << min(i, 63)) & ((1 << 64) - 1))
        seen[n // 2] = 0                                    # one that sees nothing of the chunk
        bits += [x - (1 << 64) if x >> 63 else x for x in seen]
    run(b, 8, 2, 64, dtype, kept, top, 1, recent, visible=bits, rows=set(range(0, b.T, 3)))


@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
@pytest.mark.parametrize("length,page,top", [(20000, 16, 33), (60000, 16, 64), (131000, 16, 17), (30000, 32, 1024), (9000, 16, 512)])
def test_long_sequences(kept, length, page, top):
    """Every form of the choice (1024, 4096, 32768 blocks), lists in many pieces."""
    rng = np.random.default_rng(length)
    run(Batch(rng, [2, 1], [length, length // 3], page), 4, 2, 64, "bf16", kept, top, 1, 2)


@pytest.mark.parametrize("top,first,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (5, 5, 0), (5, 0, 5), (5, 2, 3), (200, 3, 3)])
def test_blocks_that_are_always_taken(top, first, recent):
    rng = np.random.default_rng(5)
    got = run(Batch(rng, [1, 2, 1], [1, 300, 2000], 16), 4, 2, 64, "bf16", "bf16", top, first, recent)
    assert got.shape[-1] == top


def test_max_len_bounds_what_is_seen():
    rng = np.random.default_rng(6)
    run(Batch(rng, [3, 1], [900, 200], 32), 4, 2, 64, "fp16", "fp16", 5, 1, 1, max_len=333)


def test_positions_that_do_not_exist():
    rng = np.random.default_rng(7)
    b = Batch(rng, [4, 3, 1], [2, 200, 300], 16)            # two rows in front of the first sequence
    b.pages[1, 4], b.pages[1, 5], b.pages[2, 0], b.pages[2, 18] = -1, b.n_pages, 1 << 30, -5
    b.length[2] = 16 * b.width + 3                          # rows beyond the table
    run(b, 4, 2, 64, "bf16", "int8", 8, 1, 2)


def test_scores_that_tie_or_are_not_numbers():
    """Equal summaries go to the lower block; a page with a NaN key comes first; a query of NaN or of zeros ties all."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(8)
    b = Batch(rng, [4], [640], 16)
    H, heads, D, top = 1, 2, 64, 7
    x = np.tile(rng.standard_normal((1, H, 16, D)), (b.n_pages, 1, 1, 1))
    x[b.pages[0, 20], 0, 3, 5], x[b.pages[0, 30], 0, 3, 5] = np.nan, np.inf
    x[b.pages[0, 25]] *= 1.5
    k, v = pool_of(x, "bf16", "bf16"), pool_of(rng.standard_normal(x.shape), "bf16", "bf16")
    q, _ = rounded(rng.standard_normal((4, heads, D)), "bf16")
    q[1, 0, 0], q[2] = float("nan"), 0.0
    q[3, 1, 7] = float("inf")
    p = C.SparseParams(C.AttendParams(b.params(H, D, "bf16", "bf16"), heads, 640, 0.1), top, 1, 1)
    summary = C.block_alloc(p.attend.cache)
    whole = b.params(H, D, "bf16", "bf16")
    whole.n_tokens = 640
    C.block_summary(whole, torch.tensor([0, 640], dtype=torch.int32, device="cuda"), *b.device()[1:], upload(k, v), summary)
    _, _, got = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), summary)
    codes, scale = summaries(b, k32_of(k), H, D)
    assert np.isnan(scale[b.pages[0, 20], 0]) and np.isnan(scale[b.pages[0, 30], 0])
    want = wanted_blocks(b, codes, scale, q.float().numpy(), heads, H, top, 1, 1, False, 640)
    np.testing.assert_array_equal(got.cpu().numpy(), want)
    assert {20, 25, 30} <= set(want[0, 0]) and list(want[1, 0]) == [0, 1, 2, 3, 4, 5, 39] == list(want[3, 0])
    assert list(want[2, 0]) == [0, 1, 2, 3, 20, 30, 39]     # zeros: every block scores zero but those with NaN


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("heads", [4, 40])
def test_what_a_row_does_not_see_has_no_effect(dtype, kept, heads):
    """NaN and infinities in the pages behind the row, in its own page behind it, in blocks that are not listed, on a page that does not exist."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(9)
    b = Batch(rng, [3], [203], 32)
    H, D, top = 1, 64, 4
    k, v, q, q32 = make(rng, b, heads, H, D, dtype, kept)
    k64, v64 = np.array(k[2]), np.array(v[2])
    p = C.SparseParams(C.AttendParams(b.params(H, D, dtype, kept), heads, 203, 0.1), top)
    lists = np.array([[[6, 2, -1, 3]], [[6, 2, -1, 3]], [[3, 2, 6, 4]]], dtype=np.int32)
    b.pages[0, 4] = -1                                      # listed by the last row; the first page of the pool is loaded in its place
    clean = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), None, blocks=torch.from_numpy(lists).cuda(), want_lse=True)
    for pool in (k, v):
        t, bad = pool[0], float("nan")
        for pg, of in [(b.pages[0, 6], slice(11, None)), (b.pages[0, 1], slice(None)), (b.pages[0, 5], slice(None)), (0, slice(None)) if 0 not in b.pages[0, [2, 3, 6]] else (b.pages[0, 1], slice(None))]:
            if kept == "int8":
                t[pg, :, of] = 127
            else:
                t[pg, :, of] = bad
            if pool[1] is not None:
                pool[1][pg, :, of] = bad
    spoilt = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), None, blocks=torch.from_numpy(lists).cuda(), want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(clean[0], spoilt[0]) and torch.equal(clean[1], spoilt[1])
    check_rows(b, lists, heads, H, D, dtype, kept, k64, v64, q32, spoilt[0], spoilt[1], 0.1, None, 203)


def test_a_value_that_is_not_finite_reaches_the_rows_that_see_it():
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(10)
    b = Batch(rng, [2], [100], 16)
    k, v, q, _ = make(rng, b, 4, 1, 64, "bf16", "bf16")
    v[0][b.pages[0, 6], 0, 3, 9] = float("inf")             # position 99: the last row's own
    p = C.SparseParams(C.AttendParams(b.params(1, 64, "bf16", "bf16"), 4, 100, 0.1), 3)
    blocks = torch.tensor([[[0, 5, 6]]] * 2, dtype=torch.int32, device="cuda")
    out, _, _ = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), None, blocks=blocks)
    assert bool(torch.isfinite(out[0]).all()) and bool(torch.isinf(out[1, :, 9]).all()) and bool(torch.isfinite(out[1, :, :9]).all())


@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
def test_lists_of_the_caller(kept):
    """Any order, entries that are no block, the same block twice, lists of nothing; a list of all blocks is the attention over the whole cache."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(11)
    b = Batch(rng, [3, 1, 2], [200, 64, 5], 16, pad=1)
    H, heads, D, top = 2, 8, 64, 20
    k, v, q, q32 = make(rng, b, heads, H, D, "bf16", kept)
    a = C.AttendParams(b.params(H, D, "bf16", kept), heads, 200, 0.125)
    p = C.SparseParams(a, top)
    lists = rng.integers(-3, 14, (b.T, H, top)).astype(np.int32)
    lists[0, 0], lists[1, 1] = -1, 1 << 30
    lists[2, 0, :4] = [2, 2, 2, -2 ** 31]
    out, lse, same = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), None, blocks=(given := torch.from_numpy(lists).cuda()), want_lse=True)
    assert same is given and torch.equal(given.cpu(), torch.from_numpy(lists))
    usable = np.where(lists < b.width, lists, -1)
    check_rows(b, usable, heads, H, D, "bf16", kept, k[2], v[2], q32, out, lse, 0.125, None, 200)
    every = torch.arange(top, dtype=torch.int32, device="cuda").expand(b.T, H, top).contiguous()
    out, lse, _ = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), None, blocks=every, want_lse=True)
    whole, lse2 = C.attend(a, q.cuda(), *b.device(), upload(k, v), want_lse=True)
    n = int(b.start[-1])
    assert bool((lse[:n] - lse2[:n]).abs().max() < 1e-4) and bool((out[:n].float() - whole[:n].float()).abs().max() < 0.1)


@pytest.mark.parametrize("scale", [0.0, -0.2, 2.0])
def test_scales_of_the_scores(scale):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(12)
    b = Batch(rng, [2], [150], 16)
    k, v, q, q32 = make(rng, b, 4, 2, 64, "fp16", "fp16")
    lists = np.tile(np.array([1, 4, 9], dtype=np.int32), (2, 2, 1))
    p = C.SparseParams(C.AttendParams(b.params(2, 64, "fp16", "fp16"), 4, 150, scale), 3)
    out, lse, _ = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), None, blocks=torch.from_numpy(lists).cuda(), want_lse=True)
    check_rows(b, lists, 4, 2, 64, "fp16", "fp16", k[2], v[2], q32, out, lse, scale, None, 150)


def test_queries_and_outputs_as_columns_of_wider_rows():
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(13)
    b = Batch(rng, [3, 1], [300, 90], 16, pad=2)
    k, v, q, _ = make(rng, b, 4, 2, 64, "bf16", "bf16")
    codes, scale = summaries(b, k32_of(k), 2, 64)
    summary = torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda()
    p = C.SparseParams(C.AttendParams(b.params(2, 64, "bf16", "bf16"), 4, 300, 0.1), 5)
    want = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), summary, want_lse=True)
    wide = torch.full((b.T, 11, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:7] = q.cuda()
    got = C.sparse_attend(p, wide[:, 3:7], *b.device(), upload(k, v), summary, out=wide[:, 7:], want_lse=True)
    n = 4
    assert torch.equal(got[0][:n], want[0][:n]) and torch.equal(got[1][:n], want[1][:n]) and torch.equal(got[2][:n], want[2][:n])
    assert bool((wide[:, :3] == 7.0).all()) and bool((wide[n:, 7:] == 7.0).all()) and torch.equal(wide[:, 3:7], q.cuda())


def test_pools_beyond_four_gigabytes():
    import torch
    import paper_2605_02218_amd as C
    n_pages, page, H, D = 34000, 1024, 1, 128               # 8.9 GB in each pool
    p = C.CacheParams(1, 1, H, D, page, n_pages, 4, C.BF16, C.BF16)
    pool = C.cache_alloc(p)
    pages = torch.tensor([[33999, 5, 33990, 17000]], dtype=torch.int32, device="cuda")
    for i in pages[0].tolist():
        pool[0][i], pool[1][i] = 0.0, float(i)
    pool[1][33990, 0, 1:].fill_(float("nan"))
    start, length = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1], [2 * page + 1]))
    summary = C.block_alloc(p)
    C.block_summary(p, start, length, pages, pool, summary)
    q = torch.ones(1, 1, D, dtype=torch.bfloat16, device="cuda")
    out, _, blocks = C.sparse_attend(C.SparseParams(C.AttendParams(p, 1, 4 * page, 1.0), 2, 1, 1), q, start, length, pages, pool, summary)
    want = (33999.0 * page + 33990.0) / (page + 1)
    assert blocks[0, 0].tolist() == [0, 2] and abs(float(out[0, 0, 0]) - want) <= want * 2.0 ** -8


@pytest.mark.parametrize("S", [63, 64, 65, 130, 1100])
def test_many_sequences(S):
    """A token or none of each of many sequences; padding in front of none, behind all."""
    rng = np.random.default_rng(S)
    new = [int(n) for n in rng.integers(0, 3, S)]
    new[-1] = 1
    run(Batch(rng, new, [n + int(rng.integers(0, 130)) for n in new], 16, pad=3), 2, 1, 64, "bf16", "bf16", 4, 1, 1)


def test_queries_of_nan_choose_no_page_that_does_not_exist():
    rng = np.random.default_rng(15)
    b = Batch(rng, [2, 1], [300, 300], 16)
    b.pages[0, [2, 5]], b.pages[1, [1, 7]] = -1, b.n_pages
    import torch
    import paper_2605_02218_amd as C
    k, v, q, _ = make(rng, b, 4, 1, 64, "bf16", "bf16")
    q[0], q[2, 1, 3] = float("nan"), float("inf")
    codes, scale = summaries(b, k32_of(k), 1, 64)
    p = C.SparseParams(C.AttendParams(b.params(1, 64, "bf16", "bf16"), 4, 300, 0.1), 9, 1, 1)
    _, _, got = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), (torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda()))
    want = wanted_blocks(b, codes, scale, q.float().numpy(), 4, 1, 9, 1, 1, False, 300)
    np.testing.assert_array_equal(got.cpu().numpy(), want)
    assert list(want[0, 0]) == [0, 1, 3, 4, 6, 7, 8, 9, 18] and list(want[2, 0]) == [0, 2, 3, 4, 5, 6, 8, 9, 18]


@pytest.mark.parametrize("chosen", [True, False])
@pytest.mark.parametrize("T,S", [(9, 4), (300, 200)])
def test_arrays_without_sense_stay_inside_their_memory(chosen, T, S):
    """Starts that do not ascend, lengths, pages and blocks that are anything: marked memory around everything that is written."""
    import ctypes
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(T)
    H, heads, D, page, n_pages, width, top = 2, 4, 64, 16, 30, 6, 5
    p = C.SparseParams(C.AttendParams(C.CacheParams(S, T, H, D, page, n_pages, width, C.BF16, C.E4M3), heads, page * width, 0.1), top, 1, 1)
    wild = lambda *n: torch.from_numpy(rng.choice([-2 ** 31, -1, 0, 1, 3, 5, 29, 30, 50, 95, 2 ** 31 - 1], n).astype(np.int32)).cuda()        # noqa: E731
    for _ in range(4):
        rooms = []

        def guard(shape, dtype):
            n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
            room = torch.full((n + 1024,), 0x5A, dtype=torch.uint8, device="cuda")
            rooms.append((room, n))
            return room[512:512 + n].view(dtype).view(shape)

        cache = tuple(guard((n_pages, H, page, D), torch.float8_e4m3fn) for _ in range(2)) + tuple(guard((n_pages, H, page), torch.float32) for _ in range(2))
        summary = guard((n_pages, H, 2, D), torch.int8), guard((n_pages, H), torch.float32)
        q, out, lse = guard((T, heads, D), torch.bfloat16), guard((T, heads, D), torch.bfloat16), guard((T, heads), torch.float32)
        blocks = guard((T, H, top), torch.int32)
        blocks.copy_(wild(T, H, top))
        q.copy_(torch.randn(T, heads, D))
        start, length, pages = wild(S + 1), wild(S), wild(S, width)
        steps, c = C.rotary_steps(D), p.attend.cache
        C.rotate_write(C.RotaryParams(S, T, heads, H, D), c, q, q[:, :H], q[:, H:], steps, start, length, pages, cache, q_out=out)
        C.block_summary(c, start, length, pages, cache, summary)
        need = C.sparse_workspace_size(p, given=not chosen)
        ws = torch.full((need + 1024,), 0x5A, dtype=torch.uint8, device="cuda")
        at = (ws.data_ptr() + 255) // 256 * 256
        cs = p.c_struct(given=not chosen)
        st = C.load_library().covspec_sparse_attend(ctypes.byref(cs), q.data_ptr(), start.data_ptr(), length.data_ptr(), pages.data_ptr(), *[t.data_ptr() for t in cache],
                                                    *[t.data_ptr() for t in summary], None, blocks.data_ptr(), out.data_ptr(), lse.data_ptr(), at, need,
                                                    torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == 0
        for room, n in rooms:
            assert bool((room[:512] == 0x5A).all()) and bool((room[512 + n:] == 0x5A).all())
        assert bool((ws[at - ws.data_ptr() + need:] == 0x5A).all())


@pytest.mark.parametrize("heads", [2, 20])
@pytest.mark.parametrize("new,length,top", [([3], [600], 4), ([2], [6000], 4), ([140], [6000], 4), ([1, 2], [5000, 4800], 40)])
def test_scales_of_any_nan_come_first_and_choose_no_more_than_top(heads, new, length, top):
    """A summary's scale that is a NaN of either sign and any payload, quiet or not: the largest score, ties to the lower block, and the list ends where it ends."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(heads + sum(new))
    b = Batch(rng, new, length, 16)
    k, v, q, q32 = make(rng, b, heads, 1, 64, "bf16", "bf16")
    codes, scale = summaries(b, k32_of(k), 1, 64)
    bits = scale.view(np.uint32)
    for s in range(b.S):
        for i, blk in enumerate(range(3, 3 + 2 * 9, 2)):
            bits[b.pages[s][blk], 0] = [0x7FC00000, 0xFFC00000, 0x7FFFFFFF, 0xFFFFFFFF, 0x7F800001, 0xFF800001, 0x7FFFFFFE, 0xFFFFFFFE, 0x7FA00000][i]
    p = C.SparseParams(C.AttendParams(b.params(1, 64, "bf16", "bf16"), heads, max(length), 0.1), top, 1, 1)
    room = torch.full((b.T * top + 512,), 77, dtype=torch.int32, device="cuda")
    blocks = room[256:256 + b.T * top].view(b.T, 1, top)
    _, _, got = C.sparse_attend(p, q.cuda(), *b.device(), upload(k, v), (torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda()), blocks_out=blocks)
    want = wanted_blocks(b, codes, scale, q32, heads, 1, top, 1, 1, False, max(length))
    np.testing.assert_array_equal(got.cpu().numpy()[:sum(new)], want[:sum(new)])
    assert bool((room[:256] == 77).all()) and bool((room[256 + b.T * top:] == 77).all())
    assert set(want[0, 0]) >= {0, *range(3, 3 + 2 * min(9, top - 2), 2)}


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("D,heads,H,page,top,tree", [(128, 8, 4, 16, 9, False), (128, 8, 8, 32, 5, True), (96, 10, 5, 16, 6, False), (64, 16, 4, 16, 7, True), (128, 51, 3, 64, 3, False)])
def test_many_rows(dtype, kept, D, heads, H, page, top, tree):
    """More items than workgroups of eight waves are for: chunks of many rows beside single tokens and padding, positions that do not exist."""
    rng = np.random.default_rng(D + heads + top)
    new = [33, 1, 0, 13, 2]
    b = Batch(rng, new, [333, 400, 20, 13, 1], page)
    b.pages[0, 2], b.pages[1, 0] = -1, b.n_pages
    bits = rng.integers(-2 ** 63, 2 ** 63, b.T, dtype=np.int64) if tree else None
    run(b, heads, H, D, dtype, kept, top, seed=top, visible=bits)


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("D,H,new,length", [(64, 2, [1, 0, 5, 130], [129, 7, 4, 300]), (96, 3, [1], [128]), (128, 9, [1] * 40, [131 * s % 300 + 1 for s in range(40)])])
def test_summaries_of_pages_of_128(dtype, kept, D, H, new, length):
    """By workgroups where they are few, by waves beyond."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(D)
    b = Batch(rng, new, length, 128)
    k, v, _, _ = make(rng, b, H, H, D, dtype, kept)
    cache = b.params(H, D, dtype, kept)
    summary = C.block_alloc(cache)
    summary[0].fill_(7)
    summary[1].fill_(1e30)
    C.block_summary(cache, *b.device(), upload(k, v), summary)
    codes, scale = summaries(b, k32_of(k), H, D)
    touched = {int(b.pages[s][x // 128]) for s in range(b.S) for x in range(max(length[s] - new[s], 0), length[s])}
    for page in range(b.n_pages):
        if page not in touched:
            codes[page], scale[page] = 7, 1e30
    np.testing.assert_array_equal(summary[0].cpu().numpy(), codes)
    np.testing.assert_array_equal(summary[1].cpu().numpy(), scale)
