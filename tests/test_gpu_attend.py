"""GPU parity of covspec_attend with oracle/round_oracle.py (fp64).

Tolerance of an output, with u = half a step of the 16-bit type relative to the value, A = sum p |v| / sum p of the oracle and S = the largest
sum |q k| scale of the row:
  u |o|           the output's own rounding
  u A             p is rounded to 16 bits for its product with v, by at most u each;
  u A             in 8 bits: v = code * scale may be rounded to 16 bits as well
  e A, e = 2 (D + 64) 2^-24 S + 2^-19
                  scores off by the fp32 sums (a rounding per term, of the running sum) move every p by that much, numerator and denominator;
                  fp32 exponentials (argument up to 2^7, half a step 2^-18 of its fraction at worst for the smallest p only; the
                  large ones have arguments near 0), sums over the positions and the joining of pieces: 2^-19
  t V             fp16: p below 2^-14 has fixed steps of 2^-24, off by half a step, over a sum of at least one: 2^-25 sum |v|
  2^-25           the same for the output itself
The log-sum: 2 (D + 64) 2^-24 S + 2^-20 (1 + |lse|).
"""
import math

import numpy as np
import pytest

from oracle import round_oracle as RO
from round_util import HALF_STEP, Batch, pool_of, rounded, torch_dtype

pytestmark = pytest.mark.gpu


def setup(rng, b, heads, H, D, dtype, kept, spread=1.0):
    x = rng.standard_normal((b.n_pages, H, b.page, D)) + 0.5 * rng.standard_normal((1, H, 1, D))
    x[..., 3::29] *= 4.0
    v = rng.standard_normal((b.n_pages, H, b.page, D)) * np.exp(0.5 * rng.standard_normal((b.n_pages, H, b.page, 1)))
    q, q64 = rounded(rng.standard_normal((b.T, heads, D)) * spread, dtype)
    return pool_of(x, kept, dtype), pool_of(v, kept, dtype), q, q64.astype(np.float64)


def upload(k, v):
    return tuple(None if t is None else t.cuda() for t in (k[0], v[0], k[1], v[1]))


def check(b, heads, H, D, dtype, kept, k64, v64, q64, out, lse, scale, window=0, visible=None, max_len=None, rows=None, pad_value=None):
    G, u = heads // H, HALF_STEP[dtype]
    out, lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    for s in range(b.S):
        n, length = b.new[s], b.length[s]
        for i in range(n):
            t = int(b.start[s]) + i
            if rows is not None and t not in rows:
                continue
            seen = RO.seen_by(i, n, length, window, None if visible is None else int(visible[t]) & ((1 << 64) - 1), max_len)
            at = [p for p in (RO.place(j, b.pages[s], b.page, b.n_pages) for j in seen) if p is not None]
            pg, of = np.array([p[0] for p in at], dtype=int), np.array([p[1] for p in at], dtype=int)
            for h in range(heads):
                K, V = k64[pg, h // G, of], v64[pg, h // G, of]
                o, e, A, size = RO.attend_row(q64[t, h], K.reshape(-1, D), V.reshape(-1, D), scale)
                rel = 2 * (D + 64) * 2.0 ** -24 * size
                tol = u * np.abs(o) + (u * (2 if kept != dtype else 1) + rel + 2.0 ** -19) * A + 2.0 ** -25
                if dtype == "fp16" and len(at):
                    tol = tol + 2.0 ** -25 * np.abs(V).reshape(-1, D).sum(0)
                where = "sequence %d row %d head %d (%d seen)" % (s, i, h, len(at))
                err = np.abs(out[t, h] - o) - tol
                assert np.all(err <= 0), "%s: off by %g beyond the tolerance" % (where, err.max())
                if len(at) == 0:
                    assert lse[t, h] == -math.inf and not out[t, h].any(), where
                else:
                    assert abs(lse[t, h] - e) <= rel + 2.0 ** -20 * (1 + abs(e)), where
    if pad_value is not None:
        assert np.all(out[int(b.start[-1]):] == pad_value)


def run(b, heads, H, D, dtype, kept, seed=0, window=0, visible=None, max_len=None, rows=None, spread=1.0):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(seed)
    k, v, q, q64 = setup(rng, b, heads, H, D, dtype, kept, spread)
    p = C.AttendParams(cache=b.params(H, D, dtype, kept), n_heads=heads, max_len=max_len or max(max(b.length), 1), window=window, scale=D ** -0.5)
    out = torch.full((b.T, heads, D), 7.0, dtype=torch_dtype(dtype), device="cuda")
    vis = None if visible is None else torch.from_numpy(np.asarray(visible, dtype=np.int64)).cuda()
    out, lse = C.attend(p, q.cuda(), *b.device(), upload(k, v), visible=vis, out=out, want_lse=True)
    torch.cuda.synchronize()
    check(b, heads, H, D, dtype, kept, k[2], v[2], q64, out, lse, D ** -0.5, window, visible, max_len, rows, pad_value=7.0)


KINDS = [("bf16", "bf16"), ("bf16", "int8"), ("bf16", "e4m3"), ("fp16", "fp16"), ("fp16", "int8"), ("fp16", "e4m3")]


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("D,page", [(64, 16), (96, 32), (128, 64), (128, 16)])
def test_single_tokens(dtype, kept, D, page):
    rng = np.random.default_rng(1)
    run(Batch(rng, [1] * 6, [1, 2, 63, 64, 65, 700], page, pad=2), 8, 2, D, dtype, kept)


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("heads,H,D,page", [(6, 6, 64, 64), (16, 2, 128, 64), (5, 1, 96, 16), (12, 4, 128, 256)])
def test_drafted_segments(dtype, kept, heads, H, D, page):
    rng = np.random.default_rng(2)
    run(Batch(rng, [8, 5, 0, 1, 9, 3], [300, 5, 40, 129, 64, 1000], page, pad=1), heads, H, D, dtype, kept)


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("heads,H,D,page", [(4, 2, 64, 32), (8, 1, 128, 64), (3, 3, 96, 16)])
def test_prompts_and_chunks(dtype, kept, heads, H, D, page):
    rng = np.random.default_rng(3)
    b = Batch(rng, [190, 1, 130, 333], [190, 500, 400, 333], page, pad=5)
    rows = set(range(0, b.T, 7)) | {0, 189, 190, 191, 320, 321, b.T - 6}
    run(b, heads, H, D, dtype, kept, rows=rows)


@pytest.mark.parametrize("window", [1, 17, 64, 100])
@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
def test_sliding_windows(window, kept):
    rng = np.random.default_rng(4)
    b = Batch(rng, [1, 8, 150, 1], [400, 300, 260, 3], 16)
    run(b, 8, 2, 64, "bf16", kept, window=window, rows=set(range(0, b.T, 5)) | {0, 1, 2, 8, 9, b.T - 1})


@pytest.mark.parametrize("kept", ["fp16", "int8"])
def test_trees_of_drafted_tokens(kept):
    rng = np.random.default_rng(5)
    b = Batch(rng, [11, 1, 64, 70, 4], [200, 33, 64, 90, 300], 32)
    vis = []
    for n in b.new:
        seen = []
        for i in range(n):
            seen.append((seen[int(rng.integers(0, i))] if i else 0) | (1 << i if i < 64 else 0))
        vis += seen
    vis[3] = 0                                          # a row that sees only what is in front of the chunk
    a = int(b.start[2])
    vis[a + 5] = 0                                      # and one that sees nothing: its chunk is the whole sequence
    vis[a + 6] = (1 << 64) - 1                          # later rows too
    vis = np.array([x - (1 << 64) if x >> 63 else x for x in vis], dtype=np.int64)
    run(b, 8, 2, 128, "fp16", kept, visible=vis)


@pytest.mark.parametrize("dtype,kept", [("bf16", "bf16"), ("fp16", "int8")])
def test_rows_that_see_nothing_and_positions_that_do_not_exist(dtype, kept):
    rng = np.random.default_rng(6)
    b = Batch(rng, [6, 2, 1, 5, 40], [3, 0, 0, 200, 500], 16)       # the first rows are in front of their sequences
    b.pages[3, 2] = -1                                              # a page inside, the first and the last one missing
    b.pages[3, 7] = b.n_pages
    b.pages[4, 0] = 1 << 30
    b.pages[4, 31] = -(1 << 31)
    run(b, 4, 2, 64, dtype, kept)
    b = Batch(rng, [3], [40], 16)
    b.pages[0, :] = -1
    run(b, 4, 2, 64, dtype, kept)
    b = Batch(rng, [3, 3], [100, 40], 16)
    run(b, 4, 2, 64, dtype, kept, max_len=50)                       # positions at or beyond the bound are not seen
    b = Batch(rng, [3], [64], 16)
    b.length[0] = 16 * b.width + 2                                  # longer than the table
    run(b, 4, 2, 64, dtype, kept, max_len=64)


@pytest.mark.parametrize("dtype,kept", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "int8"), ("fp16", "e4m3")])
@pytest.mark.parametrize("new,length,window", [(1, 200, 0), (8, 150, 0), (150, 300, 0), (150, 300, 40), (8, 333, 20)])
def test_what_is_not_seen_has_no_effect(dtype, kept, new, length, window):
    """NaN and infinities behind the sequence, in its last row's own token, in front of the window and in pages of nobody: the other rows'
    results stay within the tolerance of what they are without them."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(7)
    H, heads, D = 2, 8, 64
    b = Batch(rng, [new], [length], 16)
    k, v, q, q64 = setup(rng, b, heads, H, D, dtype, kept)
    p = C.AttendParams(cache=b.params(H, D, dtype, kept), n_heads=heads, max_len=length, window=window, scale=D ** -0.5)
    mine = set(int(x) for x in b.pages[0, :-(-length // 16)])
    poison = [pg for pg in range(b.n_pages) if pg not in mine]
    pool = list(upload(k, v))

    def spoil(page, place):
        for t in (pool[:2] if kept == dtype else pool[2:]):
            t[page, :, place] = float("nan")
        if kept == dtype:
            pool[1][page, :, place, ::2] = float("inf")

    for pg in poison:
        spoil(pg, slice(None))
    last = RO.place(length - 1, b.pages[0], 16, b.n_pages)
    if last[1] < 15:
        spoil(last[0], slice(last[1] + 1, 16))
    gone = set()
    if new > 1:
        spoil(*last)                                    # the last row's own token: only that row sees it
        gone.add(new - 1)
    if window:
        for j in range(0, length - new - window + 1):   # in front of every row's window
            spoil(*RO.place(j, b.pages[0], 16, b.n_pages))
    out, lse = C.attend(p, q.cuda(), *b.device(), tuple(pool), want_lse=True)
    torch.cuda.synchronize()
    for i in gone:
        assert torch.isnan(out[i]).all()
    check(b, heads, H, D, dtype, kept, k[2], v[2], q64, out, lse, D ** -0.5, window, rows=set(range(new)) - gone)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_extreme_scores(dtype):
    """Scores of thousands in both directions, one key far above the rest; equal keys; the lowest finite values."""
    rng = np.random.default_rng(8)
    run(Batch(rng, [3, 70], [500, 300], 32), 4, 2, 64, dtype, dtype, spread=200.0)
    import torch
    import paper_2605_02218_amd as C
    b = Batch(rng, [2], [130], 16)
    k, v, q, q64 = setup(rng, b, 2, 1, 64, dtype, dtype)
    low = torch.finfo(torch_dtype(dtype)).min
    kk = torch.zeros_like(k[0])
    kk[..., 0] = low                                    # every score is the same large number below zero
    q = torch.zeros_like(q)
    q[..., 0] = 1.0
    p = C.AttendParams(cache=b.params(1, 64, dtype, dtype), n_heads=2, max_len=130, scale=1.0)
    out, lse = C.attend(p, q.cuda(), *b.device(), (kk.cuda(), v[0].cuda(), None, None), want_lse=True)
    torch.cuda.synchronize()
    check(b, 2, 1, 64, dtype, dtype, kk.double().numpy(), v[2], q.double().numpy(), out, lse, 1.0)


def test_long_sequences_and_far_pages():
    """A sequence over many pieces of the split, in a pool whose offsets pass 32 bits."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(9)
    length, page, D, heads, H = 70001, 1024, 128, 4, 1
    b = Batch(rng, [3, 1], [length, 1500], page)
    b.n_pages = 18000                                   # 256 KB a page: 4.7 GB in each pool
    need = [69, 2]
    far = rng.permutation(np.concatenate([np.arange(17950, 18000), np.arange(16350, 16400)]))[:71]
    b.pages[0, :69], b.pages[1, :2] = far[:69], far[69:]
    pool = [torch.empty(b.n_pages, H, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(1)
    used = sorted(int(x) for x in far)
    host = [np.zeros((b.n_pages, 0)) for _ in range(2)]
    small = [np.zeros((len(used), H, page, D)) for _ in range(2)]
    for i in range(2):
        for n, pg in enumerate(used):
            pool[i][pg] = torch.randn(H, page, D, generator=g, device="cuda").to(torch.bfloat16)
            small[i][n] = pool[i][pg].double().cpu().numpy()
    del host, need
    q, q64 = rounded(rng.standard_normal((b.T, heads, D)), "bf16")
    p = C.AttendParams(cache=b.params(H, D, "bf16", "bf16"), n_heads=heads, max_len=length, scale=D ** -0.5)
    out, lse = C.attend(p, q.cuda(), *b.device(), (pool[0], pool[1], None, None), want_lse=True)
    torch.cuda.synchronize()
    index = {pg: n for n, pg in enumerate(used)}
    b.pages = np.array([[index.get(int(x), 0) for x in row] for row in b.pages])
    b.n_pages = len(used)
    check(b, heads, H, D, "bf16", "bf16", small[0], small[1], q64.astype(np.float64), out, lse, D ** -0.5)


def test_rows_of_wider_tensors():
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(10)
    for new in ([3, 2], [150, 40]):
        b = Batch(rng, new, [50, 230], 16)
        k, v, q, q64 = setup(rng, b, 4, 2, 64, "bf16", "bf16")
        wide = torch.zeros(b.T, 7, 64, dtype=torch.bfloat16, device="cuda")
        wide[:, 2:6] = q.cuda()
        out = torch.full((b.T, 5, 64), 3.0, dtype=torch.bfloat16, device="cuda")
        p = C.AttendParams(cache=b.params(2, 64, "bf16", "bf16"), n_heads=4, max_len=230, scale=0.125)
        got, lse = C.attend(p, wide[:, 2:6], *b.device(), upload(k, v), out=out[:, 1:], want_lse=True)
        torch.cuda.synchronize()
        assert bool((out[:, 0] == 3.0).all())
        check(b, 4, 2, 64, "bf16", "bf16", k[2], v[2], q64, got, lse, 0.125)


def test_the_same_call_gives_the_same_bits_on_any_stream():
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(11)
    b = Batch(rng, [8] * 5 + [200], [900, 4000, 333, 64, 2111, 1000], 64)
    k, v, q, _ = setup(rng, b, 16, 4, 128, "bf16", "e4m3")
    p = C.AttendParams(cache=b.params(4, 128, "bf16", "e4m3"), n_heads=16, max_len=4000, scale=0.09)
    args = (q.cuda(), *b.device(), upload(k, v))
    one, lse = C.attend(p, *args, want_lse=True)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    ws = [torch.empty(C.attend_workspace_size(p) + 256, dtype=torch.uint8, device="cuda").fill_(0xFF) for _ in streams]
    torch.cuda.synchronize()
    got = []
    for st, w in zip(streams, ws):                      # three calls at once, each with its own workspace
        with torch.cuda.stream(st):
            got.append(C.attend(p, *args, workspace=w, want_lse=True))
    torch.cuda.synchronize()
    for o, l in got:
        assert torch.equal(o, one) and torch.equal(l, lse)


def test_a_captured_call_serves_other_lengths_and_pages():
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(12)
    first = Batch(rng, [8, 8, 8], [700, 64, 1900], 32, spare=80)
    heads, H, D = 8, 2, 64
    k, v, q, q64 = setup(rng, first, heads, H, D, "bf16", "int8")
    p = C.AttendParams(cache=first.params(H, D, "bf16", "int8"), n_heads=heads, max_len=first.width * 32, scale=0.125)
    batch, pool, qd = first.device(), upload(k, v), q.cuda()
    out, lse = torch.zeros(first.T, heads, D, dtype=torch.bfloat16, device="cuda"), None
    ws = torch.empty(C.attend_workspace_size(p) + 256, dtype=torch.uint8, device="cuda")
    C.attend(p, qd, *batch, pool, workspace=ws, out=out, want_lse=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            _, lse = C.attend(p, qd, *batch, pool, workspace=ws, out=out, want_lse=True)
    for new, lengths in (([8, 8, 8], [700, 64, 1900]), ([8, 8, 8], [9, 1500, 800]), ([1, 0, 20], [1, 5, 1920]), ([24, 0, 0], [1024, 0, 0])):
        b = first
        b.new, b.length = new, lengths
        b.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        b.pages = np.stack([rng.permutation(b.n_pages)[:b.width] for _ in new]).astype(np.int32)
        for dst, src in zip(batch, b.device()):
            dst.copy_(src)
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        check(b, heads, H, D, "bf16", "int8", k[2], v[2], q64, got, lse, 0.125, pad_value=7.0)
        C.attend(p, qd, *batch, pool, workspace=ws, out=out)
        torch.cuda.synchronize()
        assert torch.equal(got, out)


def test_many_short_sequences():
    rng = np.random.default_rng(13)
    new = [int(x) for x in rng.integers(0, 4, 300)]
    b = Batch(rng, new, [n + int(rng.integers(0, 60)) for n in new], 16, pad=9)
    run(b, 2, 1, 64, "bf16", "bf16")


@pytest.mark.parametrize("dtype,kept,new,heads,H", [("bf16", "e4m3", 1, 8, 4), ("bf16", "bf16", 1, 8, 4), ("fp16", "int8", 9, 16, 4), ("bf16", "bf16", 9, 32, 4)])
def test_more_items_than_the_device_holds(dtype, kept, new, heads, H):
    """A workgroup for each item, no shares: 150 sequences x 4 key heads, more of them than lanes."""
    rng = np.random.default_rng(14)
    b = Batch(rng, [new] * 150, [new + int(x) for x in rng.integers(0, 400, 150)], 16, pad=1)
    run(b, heads, H, 64, dtype, kept, rows=set(range(0, b.T, 37)) | {0, b.T - 2})


@pytest.mark.parametrize("dtype,kept,new", [("bf16", "bf16", 1), ("fp16", "e4m3", 5)])
def test_shares_over_more_sequences_than_lanes(dtype, kept, new):
    rng = np.random.default_rng(15)
    b = Batch(rng, [new] * 120, [new + int(x) for x in rng.integers(0, 900, 120)], 16, pad=1)
    run(b, 2, 1, 64, dtype, kept, rows=set(range(0, b.T, 7)) | {0, b.T - 2})


@pytest.mark.parametrize("dtype,kept", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "int8")])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_trees_and_chunks_of_many_rows(dtype, kept, D):
    """512 rows and more: the waves of 16-bit caches take turns."""
    rng = np.random.default_rng(16)
    b = Batch(rng, [64, 70], [300, 90], 32, pad=1)
    vis = [int(x) - (1 << 63) for x in rng.integers(0, 1 << 62, b.T)]
    run(b, 16, 2, D, dtype, kept, visible=np.array(vis, dtype=np.int64), rows=set(range(0, b.T, 9)) | {63, 64, 133})
    b = Batch(rng, [129, 1, 300], [129, 400, 777], 16)
    run(b, 8, 1, D, dtype, kept, rows=set(range(0, b.T, 41)) | {0, 128, 129, 130, 429})


@pytest.mark.parametrize("scale", [-0.2, 0.0, 1e-30, 3.0])
@pytest.mark.parametrize("dtype,kept,new", [("bf16", "bf16", [1, 3]), ("fp16", "int8", [3, 1]), ("bf16", "e4m3", [150, 8]), ("fp16", "fp16", [200, 9])])
def test_scales_of_any_sign(scale, dtype, kept, new):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(17)
    b = Batch(rng, new, [333, 210], 16)
    k, v, q, q64 = setup(rng, b, 8, 2, 64, dtype, kept)
    p = C.AttendParams(cache=b.params(2, 64, dtype, kept), n_heads=8, max_len=333, scale=scale)
    out, lse = C.attend(p, q.cuda(), *b.device(), upload(k, v), want_lse=True)
    torch.cuda.synchronize()
    check(b, 8, 2, 64, dtype, kept, k[2], v[2], q64, out, lse, float(np.float32(scale)), rows=set(range(0, b.T, 11)) | {0, b.T - 1})


def test_a_batch_of_padding_only():
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(18)
    b = Batch(rng, [0, 0, 0], [5, 0, 70], 16, pad=6)
    run(b, 4, 2, 64, "bf16", "bf16")
    k, v, q, _ = setup(rng, b, 4, 2, 64, "bf16", "int8")
    pool = upload(k, v)
    before = [t.clone() for t in pool]
    x = torch.randn(b.T, 2, 64, device="cuda").to(torch.bfloat16)
    C.cache_write(b.params(2, 64, "bf16", "int8"), x, x, *b.device(), pool)
    torch.cuda.synchronize()
    for t, u in zip(pool, before):
        assert torch.equal(t, u)


@pytest.mark.parametrize("dtype,kept,heads", [("bf16", "bf16", 4), ("fp16", "e4m3", 64), ("bf16", "int8", 16)])
def test_arrays_that_describe_nothing_sensible_touch_nothing_else(dtype, kept, heads):
    """Rows that do not ascend, lengths and pages out of range: results are what they are, memory around the outputs stays as it was.  (Every index
    formed from these arrays is checked by the kernels.)"""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(19)
    H, D = 2, 64
    b = Batch(rng, [8, 8, 8], [90, 40, 64], 16)
    k, v, q, _ = setup(rng, b, heads, H, D, dtype, kept)
    pool = upload(k, v)
    p = C.AttendParams(cache=b.params(H, D, dtype, kept), n_heads=heads, max_len=b.width * 16, scale=0.1)
    room = torch.full((b.T + 2, heads, D), 7.0, dtype=torch_dtype(dtype), device="cuda")
    ws = torch.empty(C.attend_workspace_size(p) + 256, dtype=torch.uint8, device="cuda")
    x = torch.zeros(b.T, H, D, dtype=torch_dtype(dtype), device="cuda")
    for start, length in (([5, 0, 24, 3], [90, 40, 64]), ([-9, 400, -1, 7], [1 << 30, -5, 77]), ([24, 24, 0, 24], [-(1 << 31), (1 << 31) - 1, 0]), ([0, 24, 24, 0], [3, 0, 9])):
        ws.fill_(0x7F)
        dev = [torch.tensor(a, dtype=torch.int32, device="cuda") for a in (start, length)]
        pages = torch.from_numpy(rng.integers(-3, b.n_pages + 3, b.pages.shape).astype(np.int32)).cuda()
        C.attend(p, q.cuda(), *dev, pages, pool, workspace=ws, out=room[1:-1])
        C.cache_read(p.cache, pool, *dev, pages)
        C.cache_write(p.cache, x, x, *dev, pages, pool)
        torch.cuda.synchronize()
        assert bool((room[0] == 7.0).all()) and bool((room[-1] == 7.0).all())
