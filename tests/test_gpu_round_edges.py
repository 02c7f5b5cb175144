"""Edges of the entry points around a verification round that the tests of each of them leave out: calls that the documentation allows or refuses."""
import ctypes

import numpy as np
import pytest

import test_gpu_attend as TA
import test_round_tolerances as TT
from oracle import round_oracle as RO
from round_util import HALF_STEP, Batch, pool_of, rounded, torch_dtype

pytestmark = pytest.mark.gpu


def test_expanded_tensors_are_refused_before_anything_is_launched():
    import torch
    import paper_2605_02218_amd as C
    b = Batch(np.random.default_rng(1), [6, 3], [40, 30], 16)
    H, heads, D = 2, 4, 64
    p = b.params(H, D, "bf16", "bf16")
    pool, batch = C.cache_alloc(p), b.device()
    rows = lambda n: torch.zeros(b.T, n, D, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    one = lambda n: torch.zeros(1, n, D, dtype=torch.bfloat16, device="cuda").expand(b.T, n, D)  # noqa: E731
    a = C.AttendParams(cache=p, n_heads=heads, max_len=40, scale=0.1)
    for call in (lambda: C.cache_write(p, one(H), one(H), *batch, pool), lambda: C.cache_write(p, rows(H), one(H), *batch, pool),
                 lambda: C.cache_read(p, pool, *batch, k_out=one(H), v_out=one(H)), lambda: C.cache_read(p, pool, *batch, v_out=one(H)),
                 lambda: C.attend(a, one(heads), *batch, pool), lambda: C.attend(a, rows(heads), *batch, pool, out=one(heads))):
        with pytest.raises(ValueError, match="overlap"):
            call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_adjustments_without_an_effect_keep_every_number(dtype):
    """(1, 0, 0, 1) for all 16-bit patterns, or those of fp32 with the same upper halves: zeros of both signs, subnormals, infinities."""
    import torch
    import paper_2605_02218_amd as C
    bits = np.arange(1 << 16, dtype=np.uint32)
    if dtype == "fp32":
        z = torch.from_numpy((bits << 16 | bits * 40503 & 0xFFFF).astype(np.uint32).view(np.int32)).view(torch.float32)
        z[0], z[1 << 15], z[0x7F80], z[0xFF80] = 0.0, -0.0, float("inf"), -float("inf")
    else:
        z = torch.from_numpy(bits.astype(np.uint16).view(np.int16)).view(torch_dtype(dtype))
    z = z.reshape(2, 4, -1)
    V = z.shape[2]
    starts = torch.tensor([0, V, 2 * V], dtype=torch.int32, device="cuda")
    words = torch.arange(V, dtype=torch.int32, device="cuda").repeat(2)
    pen = torch.tensor([[1.0, 0, 0, 1], [1.0, 0, 0, 0]], device="cuda")
    p = C.LogitsParams(2, 4, V, {"bf16": C.BF16, "fp16": C.FP16, "fp32": C.FP32}[dtype])
    for history, at, kw in ((words[:0], torch.zeros_like(starts), {}), (words, starts, {}),
                            (words, starts, dict(prompt_len=torch.tensor([V, 7], dtype=torch.int32, device="cuda"), drafted=words[:8].reshape(2, 4).contiguous())),
                            (words, starts, dict(allowed=torch.full((2, 4, V // 32), -1, dtype=torch.int32, device="cuda")))):
        out = C.adjust_logits(p, z.cuda(), history, at, pen, **kw).cpu()
        number = ~torch.isnan(z)
        kind = torch.int32 if dtype == "fp32" else torch.int16
        assert torch.equal(out.view(kind)[number], z.view(kind)[number])
        assert bool(torch.isnan(out)[~number].all())


@pytest.mark.parametrize("most", [1 << 20, (1 << 31) - 100, (1 << 31) - 1])
def test_a_prompt_longer_than_the_history_is_all_of_it(most):
    import torch
    import paper_2605_02218_amd as C
    S, L, V = 3, 2, 4096
    z = torch.linspace(-3, 3, S * L * V, device="cuda").reshape(S, L, V)
    words = torch.arange(0, 900, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 300, 600, 900], dtype=torch.int32, device="cuda")
    pen = torch.tensor([[1.5, 0.5, 0.25, 1.0]] * S, device="cuda")
    asked = lambda n: torch.full((S,), n, dtype=torch.int32, device="cuda")  # noqa: E731
    p = C.LogitsParams(S, L, V, C.FP32)
    want = C.adjust_logits(p, z, words, starts, pen, prompt_len=asked(300))
    assert torch.equal(C.adjust_logits(p, z, words, starts, pen, prompt_len=asked(most)), want)
    # and one below zero is none
    assert torch.equal(C.adjust_logits(p, z, words, starts, pen, prompt_len=asked(-most)), C.adjust_logits(p, z, words, starts, pen))


@pytest.mark.parametrize("L", [1, 5, 64])
def test_the_last_drafted_column_has_no_effect(L):
    """The library is given an array that ends in front of its last element."""
    import torch
    import paper_2605_02218_amd as C
    S, V = 2, 2048
    z = torch.linspace(-3, 3, S * L * V, device="cuda").reshape(S, L, V).to(torch.bfloat16)
    none = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    pen = torch.tensor([[1.5, 0.5, 0.25, 1.0]] * S, device="cuda")
    drafted = torch.randint(0, 9, (S, L), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    p = C.LogitsParams(S, L, V)
    want = C.adjust_logits(p, z, none[:0], none, pen, drafted=drafted)
    for other in (0, 5, V - 1, -1, V):
        d = drafted.clone()
        d[:, -1] = other
        assert torch.equal(C.adjust_logits(p, z, none[:0], none, pen, drafted=d), want)
    short, out, cs = drafted.reshape(-1)[:-1].clone(), torch.empty_like(z), p.c_struct()
    st = C.load_library().covspec_adjust_logits(ctypes.byref(cs), z.data_ptr(), none.data_ptr(), none.data_ptr(), None, short.data_ptr(), pen.data_ptr(), None, None,
                                                None, None, out.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == 0 and torch.equal(out, want)


@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [1, 12, 30, 70, 600])
def test_a_query_of_nan_beside_scores_of_the_largest_numbers(new, kept):
    """Scores of 2^127 lie beyond the range of their own base-2 exponents; a row of NaN among them is NaN, the others the mean of v."""
    import torch
    import paper_2605_02218_amd as C
    b = Batch(np.random.default_rng(2), [new], [new + 90], 16)
    p = b.params(1, 64, "bf16", kept)
    k = torch.zeros(b.n_pages, 1, 16, 64)
    k[..., 0] = 2.0 ** (63 if kept == "bf16" else 8)
    scale = None if kept == "bf16" else torch.full(k.shape[:3], 2.0 ** 55, device="cuda")
    v, one = torch.full_like(k, 0.75), None if kept == "bf16" else torch.ones(k.shape[:3], device="cuda")
    q = torch.zeros(new, 2, 64, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 2.0 ** 64
    q[0, 0, 5] = float("nan")
    t = torch_dtype(kept)
    out, lse = C.attend(C.AttendParams(cache=p, n_heads=2, max_len=new + 90, scale=1.0), q, *b.device(), (k.to(t).cuda(), v.to(t).cuda(), scale, one), want_lse=True)
    assert bool(torch.isnan(out[0, 0]).all()) and bool(torch.isnan(lse[0, 0]))
    rest = torch.ones(new, 2, dtype=torch.bool, device="cuda")
    rest[0, 0] = False
    assert bool((out[rest] == 0.75).all()) and bool((lse[rest] == 2.0 ** 127).all())


@pytest.mark.parametrize("dtype,kept", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "e4m3"), ("bf16", "int8"), ("fp16", "int8")])
@pytest.mark.parametrize("D,new,window,tree", [(64, 1, 0, False), (128, 2, 60, False), (96, 6, 0, True), (128, 12, 0, False), (128, 30, 0, True), (96, 60, 33, False),
                                               (64, 160, 0, False), (96, 300, 0, False), (128, 300, 100, False), (64, 290, 0, True)])
def test_numbers_that_are_not_finite_reach_the_rows_that_see_them(dtype, kept, D, new, window, tree):
    """Infinities and NaN in v, some seen by all rows, some by a few, some by none, one on a page that does not exist for the sequence: of a row, the columns
    without any keep the tolerance of finite sums (tests of the attention itself), the others are what the formula gives.  Scores are within +-4 of each
    other, so that no p vanishes."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(D + new)
    H, heads, old = 2, 4, 150
    length = old + new
    b = Batch(rng, [new], [length], 16)
    k = pool_of(rng.standard_normal((b.n_pages, H, 16, D)), kept, dtype)
    v = pool_of(rng.standard_normal((b.n_pages, H, 16, D)) + 0.5, kept, dtype)
    q, q64 = rounded(0.3 * rng.standard_normal((new, heads, D)), dtype)
    b.pages[0, 4] = -1                                  # positions 64 .. 79; the first page of the pool is loaded in its place
    spoilt = [(j, float(x)) for j, x in ((3, np.inf), (70, np.nan), (old - 2, -np.inf), (old, np.nan), (length - 1, np.inf), (length - 1 - new // 2, np.inf))]
    codes, v64 = v[0].clone(), v[2].copy()
    for i, (j, x) in enumerate(spoilt):
        page, at = RO.place(j, b.pages[0], 16, b.n_pages) or (0, 5)
        cols = slice(5 * i % D, 5 * i % D + 3)
        if kept == dtype:
            codes[page, :, at, cols], v64[page, :, at, cols] = x, x
        elif kept == "e4m3" and i < 2:
            codes[page, :, at, cols], v64[page, :, at, cols] = float("nan"), np.nan       # a code that is none
        else:
            v[1][page, :, at], v64[page, :, at] = float("nan"), np.nan                    # as an infinity is written in 8 bits
    bits = None
    if tree:
        bits = [int(x) for x in rng.integers(-(1 << 63), 1 << 63, new, dtype=np.int64)]
        bits[0] = 0
    p = C.AttendParams(cache=b.params(H, D, dtype, kept), n_heads=heads, max_len=length, window=window, scale=D ** -0.5)
    pool = tuple(None if t is None else t.cuda() for t in (k[0], codes, k[1], v[1]))
    vis = None if bits is None else torch.tensor(bits, dtype=torch.int64, device="cuda")
    out, lse = C.attend(p, q.cuda(), *b.device(), pool, visible=vis, want_lse=True)
    out, lse, u = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy(), HALF_STEP[dtype]
    for i in list(range(0, new, 17)) + [new - 1, new // 2, max(new - 2, 0)]:
        seen = RO.seen_by(i, new, length, window, None if bits is None else bits[i] & ((1 << 64) - 1))
        at = [x for x in (RO.place(j, b.pages[0], 16, b.n_pages) for j in seen) if x is not None]
        pg, of = np.array([x[0] for x in at], dtype=int), np.array([x[1] for x in at], dtype=int)
        for h in range(heads):
            K, V = k[2][pg, h // 2, of], v64[pg, h // 2, of]
            z = K @ q64[i, h].astype(np.float64) * D ** -0.5
            w = np.exp(z - z.max())
            terms = w[:, None] * V / w.sum()
            with np.errstate(invalid="ignore"):
                want, A = terms.sum(0), np.abs(terms).sum(0)
            fine = np.isfinite(want)
            size = float((np.abs(K) @ np.abs(q64[i, h])).max()) * D ** -0.5
            rel = 2 * (D + 64) * 2.0 ** -24 * size
            tol = u * np.abs(want) + (2 * u + rel + 2.0 ** -19) * A + 2.0 ** -25 * (1 + np.abs(np.where(np.isfinite(V), V, 0.0)).sum(0))
            assert np.all(np.abs(out[i, h][fine] - want[fine]) <= tol[fine]), (i, h)
            np.testing.assert_array_equal(out[i, h][~fine], want[~fine], err_msg="row %d head %d" % (i, h))
            e = z.max() + np.log(w.sum())
            assert abs(lse[i, h] - e) <= rel + 2.0 ** -20 * (1 + abs(e))


KINDS = [("bf16", "bf16"), ("bf16", "int8"), ("bf16", "e4m3"), ("fp16", "fp16"), ("fp16", "int8"), ("fp16", "e4m3")]


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("new,H,window", [([8, 8, 8, 8], 2, 0), ([8] * 3 + [3, 0], 3, 90), ([8] * 150, 1, 0)])
def test_segments_of_17_to_32_rows(dtype, kept, D, new, H, window):
    """Eight tokens of four heads for each key head: a tile of 32 rows for each sequence, by shares and, with 150 of them, by items."""
    rng = np.random.default_rng(20)
    b = Batch(rng, new, [n + int(x) for n, x in zip(new, rng.integers(0, 700 if len(new) < 9 else 200, len(new)))], 32, pad=1)
    TA.run(b, 4 * H, H, D, dtype, kept, window=window, rows=set(range(0, b.T, 1 if len(new) < 9 else 61)) | {0, b.T - 2})


@pytest.mark.parametrize("dtype,kept", KINDS)
def test_two_rows_for_one_place(dtype, kept):
    """Sequences that share their pages: what they write alike is there, where they differ every element is one's or the other's, other places are untouched."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(21)
    S, n, H, D = 40, 24, 3, 96
    b = Batch(rng, [n] * S, [n] * S, 16, spare=2)
    b.pages[1::2] = b.pages[::2]                         # neighbours in pairs
    x = [rounded(rng.standard_normal((S // 2, 2, n, H, D)), dtype) for _ in range(2)]
    for t, f in x:
        t[:, 1, :16], f[:, 1, :16] = t[:, 0, :16], f[:, 0, :16]
    p = b.params(H, D, dtype, kept)
    pool = C.cache_alloc(p)
    for t in pool:
        if t is not None:
            t.view(torch.uint8).fill_(0x5A)
    before = [None if t is None else t.cpu().clone() for t in pool]
    C.cache_write(p, x[0][0].reshape(-1, H, D).cuda(), x[1][0].reshape(-1, H, D).cuda(), *b.device(), pool)
    torch.cuda.synchronize()
    for i in range(2):
        got = pool[i].cpu().float().numpy()
        scale = None if pool[2 + i] is None else pool[2 + i].cpu().numpy()
        used = np.zeros((b.n_pages, 16), dtype=bool)
        codes, scales = (x[i][1], None) if kept == dtype else RO.quantise(x[i][1], kept)
        for s in range(S // 2):
            for j in range(n):
                page, at = RO.place(j, b.pages[2 * s], 16, b.n_pages)
                used[page, at] = True
                one, two = codes[s, :, j]
                assert np.all((got[page, :, at] == one) | (got[page, :, at] == two))
                if scale is not None:
                    assert np.all((scale[page, :, at] == scales[s, 0, j]) | (scale[page, :, at] == scales[s, 1, j]))
        for t, u in ((pool[i], before[i]), (pool[2 + i], before[2 + i])):
            if t is not None:
                rest = torch.from_numpy(~used)[:, None, :].expand(t.shape[:3])
                assert torch.equal(t.cpu()[rest].contiguous().view(torch.uint8), u[rest].contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_a_drafted_word_that_is_not_allowed(dtype):
    """With the mask on the target alone it is rejected and an allowed word drawn; with the mask on both sides, which is for words drawn under it, it
    counts as accepted."""
    import torch
    import paper_2605_02218_amd as C
    S, L, V = 4, 3, 2048
    g = torch.Generator(device="cuda").manual_seed(3)
    DT = {"bf16": C.BF16, "fp16": C.FP16, "fp32": C.FP32}[dtype]
    zt = torch.randn(S, L, V, device="cuda", generator=g).to(torch_dtype(dtype))
    zd = zt.clone()                                     # alpha = 1 but for the mask
    drafted = torch.randint(64, V, (S, L), device="cuda", dtype=torch.int32, generator=g)
    drafted[:, 1] = torch.tensor([0, 31, 32, 63], device="cuda", dtype=torch.int32)
    allowed = torch.full((S, L, V // 32), -1, dtype=torch.int32, device="cuda")
    allowed[:, :, :2] = 0                               # words 0 .. 63 are not allowed
    none = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    pen = torch.tensor([[1.0, 0, 0, 1]] * S, device="cuda")
    masked = [C.adjust_logits(C.LogitsParams(S, L, V, DT), z, none[:0], none, pen, allowed=allowed) for z in (zt, zd)]
    ua, ur = torch.full((S, L), 0.5, device="cuda"), torch.rand(S, device="cuda", generator=g)
    vp = C.VerifyParams(S, L, V, DT)
    n, word, alpha = C.verify(vp, masked[0], zd, drafted, ua, ur)
    assert n.tolist() == [1] * S and alpha[:, 1].tolist() == [0.0] * S and bool((alpha[:, [0, 2]] == 1).all()) and bool((word >= 64).all())
    n, word, alpha = C.verify(vp, *masked, drafted, ua, ur)
    assert n.tolist() == [L] * S and bool((alpha == 1).all())


class _Guarded:
    """Tensors inside a larger allocation each, with marked bytes in front of and behind them that have to stay."""

    def __init__(self):
        self.all = []

    def __call__(self, t=None, shape=None, dtype=None):
        import torch
        shape, dtype = (t.shape, t.dtype) if t is not None else (shape, dtype)
        n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        room = torch.full((n + 2 * 4096 + 256,), 0x5A, dtype=torch.uint8, device="cuda")
        inside = room[4096:4096 + n].view(dtype).reshape(shape)
        if t is not None:
            inside.copy_(t)
        self.all.append((room, n))
        return inside

    def check(self):
        import torch
        torch.cuda.synchronize()
        for room, n in self.all:
            assert bool((room[:4096] == 0x5A).all()) and bool((room[4096 + n:] == 0x5A).all())


@pytest.mark.parametrize("dtype,kept,heads,new", [("bf16", "bf16", 4, 8), ("fp16", "e4m3", 64, 8), ("bf16", "int8", 16, 1), ("fp16", "fp16", 8, 300), ("bf16", "e4m3", 8, 90),
                                                  ("bf16", "bf16", 16, 4)])
def test_arrays_that_describe_nothing_sensible_write_nowhere_else(dtype, kept, heads, new):
    """Starts that do not ascend, lengths and pages out of range (every index formed from them is checked by the kernels): marked bytes around every array that
    a call is given stay, and of the pool only places that the arrays lead to change."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(22)
    H, D, S = 2, 64, 3
    b = Batch(rng, [new] * S, [new + 82, new + 32, new + 56], 16)
    T = S * new
    t = torch_dtype(dtype)
    k, v = (pool_of(rng.standard_normal((b.n_pages, H, 16, D)), kept, dtype) for _ in range(2))
    p = C.AttendParams(cache=b.params(H, D, dtype, kept), n_heads=heads, max_len=b.width * 16, scale=0.1)
    q = rounded(rng.standard_normal((T, heads, D)), dtype)[0]
    x = rounded(rng.standard_normal((T, H, D)), dtype)[0]
    top = (1 << 31) - 1
    for start, length in (([5, 0, T, 3], [90, 40, 64]), ([-9, 400, -1, 7], [1 << 30, -5, 77]), ([T, T, 0, T], [-top - 1, top, 0]), ([0, T, T, 0], [3, 0, 9]),
                          ([top, -top, 0, T], [top, top, top]), ([-top, top, -top, top], [40, -40, 1]), ([0, 0, 0, top], [60, 60, 60])):
        guard = _Guarded()
        pool = tuple(None if y is None else guard(y) for y in (k[0], v[0], k[1], v[1]))
        batch = [guard(torch.tensor(y, dtype=torch.int32)) for y in (start, length)] + [
            guard(torch.from_numpy(rng.integers(-3, b.n_pages + 3, b.pages.shape).astype(np.int32)))]
        need = C.attend_workspace_size(p)
        ws, out, gq, gx = guard(shape=(need,), dtype=torch.uint8), guard(shape=(T, heads, D), dtype=t), guard(q), guard(x)
        outs = [guard(shape=(T, H, D), dtype=t) for _ in range(2)]
        ws.fill_(0x7F)
        assert ws.data_ptr() % 256 == 0
        lse, cs = guard(shape=(T, heads), dtype=torch.float32), p.c_struct()
        at = [None if y is None else y.data_ptr() for y in (gq, *batch, *pool, None, out, lse, ws)]
        assert C.load_library().covspec_attend(ctypes.byref(cs), *at, need, torch.cuda.current_stream().cuda_stream) == 0
        C.cache_read(p.cache, pool, *batch, k_out=outs[0], v_out=outs[1])
        guard.check()
        for given, here in ((q, gq), (x, gx), (k[0], pool[0]), (v[0], pool[1])):
            assert torch.equal(given.view(torch.uint8), here.cpu().view(torch.uint8))
        C.cache_write(p.cache, gx, gx, *batch, pool)
        guard.check()
        # places on pages of the table, of heads as they were: all others keep their bytes
        table = batch[2].cpu().numpy()
        other = np.array([pg for pg in range(b.n_pages) if pg not in table], dtype=int)
        for given, here in ((k[0], pool[0]), (v[0], pool[1])):
            assert torch.equal(given[other].view(torch.uint8), here.cpu()[other].view(torch.uint8))


def test_only_the_places_of_the_rows_change():
    """A round's rows into a pool that is full: every other byte of codes and scales is what it was."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(23)
    for dtype, kept, D in (("bf16", "int8", 128), ("fp16", "e4m3", 96), ("bf16", "bf16", 64)):
        H, guard = 5, _Guarded()
        b = Batch(rng, [9, 0, 3, 17], [70, 12, 3, 300], 32, pad=4)
        k, v = (pool_of(rng.standard_normal((b.n_pages, H, 32, D)), kept, dtype) for _ in range(2))
        pool = tuple(None if y is None else guard(y) for y in (k[0], v[0], k[1], v[1]))
        x = rounded(rng.standard_normal((b.T, H, D)), dtype)[0]
        p = b.params(H, D, dtype, kept)
        C.cache_write(p, x.cuda(), x.cuda(), *b.device(), pool)
        guard.check()
        mine = np.zeros((b.n_pages, 32), dtype=bool)
        for at in b.places():
            if at not in (None, "padding"):
                mine[at] = True
        for given, here in zip((k[0], v[0], k[1], v[1]), pool):
            if given is not None:
                rest = torch.from_numpy(~mine)[:, None, :].expand(given.shape[:3])
                assert torch.equal(given[rest].contiguous().view(torch.uint8), here.cpu()[rest].contiguous().view(torch.uint8))
        outs = [guard(torch.full((b.T, H, D), 7.0, dtype=torch_dtype(dtype))) for _ in range(2)]
        C.cache_read(p, pool, *b.device(), k_out=outs[0], v_out=outs[1])
        guard.check()
        for o in outs:
            assert bool((o[int(b.start[-1]):] == 7.0).all())


@pytest.mark.parametrize("dtype,kept", [k for k in KINDS if k != ("fp16", "fp16")])
@pytest.mark.parametrize("D,new", [(64, 1), (128, 1), (96, 6), (128, 6), (128, 14), (64, 30), (96, 30), (128, 30)])
def test_products_with_v_keep_their_bits(dtype, kept, D, new):
    """Few positions whose scores are exact (small whole numbers), so that the roundings of p (v_scale) show: derived in test_round_tolerances."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(D + new)
    H, heads = 2, 8
    b = Batch(rng, [new] * 3, [new + 1, new + 34, new + 9], 16)
    codes = torch.from_numpy(rng.integers(-4, 5, (b.n_pages, H, 16, D)).astype(np.float32))
    k_scale = torch.full(codes.shape[:3], 2.0 ** -4)
    v = pool_of(rng.standard_normal(codes.shape) * np.exp(0.5 * rng.standard_normal(codes.shape[:3] + (1,))), kept, dtype)
    q = rng.integers(-1, 2, (b.T, heads, D)).astype(np.float64)
    p = C.AttendParams(cache=b.params(H, D, dtype, kept), n_heads=heads, max_len=max(b.length), scale=1.0)
    if kept == dtype:
        pool = ((codes * k_scale[..., None]).to(torch_dtype(kept)).cuda(), v[0].cuda(), None, None)
    else:
        pool = (codes.to(torch_dtype(kept)).cuda(), v[0].cuda(), k_scale.cuda(), v[1].cuda())
    out, _ = C.attend(p, torch.from_numpy(q).to(torch_dtype(dtype)).cuda(), *b.device(), pool)
    out, k64 = out.float().cpu().numpy().astype(np.float64), codes.double().numpy() * 2.0 ** -4
    for s in range(3):
        for i in range(new):
            t = int(b.start[s]) + i
            at = np.array([RO.place(j, b.pages[s], 16, b.n_pages) for j in RO.seen_by(i, new, b.length[s])])
            assert len(at) <= 64
            for h in range(heads):
                o, _, A, _ = RO.attend_row(q[t, h], k64[at[:, 0], h // 4, at[:, 1]], v[2][at[:, 0], h // 4, at[:, 1]], 1.0)
                assert np.all(np.abs(out[t, h] - o) <= TT.allowed(dtype, o, A, TT.parts(dtype, kept, new * heads // H))), (s, i, h)


@pytest.mark.parametrize("dtype,kept", [k for k in KINDS if k[0] != k[1]])
def test_rows_over_the_whole_range_of_their_type(dtype, kept):
    """A row's largest magnitude from the smallest number of the type to its largest, the border of 2^-100 among them: codes and scales to the bit, and what
    is read back."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(24)
    D, top = 64, {"bf16": range(-133, 128), "fp16": range(-24, 16)}[dtype]
    b = Batch(rng, [len(top)], [len(top) + 7], 64)
    x = np.stack([rng.uniform(-1, 1, (1, D)) for _ in top]) * 2.0 ** (np.array(top, dtype=float)[:, None, None] + 1)
    x[:, 0, 3] = (2.0 - 2.0 ** -7) * 2.0 ** np.array(top, dtype=float)             # below 2^(k + 1) in both types
    x[::5, 0, 3] = 2.0 ** np.array(top, dtype=float)[::5]
    x[::5, 0] = np.clip(x[::5, 0], -x[::5, :1, 3], x[::5, :1, 3])
    x = np.clip(x, -np.abs(x[:, :, 3:4]), np.abs(x[:, :, 3:4]))
    t, v32 = rounded(x, dtype)
    assert np.isfinite(v32).all()
    p = b.params(1, D, dtype, kept)
    pool, batch = C.cache_alloc(p), b.device()
    C.cache_write(p, t.cuda(), t.cuda(), *batch, pool)
    k, v = C.cache_read(p, pool, *batch)
    torch.cuda.synchronize()
    at = np.array(b.places())
    codes, scale = RO.quantise(v32, kept)
    for i, back in ((0, k), (1, v)):
        np.testing.assert_array_equal(pool[i].cpu().float().numpy()[at[:, 0], 0, at[:, 1]], codes[:, 0])
        np.testing.assert_array_equal(pool[2 + i].cpu().numpy()[at[:, 0], 0, at[:, 1]], scale[:, 0])
        want = torch.from_numpy(codes * scale[..., None]).to(t.dtype)
        np.testing.assert_array_equal(back.cpu().float().numpy(), want.float().numpy())


@pytest.mark.parametrize("dtype,kept,new,heads", [("bf16", "bf16", 3, 2), ("bf16", "e4m3", 8, 4), ("bf16", "bf16", 12, 8), ("fp16", "e4m3", 12, 8), ("fp16", "fp16", 25, 8),
                                                  ("bf16", "e4m3", 25, 8), ("bf16", "int8", 25, 8)])
def test_many_sequences_whose_last_token_is_not_finite(dtype, kept, new, heads):
    """A workgroup for each item: every other sequence has NaN in its last row's v, which that row alone sees."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(25)
    S, H, D = 300, 1, 64
    b = Batch(rng, [new] * S, [new + int(x) for x in rng.integers(0, 150, S)], 16)
    k, v, q, q64 = TA.setup(rng, b, heads, H, D, dtype, kept)
    pool = TA.upload(k, v)
    last = [int(b.start[s + 1]) - 1 for s in range(0, S, 2)]
    for s in range(0, S, 2):
        page, at = RO.place(b.length[s] - 1, b.pages[s], 16, b.n_pages)
        (pool[1] if kept == dtype else pool[3])[page, :, at] = float("nan")
    p = C.AttendParams(cache=b.params(H, D, dtype, kept), n_heads=heads, max_len=max(b.length), scale=D ** -0.5)
    out, lse = C.attend(p, q.cuda(), *b.device(), pool, want_lse=True)
    torch.cuda.synchronize()
    spoilt = torch.zeros(b.T, dtype=torch.bool)
    spoilt[last] = True
    assert bool(torch.isnan(out[spoilt.cuda()]).all()) and not bool(torch.isnan(out[~spoilt.cuda()]).any()) and not bool(torch.isnan(lse).any())
    rows = (set(range(0, b.T, 53)) | {t - 1 for t in last[::9]}) - set(last)
    TA.check(b, heads, H, D, dtype, kept, k[2], v[2], q64, out, lse, D ** -0.5, rows=rows)
