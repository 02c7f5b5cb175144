"""Verification rounds over long contexts, as a serving program runs them: page tables from the lengths, rotated keys into the cache, summaries, attention over the
pages they select, logits adjusted and verified, and the next lengths from what was accepted, all on the device."""
from types import SimpleNamespace

import numpy as np
import pytest

import test_gpu_sparse as TS
from oracle import round_oracle as RO
from oracle import sparse_oracle as SO
from round_util import HALF_STEP, NAMES, rounded, torch_dtype

pytestmark = pytest.mark.gpu

S, L, V, HEADS, H, D, PAGE, WIDTH, N_PAGES, TOP = 3, 4, 4096, 8, 2, 64, 16, 24, 60, 6


class Round:
    """The buffers of a program that keeps its rounds on the device."""

    def __init__(self, dtype, kept, T):
        import torch
        import paper_2605_02218_amd as C
        self.T, self.dtype = T, dtype
        self.pages_p = C.PagesParams(S, T, PAGE, N_PAGES, WIDTH)
        self.cache_p = C.CacheParams(S, T, H, D, PAGE, N_PAGES, WIDTH, NAMES[dtype], NAMES[kept])
        self.rotary_p = C.RotaryParams(S, T, HEADS, H, D, 32, True, dtype=NAMES[dtype])
        self.sparse_p = C.SparseParams(C.AttendParams(self.cache_p, HEADS, WIDTH * PAGE, D ** -0.5), TOP, 1, 2)
        self.ws = [torch.empty(n + 256, dtype=torch.uint8, device="cuda") for n in (C.pages_workspace_size(self.pages_p), C.sparse_workspace_size(self.sparse_p))]
        self.steps = C.rotary_steps(32, 10000.0, C.ROTARY_LINEAR, factor=2.0)

    def go(self, state, cache, summary, want, rows, x, visible=None):
        """Rows x [T, HEADS + 2 H, D] of the sequences' next positions: (tables of the step, queries, attention, log-sums, blocks)."""
        import paper_2605_02218_amd as C
        at = C.pages_step(self.pages_p, state, want, rows, workspace=self.ws[0])
        q = C.rotate_write(self.rotary_p, self.cache_p, x[:, :HEADS], x[:, HEADS:HEADS + H], x[:, HEADS + H:], self.steps, at.start, at.length, state[0], cache)
        C.block_summary(self.cache_p, at.start, at.length, state[0], cache, summary)
        out, lse, blocks = C.sparse_attend(self.sparse_p, q, at.start, at.length, state[0], cache, summary, visible=visible, workspace=self.ws[1], want_lse=True)
        return at, q, out, lse, blocks


@pytest.mark.parametrize("dtype,kept", [("bf16", "bf16"), ("bf16", "int8"), ("fp16", "e4m3")])
def test_rounds_that_stay_on_the_device(dtype, kept):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(23)
    prompts = [150, 20, 77]
    first, later = Round(dtype, kept, sum(prompts) + 5), Round(dtype, kept, S * L)
    state, cache, summary = C.pages_alloc(first.pages_p), C.cache_alloc(first.cache_p), C.block_alloc(first.cache_p)
    for t in cache:
        if t is not None:
            t.view(torch.uint8).fill_(0xFF)              # NaN in every type but int8, whose scales are NaN
    tables = SO.Tables(S, PAGE, N_PAGES, WIDTH, list(range(N_PAGES - 1, -1, -1)))
    steps = [v % (1 << 64) for v in first.steps.tolist()]
    want, lengths = torch.tensor(prompts, dtype=torch.int32, device="cuda"), list(prompts)
    rows = want.clone()
    held = [[] for _ in range(S)]                        # turned keys, position by position, fp64
    accepted = 0
    for turn in range(6):
        r = first if turn == 0 else later
        new = prompts if turn == 0 else [L] * S
        x, x32 = rounded(rng.standard_normal((r.T, HEADS + 2 * H, D)), dtype)
        bits = None
        if turn in (3, 4):                               # trees: each token behind the first
            bits = torch.tensor([1 << i | 1 for i in range(L)] * S, dtype=torch.int64, device="cuda")
        at, q, out, lse, blocks = r.go(state, cache, summary, want, rows, x.cuda(), bits)
        # meanwhile verification of random logits, and the lengths of the next round, without a look at any of it
        if turn > 0:
            zt = torch.from_numpy(rng.standard_normal((S, L, V)).astype(np.float32)).cuda().to(torch_dtype(dtype))
            zd = zt + 0.5 * torch.randn(S, L, V, device="cuda", generator=torch.Generator("cuda").manual_seed(turn)).to(zt.dtype)
            drafted = torch.from_numpy(rng.integers(0, V, (S, L)).astype(np.int32)).cuda()
            n_acc, _, _ = C.verify(C.VerifyParams(S, L, V, NAMES[dtype]), zt, zd, drafted, torch.from_numpy(rng.random((S, L)).astype(np.float32)).cuda(),
                                   torch.from_numpy(rng.random(S).astype(np.float32)).cuda())
            next_want = want + n_acc                     # L less those rejected, and L new ones
        else:
            next_want = want + L
        torch.cuda.synchronize()
        # the tables
        ref = tables.step(lengths, new, r.T)
        for name, got, y in zip(at._fields, at, ref):
            np.testing.assert_array_equal(got.cpu().numpy(), np.array(y), err_msg=name)
        b = SimpleNamespace(S=S, T=r.T, new=new, length=lengths, page=PAGE, n_pages=N_PAGES, width=WIDTH, start=ref[0], pages=state[0].cpu().numpy())
        # rotated queries, and keys as the cache holds them
        for s in range(S):
            del held[s][lengths[s] - new[s]:]
            for i in range(new[s]):
                t, pos = ref[0][s] + i, lengths[s] - new[s] + i
                for h in range(HEADS):
                    y, size = SO.turned(x32[t, h].astype(np.float64), [pos] * 16, steps, True)
                    assert np.all(np.abs(q[t, h].double().cpu().numpy() - y) <= HALF_STEP[dtype] * np.abs(y) + 2.0 ** -21 * size + 2.0 ** -25)
                held[s].append(np.stack([SO.turned(x32[t, HEADS + h].astype(np.float64), [pos] * 16, steps, True)[0] for h in range(H)]))
        pool = [(cache[i].cpu(), None if cache[2 + i] is None else cache[2 + i].cpu()) for i in range(2)]
        k32 = TS.k32_of(pool[0])
        k64, v64 = ((p[0].double().numpy() if p[1] is None else p[0].double().numpy() * p[1].double().numpy()[..., None]) for p in pool)
        half = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "int8": 2.0 ** -8, "e4m3": 2.0 ** -4}[kept]
        for s in range(S):
            for j in range(lengths[s]):
                pg, of = RO.place(j, b.pages[s], PAGE, N_PAGES)
                # 16 bits and e4m3: half a step of the value; int8, and e4m3 near zero, of the row's largest
                top = np.abs(held[s][j]).max(-1, keepdims=True)
                assert np.all(np.abs(k64[pg, :, of] - held[s][j]) <= (half * (top if kept == "int8" else np.abs(held[s][j])) + 2.0 ** -18 * top) * 1.01 + 2.0 ** -25), (s, j)
        # every page's summary is that of the positions its sequence has now
        codes, scale = TS.summaries(b, k32, H, D)
        for s in range(S):
            for blk in range(-(-lengths[s] // PAGE)):
                pg = b.pages[s, blk]
                assert np.array_equal(summary[0][pg].cpu().numpy(), codes[pg]) and np.array_equal(summary[1][pg].cpu().numpy(), scale[pg]), (s, blk)
        q32 = q.float().cpu().numpy()
        want_blocks = TS.wanted_blocks(b, codes, scale, q32, HEADS, H, TOP, 1, 2, bits is not None, WIDTH * PAGE)
        n = ref[0][-1]
        np.testing.assert_array_equal(blocks.cpu().numpy()[:n], want_blocks[:n])
        some = set(range(0, n, 11)) if turn == 0 else None
        TS.check_rows(b, want_blocks, HEADS, H, D, dtype, kept, k64, v64, q32, out, lse, D ** -0.5, None if bits is None else bits.cpu().numpy(), WIDTH * PAGE, some)
        if turn > 0:
            accepted += int(n_acc.sum())
        want, rows = next_want, torch.full_like(want, L)
        lengths = next_want.tolist()
    assert 0 < accepted < 5 * S * L


@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
def test_a_round_in_one_graph(kept):
    """Tables, rotation, summaries and attention captured together and replayed with other lengths and rows, with the program's own work between, against
    eager calls from the same state."""
    import torch
    import paper_2605_02218_amd as C
    r = Round("bf16", kept, S * L)
    want, rows = torch.tensor([100, 40, 7], dtype=torch.int32, device="cuda"), torch.full((S,), L, dtype=torch.int32, device="cuda")
    x = torch.randn(r.T, HEADS + 2 * H, D, device="cuda").to(torch.bfloat16)

    def fresh():
        state, cache, summary = C.pages_alloc(r.pages_p), C.cache_alloc(r.cache_p), C.block_alloc(r.cache_p)
        g = torch.Generator("cuda").manual_seed(5)
        for t in cache[:2]:
            t.view(torch.int8).copy_(torch.randint(-100, 60, t.view(torch.int8).shape, generator=g, device="cuda", dtype=torch.int32).to(torch.int8))
        for t in cache[2:]:
            if t is not None:
                t.fill_(0.01)
        return state, cache, summary

    a, b = fresh(), fresh()
    r.go(*a, want, rows, x)
    r.go(*b, want, rows, x)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            captured = r.go(*a, want, rows, x)
    for lens in ([104, 43, 9], [300, 4, 150], [96, 41, 3], [0, 300, 80], [33, 301, 79]):
        want.copy_(torch.tensor(lens, dtype=torch.int32))
        x.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in tuple(captured[0]) + captured[1:]]
        eager = r.go(*b, want, rows, x)
        torch.cuda.synchronize()
        n = int(got[0][-1])
        for i, (u, v) in enumerate(zip(got, tuple(eager[0]) + eager[1:])):
            u, v = (u[:n], v[:n]) if i >= 5 else (u, v)          # padding rows of new tensors are unspecified
            assert torch.equal(u.view(torch.uint8), v.view(torch.uint8)), i
        for u, v in zip(a[0][1:2] + a[0][3:] + a[1] + a[2], b[0][1:2] + b[0][3:] + b[1] + b[2]):
            if u is not None:
                assert torch.equal(u.view(torch.uint8), v.view(torch.uint8))


def test_two_streams_with_workspaces_of_their_own():
    """Two batches of one pool at the same time, on pages of their own; the same calls give the same bits."""
    import torch
    import paper_2605_02218_amd as C
    rounds = [Round("fp16", "fp16", S * L) for _ in range(2)]
    cache, summary = C.cache_alloc(rounds[0].cache_p), C.block_alloc(rounds[0].cache_p)
    g = torch.Generator("cuda").manual_seed(6)
    for t in cache[:2]:
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    whole = C.CacheParams(1, N_PAGES * PAGE, H, D, PAGE, N_PAGES, N_PAGES, C.FP16, C.FP16)
    C.block_summary(whole, torch.tensor([0, N_PAGES * PAGE], dtype=torch.int32, device="cuda"), torch.tensor([N_PAGES * PAGE], dtype=torch.int32, device="cuda"),
                    torch.arange(N_PAGES, dtype=torch.int32, device="cuda").view(1, -1), cache, summary)
    jobs = []
    for i, r in enumerate(rounds):
        table = (torch.arange(N_PAGES // 2, device="cuda") * 2 + i).to(torch.int32)[:S * 10].view(S, 10)
        pages = torch.zeros(S, WIDTH, dtype=torch.int32, device="cuda")
        pages[:, :10] = table
        q = torch.randn(S * L, HEADS, D, generator=g, device="cuda").to(torch.float16)
        start, length = torch.arange(0, S * L + 1, L, dtype=torch.int32, device="cuda"), torch.tensor([160, 90, 33], dtype=torch.int32, device="cuda")
        jobs.append((r, q, start, length, pages))

    def go(j):
        r, q, start, length, pages = j
        C.block_summary(r.cache_p, start, length, pages, cache, summary)
        return C.sparse_attend(r.sparse_p, q, start, length, pages, cache, summary, workspace=r.ws[1], want_lse=True)

    wanted = [go(j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(3):
        got = []
        for st, j in zip(streams, jobs):
            with torch.cuda.stream(st):
                got.append(go(j))
        torch.cuda.synchronize()
        for x, y in zip(got, wanted):
            assert all(torch.equal(u, v) for u, v in zip(x, y))
