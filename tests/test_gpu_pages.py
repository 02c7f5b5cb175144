"""GPU parity of covspec_pages_step with oracle/sparse_oracle.py: integers, compared as they are."""
import numpy as np
import pytest

from oracle import sparse_oracle as SO

pytestmark = pytest.mark.gpu


class Both:
    """The state on the device and the oracle's, from the same free pages."""

    def __init__(self, rng, S, page, n_pages, width, T):
        import torch
        import paper_2605_02218_amd as C
        self.p, self.T, self.S = C.PagesParams(S, T, page, n_pages, width), T, S
        free = rng.permutation(n_pages)
        self.oracle = SO.Tables(S, page, n_pages, width, [int(x) for x in free])
        self.state = C.pages_alloc(self.p)
        self.state[3].copy_(torch.from_numpy(free.astype(np.int32)))
        self.ws = torch.empty(C.pages_workspace_size(self.p) + 256, dtype=torch.uint8, device="cuda")

    def check_state(self):
        pages, held, borrowed, free, n_free = (t.cpu().numpy() for t in self.state)
        assert held.tolist() == [len(h) for h in self.oracle.held] and borrowed.tolist() == self.oracle.borrowed
        for s, h in enumerate(self.oracle.held):
            assert pages[s, :len(h)].tolist() == h, s
        assert int(n_free[0]) == len(self.oracle.free) and free[:len(self.oracle.free)].tolist() == self.oracle.free

    def step(self, want, rows):
        import torch
        import paper_2605_02218_amd as C
        self.ws.fill_(0xA5)
        up = lambda x: torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()        # noqa: E731
        got = C.pages_step(self.p, self.state, up(want), up(rows), workspace=self.ws)
        torch.cuda.synchronize()
        for name, x, y in zip(got._fields, got, self.oracle.step(want, rows, self.T)):
            if self.T > 0 or name not in ("slots", "positions"):
                np.testing.assert_array_equal(x.cpu().numpy(), np.array(y), err_msg=name)
        self.check_state()
        return got


@pytest.mark.parametrize("S,page,T", [(1, 16, 40), (3, 16, 100), (64, 32, 500), (65, 16, 6000), (1024, 64, 4096), (1025, 16, 3000), (2300, 16, 2000), (5000, 16, 30000)])
@pytest.mark.parametrize("tight", [False, True])
def test_steps_equal_the_oracle(S, page, T, tight):
    rng = np.random.default_rng(S + T)
    most = 300
    width = -(-most // page) + 1
    b = Both(rng, S, page, max(2, S * (3 if tight else width)), width, T)
    want = np.zeros(S, dtype=np.int64)
    for k in range(8):
        grow, kind = rng.integers(-9, 12, S), rng.random(S)
        want = np.where(kind < 0.1, 0, np.where(kind < 0.25, rng.integers(1, most + 40, S), np.maximum(want, 0) + grow))    # a few ask for more than the table holds
        rows = np.where(kind < 0.25, rng.integers(0, 40, S), rng.integers(-1, 10, S))
        if k == 6 and S > 2:
            b.oracle.borrowed = [min(int(x), len(h)) for x, h in zip(rng.integers(0, 4, S), b.oracle.held)]
            import torch
            b.state[2].copy_(torch.tensor(b.oracle.borrowed, dtype=torch.int32))
        b.step(want, rows)


def test_prompts_of_many_rows_and_no_rows_at_all():
    rng = np.random.default_rng(3)
    b = Both(rng, 7, 128, 3000, 400, 120000)
    b.step([40000, 1, 0, 30000, 128, 129, 9], [40000, 1, 0, 30000, 128, 1, 0])
    b.step([0, 2, 50000, 30001, 0, 0, 9], [0, 1, 50000, 1, 0, 0, 0])
    b = Both(rng, 7, 16, 100, 20, 0)
    b.step([5] * 7, [1] * 7)
    b.step([0] * 7, [0] * 7)


def test_back_and_forth_leaves_everything_as_it_was():
    import torch
    rng = np.random.default_rng(4)
    b = Both(rng, 200, 16, 4000, 30, 5000)
    first, one = rng.integers(0, 400, 200), np.ones(200, dtype=int)
    b.step(first, one)
    before = [t.clone() for t in b.state]
    for _ in range(3):
        b.step(rng.integers(0, 400, 200), one)
        b.step(first, one)
        assert torch.equal(b.state[3], before[3]) and torch.equal(b.state[1], before[1])


@pytest.mark.parametrize("T", [64, 20000])
def test_a_state_without_sense_stays_inside_its_arrays(T):
    """Marked bytes around every array; what the arrays hold is anything."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(5)
    S, width, n_pages = 40, 6, 50
    p = C.PagesParams(S, T, 16, n_pages, width)
    guarded = []

    def guard(n, dtype, fill):
        room = torch.full((n + 512,), 0x5A5A5A5A, dtype=dtype, device="cuda")
        t = room[256:256 + n]
        t.copy_(torch.from_numpy(np.asarray(fill)).to(dtype))
        guarded.append((room, n))
        return t

    wild = lambda n: rng.choice([-2 ** 31, -1, 0, 1, 3, 49, 50, 77, 2 ** 31 - 1], n)        # noqa: E731
    for _ in range(6):
        guarded.clear()
        state = (guard(S * width, torch.int32, wild(S * width)).view(S, width), *(guard(n, torch.int32, wild(n)) for n in (S, S, n_pages, 1)))
        want, rows = guard(S, torch.int32, wild(S)), guard(S, torch.int32, wild(S))
        outs = [guard(n, t, np.zeros(n)) for n, t in ((S + 1, torch.int32), (S, torch.int32), (S, torch.int32), (T, torch.int64), (T, torch.int32))]
        n = C.pages_workspace_size(p)
        ws = torch.full((n + 512,), 0x5A, dtype=torch.uint8, device="cuda")
        import ctypes
        cs, at = p.c_struct(), (ws.data_ptr() + 255) // 256 * 256
        st = C.load_library().covspec_pages_step(ctypes.byref(cs), want.data_ptr(), rows.data_ptr(), *[t.data_ptr() for t in state], *[t.data_ptr() for t in outs], at, n,
                                                 torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == 0
        for room, n_ in guarded:
            assert bool((room[:256] == 0x5A5A5A5A).all()) and bool((room[256 + n_:] == 0x5A5A5A5A).all())
        assert bool((ws[at - ws.data_ptr() + n:] == 0x5A).all())
        start = outs[0].cpu().numpy()
        assert start[0] == 0 and np.all(np.diff(start) >= 0) and start[-1] <= T
        held, n_free = state[1].cpu().numpy(), int(state[4][0])
        assert np.all((held >= 0) & (held <= width)) and 0 <= n_free <= n_pages
        slots = outs[3].cpu().numpy()
        assert np.all((slots >= -1) & (slots < n_pages * 16))


def test_captured_steps_follow_the_lengths():
    """A graph of one step, replayed with other lengths, against eager steps from the same state."""
    import torch
    import paper_2605_02218_amd as C
    S, T = 30, 400
    p = C.PagesParams(S, T, 16, 600, 24)
    a, b = C.pages_alloc(p), C.pages_alloc(p)
    ws = [torch.empty(C.pages_workspace_size(p) + 256, dtype=torch.uint8, device="cuda") for _ in range(2)]
    want, rows = (torch.zeros(S, dtype=torch.int32, device="cuda") for _ in range(2))
    C.pages_step(p, a, want, rows, workspace=ws[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = C.pages_step(p, a, want, rows, workspace=ws[0])
    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(5):
        want.copy_(torch.randint(0, 300, (S,), generator=g, device="cuda"))
        rows.copy_(torch.randint(0, 20, (S,), generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        ref = C.pages_step(p, b, want, rows, workspace=ws[1])
        for x, y in zip(tuple(got) + a, tuple(ref) + b):
            assert torch.equal(x, y)
        torch.cuda.synchronize()
