"""Page tables and attention over selected pages without a workspace of the caller's: what the binding allocates for the call is nobody else's memory."""
import numpy as np
import pytest

import test_gpu_sparse as TS
from round_util import Batch
from test_gpu_pages import Both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S,T", [(64, 5000), (1024, 4097), (1025, 3000), (1100, 20000), (2, 100), (65536, 300000)])
def test_page_steps_equal_the_oracle(S, T):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(S)
    b = Both(rng, S, 16, 12 * S, 20, T)
    up = lambda x: torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()        # noqa: E731
    for _ in range(4):
        want, rows = rng.integers(0, 300, S), rng.integers(0, 80, S)
        got = C.pages_step(b.p, b.state, up(want), up(rows))
        torch.cuda.synchronize()
        for name, x, y in zip(got._fields, got, b.oracle.step(want, rows, T)):
            np.testing.assert_array_equal(x.cpu().numpy(), np.array(y), err_msg=name)
        b.check_state()


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("new,length,top", [([1], [9000], 128), ([4], [20000], 128), ([30, 30], [4000, 3000], 9), ([600], [6000], 9), ([1, 1], [100, 60], 4)])
def test_attention_is_that_with_a_workspace_and_repeats_itself(new, length, top, given):
    """Scores in a launch of their own, lists in pieces, the choice apart and inside; log-sums, which are allocated behind the workspace."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(sum(length))
    b, heads, H, D = Batch(rng, new, length, 16), 4, 2, 64
    k, v, q, _ = TS.make(rng, b, heads, H, D, "bf16", "bf16")
    codes, scale = TS.summaries(b, TS.k32_of(k), H, D)
    summary = torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda()
    p = C.SparseParams(C.AttendParams(b.params(H, D, "bf16", "bf16"), heads, max(length), 0.125), top)
    q, batch, pool = q.cuda(), b.device(), TS.upload(k, v)
    ws = torch.full((C.sparse_workspace_size(p) + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    want = C.sparse_attend(p, q, *batch, pool, summary, workspace=ws, want_lse=True)
    blocks = want[2] if given else None
    for _ in range(3):
        got = C.sparse_attend(p, q, *batch, pool, None if given else summary, blocks=blocks, want_lse=True)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
