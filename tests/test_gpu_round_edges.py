"""Edges of the entry points around a verification round that the tests of each of them leave out: calls that the documentation allows or refuses."""
import numpy as np
import pytest

from round_util import Batch

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
