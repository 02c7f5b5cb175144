"""GPU parity of covspec_cache_write and covspec_cache_read with oracle/round_oracle.py.  Codes, scales and what is read back are defined in
fp32 arithmetic with each operation rounded on its own, so everything is compared bit for bit."""
import numpy as np
import pytest

from oracle import round_oracle as RO
from round_util import Batch, pool_of, rounded, torch_dtype

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "bf16"), ("bf16", "int8"), ("bf16", "e4m3"), ("fp16", "fp16"), ("fp16", "int8"), ("fp16", "e4m3")]


def _bytes(t):
    import torch
    return t.contiguous().view(torch.uint8).cpu().numpy()


def _sentinel_pool(p, kept):
    """A pool full of marked bytes, so that a place that should not change shows."""
    import torch
    import paper_2605_02218_amd as C
    pool = C.cache_alloc(p)
    for t in pool:
        if t is not None:
            t.view(torch.uint8).fill_(0x5A)
    return pool


def _write_case(dtype, kept, H, D, b, rng, special=False):
    """Writes a batch and compares the whole pool."""
    import torch
    import paper_2605_02218_amd as C
    x = {n: rng.standard_normal((b.T, H, D)) * np.exp(rng.standard_normal((b.T, H, 1)) * 2) for n in "kv"}
    if special:
        for a in x.values():
            a[0, 0] = 0.0
            a[min(1, b.T - 1), 0, 3] = np.inf
            a[min(2, b.T - 1), 0, 5] = np.nan
            a[min(3, b.T - 1), 0] *= 1e-38 if dtype == "bf16" else 1e-6       # bf16: below the smallest that is kept
    host = {n: rounded(a, dtype) for n, a in x.items()}
    p = b.params(H, D, dtype, kept)
    pool = _sentinel_pool(p, kept)
    want = [None if t is None else t.cpu().clone() for t in pool]
    # k and v as columns of one wider row, queries in front of them
    wide = torch.zeros(b.T, 3 * H, D, dtype=torch_dtype(dtype))
    wide[:, H:2 * H], wide[:, 2 * H:] = host["k"][0], host["v"][0]
    wide = wide.cuda()
    start, length, pages = b.device()
    C.cache_write(p, wide[:, H:2 * H], wide[:, 2 * H:], start, length, pages, pool)
    torch.cuda.synchronize()
    for t, to in enumerate(b.places()):
        if to is None or to == "padding":
            continue
        for i, n in enumerate("kv"):
            if kept == dtype:
                want[i][to[0], :, to[1]] = host[n][0][t]
            else:
                c, s = RO.quantise(host[n][1][t], kept)
                want[i][to[0], :, to[1]] = torch.from_numpy(c).to(torch_dtype(kept))
                want[2 + i][to[0], :, to[1]] = torch.from_numpy(s)
    for name, got, ref in zip(("k", "v", "k_scale", "v_scale"), pool, want):
        if ref is not None:
            if name.endswith("scale"):
                np.testing.assert_array_equal(got.cpu().numpy().view(np.uint32) & 0x7FFFFFFF, ref.numpy().view(np.uint32) & 0x7FFFFFFF, err_msg=name)
            else:
                a, r = _bytes(got), _bytes(ref)
                if kept == "e4m3":          # zeros of either sign are equal
                    a, r = np.where(a == 0x80, 0, a), np.where(r == 0x80, 0, r)
                np.testing.assert_array_equal(a, r, err_msg=name)


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("D,H,page", [(64, 3, 16), (96, 2, 32), (128, 8, 64), (128, 1, 1024)])
def test_write_equals_the_oracle(dtype, kept, D, H, page):
    rng = np.random.default_rng(D * 7 + H)
    b = Batch(rng, [5, 0, 1, 40], [5, 30, 77, 131], page, pad=3)
    _write_case(dtype, kept, H, D, b, rng, special=True)


@pytest.mark.parametrize("kept", ["bf16", "int8"])
def test_rows_without_a_place_write_nothing(kept):
    rng = np.random.default_rng(5)
    b = Batch(rng, [4, 6, 3], [2, 70, 40], 16)          # two rows of the first sequence are in front of it
    b.length[2] = 16 * b.width + 1                      # the last row of the third lies beyond the table
    b.pages[1, 4] = b.n_pages                           # the last six rows of the second: no such page ...
    b.pages[2, b.width - 1] = -1                        # ... and those of the third on page -1
    assert sum(x is None for x in b.places()) == 2 + 6 + 3
    _write_case("bf16", kept, 2, 64, b, rng)
    b = Batch(rng, [1], [1], 16)
    b.length[0] = 0
    _write_case("bf16", kept, 2, 64, b, rng)


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("D,H,page", [(64, 5, 32), (96, 4, 16), (128, 8, 128)])
def test_read_equals_the_oracle(dtype, kept, D, H, page):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(D + H)
    b = Batch(rng, [7, 0, 100, 1], [7, 12, 230, 64], page, pad=2)
    b.new[0], b.length[0] = 7, 5                        # two positions that do not exist read as zeros
    b.pages[3, 0] = -7 if page > 32 else b.pages[3, 0]
    codes, scales = [], []
    for _ in range(2):
        c, s, _ = pool_of(rng.standard_normal((b.n_pages, H, page, D)) * 3, kept, dtype)
        if s is not None:
            s[0, 0, 0] = float("nan")                   # a row that held an infinity
        codes.append(c)
        scales.append(s)
    p = b.params(H, D, dtype, kept)
    pool = tuple(t.cuda() for t in codes) + tuple(None if s is None else s.cuda() for s in scales)
    wide = torch.full((b.T, 2 * H + 1, D), 7.0, dtype=torch_dtype(dtype), device="cuda")
    out = C.cache_read(p, pool, *b.device(), k_out=wide[:, :H], v_out=wide[:, H:2 * H])
    torch.cuda.synchronize()
    want = torch.full((b.T, 2 * H + 1, D), 7.0, dtype=torch_dtype(dtype))
    for t, at in enumerate(b.places()):
        if at == "padding":
            continue
        for i in range(2):
            if at is None:
                row = torch.zeros(H, D, dtype=torch_dtype(dtype))
            elif scales[i] is None:
                row = codes[i][at[0], :, at[1]]
            else:
                row = (codes[i][at[0], :, at[1]].float() * scales[i][at[0], :, at[1], None]).to(torch_dtype(dtype))
            want[t, i * H:(i + 1) * H] = row
    got, ref = wide.cpu().float().numpy(), want.float().numpy()
    np.testing.assert_array_equal(got, ref)             # NaN where NaN is wanted
    assert out[0].data_ptr() == wide.data_ptr()


def test_many_sequences_and_what_is_written_comes_back():
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(11)
    new = list(rng.integers(0, 4, 700))
    b = Batch(rng, new, [n + int(rng.integers(0, 40)) for n in new], 16)
    p = b.params(4, 64, "fp16", "fp16")
    k, v = (rounded(rng.standard_normal((b.T, 4, 64)), "fp16")[0].cuda() for _ in range(2))
    pool = _sentinel_pool(p, "fp16")
    batch = b.device()
    C.cache_write(p, k, v, *batch, pool)
    k2, v2 = C.cache_read(p, pool, *batch)
    assert torch.equal(k, k2) and torch.equal(v, v2)


def test_pools_beyond_four_gigabytes():
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(3)
    b = Batch(rng, [20], [40], 1024, spare=0)
    b.n_pages = 34000                                   # 1024 x 128 x 2 bytes a page: 8.9 GB in each pool
    b.pages[0, 0] = b.n_pages - 1
    p = b.params(1, 128, "bf16", "bf16")
    k, v = (rounded(rng.standard_normal((b.T, 1, 128)), "bf16")[0].cuda() for _ in range(2))
    pool = C.cache_alloc(p)
    for t in pool[:2]:
        t[-1].zero_()
        t[(b.n_pages - 1) % 16384].zero_()              # where an offset of 32 bits would land
    batch = b.device()
    C.cache_write(p, k, v, *batch, pool)
    k2, v2 = C.cache_read(p, pool, *batch)
    assert torch.equal(k, k2) and torch.equal(v, v2)
    assert torch.equal(pool[0][-1, 0, 20:40], k[:, 0]) and not pool[0][(b.n_pages - 1) % 16384].any() and not pool[0][-1, 0, 40:].any()
