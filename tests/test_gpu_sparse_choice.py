"""The choice of pages where rows times key heads are many, which a launch with a wave for each of them makes (1024 and more, several rows a sequence), and beside it in its
other forms: by a workgroup each, by the attention's own.  Lists are compared with oracle/sparse_oracle.py as they are, between marked words."""
import numpy as np
import pytest

import test_gpu_sparse as TS
from round_util import Batch

pytestmark = pytest.mark.gpu

PAGE, D = 16, 64


def patterned(rng, b, H, kinds):
    """Codes and scales of all pages, of `kinds` different ones, so that many tie."""
    codes = rng.integers(-127, 128, (kinds, H, 2, D)).astype(np.int8)
    codes.sort(axis=2)
    codes = codes[:, :, ::-1]                               # the largest first
    scale = rng.uniform(0.01, 0.05, (kinds, H)).astype(np.float32)
    kind = rng.integers(0, kinds, b.n_pages)
    return np.ascontiguousarray(codes[kind]), scale[kind]


def check(rng, b, heads, H, codes, scale, top, first=1, recent=1, visible=None, rows=(), positive=False, shrink=1.0):
    import torch
    import paper_2605_02218_amd as C
    k, v, q, q32 = TS.make(rng, b, heads, H, D, "bf16", "bf16")
    q, q32 = q * shrink, q32 * np.float32(shrink)           # a power of two
    if positive:                                            # every score has the sign of its page's codes
        q, q32 = q.abs(), np.abs(q32)
    cap = min(max(b.length), b.width * b.page)
    p = C.SparseParams(C.AttendParams(b.params(H, D, "bf16", "bf16"), heads, cap, 0.125), top, first, recent)
    room = torch.full((b.T * H * top + 4096,), 77, dtype=torch.int32, device="cuda")
    blocks = room[2048:2048 + b.T * H * top].view(b.T, H, top)
    vis = None if visible is None else torch.from_numpy(visible).cuda()
    out, lse, got = C.sparse_attend(p, q.cuda(), *b.device(), TS.upload(k, v), (torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda()), visible=vis, blocks_out=blocks,
                                    want_lse=True)
    torch.cuda.synchronize()
    n = int(b.start[-1])
    want = TS.wanted_blocks(b, codes, scale, q32, heads, H, top, first, recent, visible is not None, cap)
    np.testing.assert_array_equal(got.cpu().numpy()[:n], want[:n])
    assert bool((room[:2048] == 77).all()) and bool((room[2048 + n * H * top:] == 77).all())
    TS.check_rows(b, want, heads, H, D, "bf16", "bf16", k[2], v[2], q32, out, lse, 0.125, visible, cap, set(rows))
    return want


@pytest.mark.parametrize("nb", [300, 500, 1500, 2000])
@pytest.mark.parametrize("T,H", [(130, 8), (6, 2), (1, 1)])
def test_more_nan_scales_than_places_beside_negative_scores(nb, T, H):
    rng = np.random.default_rng(nb + T)
    b = Batch(rng, [T], [PAGE * nb], PAGE, pad=2)
    codes = np.full((b.n_pages, H, 2, D), 90, dtype=np.int8)
    scale = np.full((b.n_pages, H), 0.02, dtype=np.float32)
    scale[b.pages[0, rng.permutation(np.arange(1, nb - 12))[:100]]] = np.nan
    low = int(np.flatnonzero(~np.isnan(scale[b.pages[0, 1:], 0]))[0]) + 1
    codes[b.pages[0, low]] = -90
    want = check(rng, b, 2 * H, H, codes, scale, 48, rows=[0, T - 1], positive=True)
    assert np.isnan(scale[b.pages[0, want[0, 0, 1:47]], 0]).all()


@pytest.mark.parametrize("nb", [9, 255, 256, 257, 1000, 2047, 2048])
@pytest.mark.parametrize("top,first,recent", [(1, 0, 0), (7, 1, 2), (48, 0, 1), (300, 3, 3)])
def test_many_rows_of_a_sequence(nb, top, first, recent):
    """Up to the most blocks that a wave holds; pages that tie, some of no score, some that do not exist; lists longer than the sequence."""
    rng = np.random.default_rng(nb + top)
    b = Batch(rng, [130], [PAGE * nb], PAGE, pad=1)
    H = 8
    codes, scale = patterned(rng, b, H, 7)
    scale[b.pages[0, nb // 2]], scale[b.pages[0, nb // 3]] = np.nan, 0.0
    b.pages[0, nb // 4], b.pages[0, nb - 2] = -1, b.n_pages
    check(rng, b, H, H, codes, scale, top, first, recent, rows=[0, 64, 129])


@pytest.mark.parametrize("kinds", [1, 3, 10 ** 6])
@pytest.mark.parametrize("heads,H", [(16, 16), (24, 8), (40, 4)])
@pytest.mark.parametrize("tree", [False, True])
def test_many_rows_of_sequences_of_all_lengths(kinds, heads, H, tree):
    rng = np.random.default_rng(kinds % 97 + heads)
    scaled = 16 // H
    new = [40 * scaled, 0, 65 * scaled, 1, 25 * scaled]
    b = Batch(rng, new, [20000, 40, 16 * 1023 + 5, 1, 25 * scaled], PAGE, pad=3)
    codes, scale = patterned(rng, b, H, min(kinds, b.n_pages))
    b.pages[0, [3, 700]], b.pages[2, 11] = -5, 1 << 30
    visible = rng.integers(-2 ** 63, 2 ** 63, b.T, dtype=np.int64) if tree else None
    check(rng, b, heads, H, codes, scale, 20, 2, 2, visible=visible, rows=range(0, b.T, 29))


@pytest.mark.parametrize("nb", [250, 1500])
@pytest.mark.parametrize("T,H", [(130, 8), (6, 2), (1, 1)])
def test_scores_that_round_to_zero_tie_whatever_their_sign(nb, T, H):
    """Below half of the smallest number a negative score is -0 and a positive one +0: equal, so the lower blocks are taken."""
    rng = np.random.default_rng(nb + T)
    b = Batch(rng, [T], [PAGE * nb], PAGE)
    codes = np.full((b.n_pages, H, 2, D), 127, dtype=np.int8)
    codes[b.pages[0, 1:nb:2]] = -127
    scale = np.full((b.n_pages, H), 2.0 ** -95, dtype=np.float32)
    want = check(rng, b, H, H, codes, scale, 12, rows=[0, T - 1], positive=True, shrink=2.0 ** -85)
    assert want[0, 0, :11].tolist() == list(range(11))


@pytest.mark.parametrize("nb", [250, 1500])
@pytest.mark.parametrize("T,H", [(130, 8), (6, 2), (1, 1)])
def test_scores_below_the_normal_numbers(nb, T, H):
    rng = np.random.default_rng(nb + T)
    b = Batch(rng, [T], [PAGE * nb], PAGE)
    codes, scale = patterned(rng, b, H, 10 ** 4)
    check(rng, b, 2 * H, H, codes, scale * np.float32(2.0 ** -60), 12, rows=[0, T - 1], shrink=2.0 ** -82)


@pytest.mark.parametrize("nb,T,H,top", [(32768, 2, 1, 1024), (32768, 1, 1, 1), (32767, 3, 1, 48), (2049, 130, 8, 48), (4200, 130, 8, 7)])
def test_more_blocks_than_a_wave_holds(nb, T, H, top):
    """By a workgroup each: up to the most blocks there can be, and many rows."""
    rng = np.random.default_rng(nb + T)
    b = Batch(rng, [T], [PAGE * nb], PAGE, pad=1)
    codes, scale = patterned(rng, b, H, 5000)
    scale[b.pages[0, nb // 2:nb // 2 + 60]] = np.nan
    b.pages[0, [nb // 4, nb - 5]] = -1, b.n_pages
    check(rng, b, H, H, codes, scale, top, min(top, 2) - 1, min(top, 2) - 1, rows=[0, T - 1])
