"""Host-side checks of what the binding makes of tensors before the library sees them (no GPU work is launched)."""
import ctypes

import pytest

import paper_2605_02218_amd as C
from paper_2605_02218_amd import binding as Bd


class _OnDevice:
    """What the binding asks of a device tensor, for its checks on the host."""

    def __init__(self, host):
        self.host, self.is_cuda, self.dtype, self.shape, self.device = host, True, host.dtype, host.shape, "a device"

    def __getattr__(self, name):
        return getattr(self.host, name)


@pytest.mark.parametrize("heads", [1, 8])
def test_rows_that_overlap_are_refused(heads):
    """Rows 0 elements apart (an expanded tensor) are no dense rows, for which 0 stands in the library's parameters."""
    import torch
    x = torch.zeros(5, heads, 128, dtype=torch.bfloat16)
    assert Bd._rows(_OnDevice(x), "k", 5, heads, 128, torch.bfloat16) == (x.data_ptr(), heads * 128)
    assert Bd._rows(_OnDevice(x[:1]), "k", 1, heads, 128, torch.bfloat16) == (x.data_ptr(), heads * 128)
    assert Bd._rows(_OnDevice(x[:1].expand(1, heads, 128)), "k", 1, heads, 128, torch.bfloat16) == (x.data_ptr(), heads * 128)
    wide = torch.zeros(5, heads + 3, 128, dtype=torch.bfloat16)[:, 2:2 + heads]
    assert Bd._rows(_OnDevice(wide), "k", 5, heads, 128, torch.bfloat16) == (wide.data_ptr(), (heads + 3) * 128)
    for bad in (x[:1].expand(5, heads, 128), x.view(-1).as_strided((5, heads, 128), (8, 128, 1))):
        with pytest.raises(ValueError, match="overlap"):
            Bd._rows(_OnDevice(bad), "k", 5, heads, 128, torch.bfloat16)


def test_a_workspace_is_what_lies_behind_its_first_aligned_byte():
    import torch
    x = torch.zeros(2048, dtype=torch.uint8)
    first = -x.data_ptr() % 256
    assert Bd._ws_args(_OnDevice(x[first:])) == (x.data_ptr() + first, 2048 - first)
    assert Bd._ws_args(_OnDevice(x[first:first + 1024].view(torch.float32))) == (x.data_ptr() + first, 1024)
    assert Bd._ws_args(_OnDevice(x[first + 1:first + 600])) == (x.data_ptr() + first + 256, 600 - 256)
    # it ends in front of that byte: nothing is left, not a size below zero, which the library would take for a huge one
    assert Bd._ws_args(_OnDevice(x[first + 1:first + 11]))[1] == 0
    for bad in (_OnDevice(x[:1].expand(4096)), _OnDevice(x[::2]), x):       # the last one is not on a device
        with pytest.raises(ValueError):
            Bd._ws_args(bad)


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16, C.FP16])
def test_vocabularies_beyond_the_word_indexes_are_refused(dtype):
    fake = 4096                 # never dereferenced
    for vocab in ((1 << 31) - 8, 1 << 30):
        cs = C.LogitsParams(1, 1, vocab, dtype).c_struct()
        assert C.load_library().covspec_adjust_logits(ctypes.byref(cs), *[fake] * 11, None) == Bd.UNSUPPORTED


@pytest.mark.parametrize("heads,tile", [(8, 16), (32, 32)])
def test_shares_are_as_many_as_are_at_work_at_once(heads, tile):
    """8 tokens, 8 key heads of 128, a 16-bit cache: four waves with 16-bit tiles of their own fill a compute unit's LDS, 256 shares; over codes two
    workgroups fit.  A share keeps two tiles of partial sums and their statistics."""
    for kept, shares in ((C.BF16, 256), (C.E4M3, 512)):
        c = C.CacheParams(n_seq=1, n_tokens=8, n_kv_heads=8, head_dim=128, page_size=64, n_pages=100, max_pages=100, dtype=C.BF16, cache_dtype=kept)
        need = C.attend_workspace_size(C.AttendParams(cache=c, n_heads=heads, max_len=6000, scale=0.1))
        sums = 2 * shares * tile * (128 + 2) * 4
        assert sums < need < sums + 4096
