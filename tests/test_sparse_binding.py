"""What the binding of page tables and attention over selected pages allocates by itself, on the host (no GPU work is launched): the workspace that a caller leaves out
is there, and is nobody else's memory, when the library is called."""
import weakref
from types import SimpleNamespace

import pytest

import paper_2605_02218_amd as C
from paper_2605_02218_amd import binding as Bd


class _Allocations:
    """Stands for what the binding asks of torch and of tensors on a device; memory is the host's."""

    def __init__(self, monkeypatch):
        import torch
        Bd._types()
        self.made, self.called, at_call = [], [], self.at_call

        def empty(*shape, dtype, device):
            t = torch.empty(*shape, dtype=dtype)
            self.made.append((weakref.ref(t), t.data_ptr(), t.numel() * t.element_size()))
            return t

        monkeypatch.setitem(Bd._TORCH, "torch", SimpleNamespace(empty=empty))
        monkeypatch.setattr(Bd, "_device_of", lambda t: torch.device("cpu"))
        monkeypatch.setattr(Bd, "_given", lambda dev, *items: [4096] * len(items))
        monkeypatch.setattr(Bd, "_given_rows", lambda dev, t, name, n, heads, dim, dtype: (4096, heads * dim))
        monkeypatch.setattr(Bd, "_ptr", lambda t: t.data_ptr())
        monkeypatch.setattr(Bd, "_launch", at_call)

    def at_call(self, dev, name, *args):
        assert all(t() is not None for t, _, _ in self.made), "freed before %s is called" % name
        spans = sorted((at, at + n) for _, at, n in self.made)
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
        at, n = args[-2:]
        assert any(lo <= at and at + n <= hi for lo, hi in spans)
        self.called.append(name)


@pytest.mark.parametrize("S,T", [(3, 8), (64, 5000), (1100, 20), (4, 0)])
@pytest.mark.parametrize("want_slots", [True, False])
def test_page_steps_hold_their_workspace(monkeypatch, S, T, want_slots):
    a = _Allocations(monkeypatch)
    p = C.PagesParams(S, T, 16, 100, 9)
    C.pages_step(p, [object()] * 5, object(), object(), want_slots=want_slots)
    assert a.called == ["covspec_pages_step"] and len(a.made) >= 2


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("tokens,max_len,top", [(1, 32000, 64), (4, 1000003, 128), (130, 4000, 9), (1, 100, 2)])
def test_sparse_attention_holds_its_workspace(monkeypatch, given, tokens, max_len, top):
    a = _Allocations(monkeypatch)
    cache = C.CacheParams(1, tokens, 2, 64, 64, 20000, 20000)
    p = C.SparseParams(C.AttendParams(cache, 16, max_len, 0.125), top)
    some = object()
    C.sparse_attend(p, some, some, some, some, [some] * 4, None if given else (some, some), blocks=some if given else None, want_lse=True)
    assert a.called == ["covspec_sparse_attend"] and len(a.made) >= 3
