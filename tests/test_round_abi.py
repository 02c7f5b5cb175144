"""Host-side checks of the entry points around a verification round: layouts, refusals (no GPU work is launched)."""
import ctypes

import pytest

import paper_2605_02218_amd as C
from paper_2605_02218_amd import binding as Bd

FAKE, BIG = 4096, 1 << 50       # pointers are never dereferenced: validation fails first


def _cache(**kw):
    base = dict(n_seq=3, n_tokens=24, n_kv_heads=8, head_dim=128, page_size=64, n_pages=100, max_pages=16, dtype=C.BF16, cache_dtype=C.BF16)
    base.update(kw)
    return C.CacheParams(**base)


CACHE_REFUSALS = [
    (dict(n_seq=0), Bd.INVALID_ARG), (dict(n_tokens=0), Bd.INVALID_ARG), (dict(n_kv_heads=0), Bd.INVALID_ARG), (dict(n_pages=0), Bd.INVALID_ARG),
    (dict(max_pages=0), Bd.INVALID_ARG), (dict(page_size=0), Bd.INVALID_ARG), (dict(head_dim=-64), Bd.INVALID_ARG),
    (dict(dtype=C.FP32), Bd.INVALID_ARG), (dict(dtype=C.INT8), Bd.INVALID_ARG), (dict(cache_dtype=C.FP16), Bd.INVALID_ARG), (dict(cache_dtype=C.FP32), Bd.INVALID_ARG),
    (dict(cache_dtype=5), Bd.INVALID_ARG), (dict(head_dim=80), Bd.UNSUPPORTED), (dict(head_dim=256), Bd.UNSUPPORTED), (dict(page_size=8), Bd.UNSUPPORTED),
    (dict(page_size=48), Bd.UNSUPPORTED), (dict(page_size=2048), Bd.UNSUPPORTED), (dict(n_tokens=1 << 28), Bd.UNSUPPORTED), (dict(n_tokens=1 << 24), Bd.UNSUPPORTED), (dict(max_pages=1 << 24), Bd.UNSUPPORTED),
    (dict(n_pages=1 << 30, page_size=1024), Bd.UNSUPPORTED),
]


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(Bd.CovspecCacheParams) == 48 and Bd.CovspecCacheParams.row_pitch.offset == 40
    assert ctypes.sizeof(Bd.CovspecAttendParams) == 80 and Bd.CovspecAttendParams.q_pitch.offset == 64
    assert ctypes.sizeof(Bd.CovspecLogitsParams) == 16


@pytest.mark.parametrize("kw,status", CACHE_REFUSALS)
def test_cache_parameters_are_refused_on_the_host(kw, status):
    lib = C.load_library()
    cs = _cache(**kw).c_struct()
    assert lib.covspec_cache_write(ctypes.byref(cs), *[FAKE] * 9, None) == status
    assert lib.covspec_cache_read(ctypes.byref(cs), *[FAKE] * 9, None) == status
    a = C.AttendParams(cache=_cache(**kw), n_heads=8, max_len=100, scale=0.1)
    assert C.attend_workspace_size(a) == 0
    ac = a.c_struct()
    assert lib.covspec_attend(ctypes.byref(ac), *[FAKE] * 8, None, FAKE, None, FAKE, BIG, None) == status


def test_cache_pointers_and_pitch_are_checked():
    lib = C.load_library()
    cs = _cache(cache_dtype=C.INT8).c_struct()
    for hole in range(9):
        for call in (lib.covspec_cache_write, lib.covspec_cache_read):
            assert call(ctypes.byref(cs), *[None if i == hole else FAKE for i in range(9)], None) == Bd.INVALID_ARG
    # order: k v start length pages k_cache v_cache k_scale v_scale
    for i in (0, 1, 5, 6):
        assert lib.covspec_cache_write(ctypes.byref(cs), *[FAKE + 8 if j == i else FAKE for j in range(9)], None) == Bd.INVALID_ARG
    for i in (2, 3, 4, 7, 8):
        assert lib.covspec_cache_write(ctypes.byref(cs), *[FAKE + 2 if j == i else FAKE for j in range(9)], None) == Bd.INVALID_ARG
    for pitch in (-8, 8, 1016, 1028):
        cs = _cache().c_struct(pitch)
        assert lib.covspec_cache_write(ctypes.byref(cs), *[FAKE] * 9, None) == Bd.INVALID_ARG
    assert lib.covspec_cache_write(None, *[FAKE] * 9, None) == Bd.INVALID_ARG


def test_attend_parameters_are_checked():
    lib = C.load_library()
    ok = dict(cache=_cache(), n_heads=64, max_len=1024, scale=0.1)
    need = C.attend_workspace_size(C.AttendParams(**ok))
    assert need > 0
    args = lambda **kw: [kw.get(n, FAKE) for n in ("q", "start", "length", "pages", "kc", "vc", "ks", "vs")] + [  # noqa: E731
        kw.get("visible"), kw.get("out", FAKE), kw.get("lse"), kw.get("ws", FAKE), kw.get("bytes", BIG), None]
    for kw, status in [(dict(n_heads=0), Bd.INVALID_ARG), (dict(n_heads=12), Bd.INVALID_ARG), (dict(max_len=0), Bd.INVALID_ARG), (dict(max_len=1025), Bd.INVALID_ARG),
                       (dict(window=-1), Bd.INVALID_ARG), (dict(scale=float("nan")), Bd.INVALID_ARG), (dict(scale=float("inf")), Bd.INVALID_ARG),
                       (dict(n_heads=8 * 65), Bd.UNSUPPORTED), (dict(cache=_cache(n_tokens=1 << 25), n_heads=64), Bd.UNSUPPORTED),
                       (dict(cache=_cache(n_seq=1 << 27)), Bd.UNSUPPORTED), (dict(cache=_cache(n_seq=1 << 26), n_heads=512), Bd.UNSUPPORTED)]:
        p = C.AttendParams(**{**ok, **kw})
        assert C.attend_workspace_size(p) == 0, kw
        cs = p.c_struct()
        assert lib.covspec_attend(ctypes.byref(cs), *args()) == status, kw
    cs = C.AttendParams(**ok).c_struct()
    for n in ("q", "start", "length", "pages", "kc", "vc", "out", "ws"):
        assert lib.covspec_attend(ctypes.byref(cs), *args(**{n: None})) == Bd.INVALID_ARG, n
    for n, by in (("q", 8), ("out", 8), ("kc", 8), ("ws", 128), ("visible", 4), ("lse", 2)):
        assert lib.covspec_attend(ctypes.byref(cs), *args(**{n: FAKE + by})) == Bd.INVALID_ARG, n
    assert lib.covspec_attend(ctypes.byref(cs), *args(bytes=need - 1)) == Bd.WORKSPACE_TOO_SMALL
    assert lib.covspec_attend(None, *args()) == Bd.INVALID_ARG
    cs = C.AttendParams(**ok, window=5).c_struct()
    assert lib.covspec_attend(ctypes.byref(cs), *args(visible=FAKE)) == Bd.INVALID_ARG            # a tree has no window
    cs = C.AttendParams(**{**ok, "cache": _cache(cache_dtype=C.E4M3)}).c_struct()
    assert lib.covspec_attend(ctypes.byref(cs), *args(ks=None)) == Bd.INVALID_ARG
    for q, o in ((8, 0), (0, 64 * 128 + 4), (-8, 0)):
        cs = C.AttendParams(**ok).c_struct(q, o)
        assert lib.covspec_attend(ctypes.byref(cs), *args()) == Bd.INVALID_ARG


def test_adjust_parameters_are_checked():
    lib = C.load_library()
    good = [FAKE] * 11          # z history history_start prompt_len drafted penalties bias_start bias_word bias_value allowed z_out
    for p, status in [(C.LogitsParams(0, 1, 4096), Bd.INVALID_ARG), (C.LogitsParams(1, 0, 4096), Bd.INVALID_ARG), (C.LogitsParams(1, 1, 1), Bd.INVALID_ARG),
                      (C.LogitsParams(1, 1, 4096, C.INT8), Bd.INVALID_ARG), (C.LogitsParams(1, 65, 4096), Bd.UNSUPPORTED), (C.LogitsParams(8192, 8, 4096), Bd.UNSUPPORTED),
                      (C.LogitsParams(1, 1, 4100, C.BF16), Bd.UNSUPPORTED), (C.LogitsParams(1, 1, 4098, C.FP32), Bd.UNSUPPORTED)]:
        cs = p.c_struct()
        assert lib.covspec_adjust_logits(ctypes.byref(cs), *good, None) == status
    cs = C.LogitsParams(2, 3, 4096).c_struct()
    for hole in (0, 1, 2, 5, 6, 7, 8, 10):      # one of the three bias arrays missing counts too
        assert lib.covspec_adjust_logits(ctypes.byref(cs), *[None if i == hole else FAKE for i in range(11)], None) == Bd.INVALID_ARG
    for i in range(11):
        off = 8 if i in (0, 10) else 2
        assert lib.covspec_adjust_logits(ctypes.byref(cs), *[FAKE + off if j == i else FAKE for j in range(11)], None) == Bd.INVALID_ARG
    assert lib.covspec_adjust_logits(None, *good, None) == Bd.INVALID_ARG


def test_the_binding_refuses_tensors_that_do_not_fit():
    import torch
    p = _cache(n_seq=1, n_tokens=2, n_pages=2, max_pages=2)
    host = torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        C.cache_write(p, host, host, i, i[:1], i.view(1, 2), (host, host, None, None))             # not on a device
    with pytest.raises(ValueError):
        Bd._expect(i, "start", (3,), torch.int32)
    with pytest.raises(ValueError):
        Bd._expect(i, "start", (2,), torch.int64)
    with pytest.raises(ValueError):
        Bd._rows(host, "k", 2, 8, 64, torch.bfloat16)
    with pytest.raises(ValueError):
        Bd._same_device(host, None)
