"""Host-side checks of page tables, rotary positions and attention over selected pages: layouts, refusals, the steps of an angle (no GPU work is launched)."""
import ctypes

import pytest

import paper_2605_02218_amd as C
from oracle import sparse_oracle as SO
from paper_2605_02218_amd import binding as Bd

FAKE, BIG = 4096, 1 << 50       # pointers are never dereferenced: validation fails first


def _cache(**kw):
    base = dict(n_seq=3, n_tokens=24, n_kv_heads=8, head_dim=128, page_size=64, n_pages=100, max_pages=16, dtype=C.BF16, cache_dtype=C.BF16)
    base.update(kw)
    return C.CacheParams(**base)


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(Bd.CovspecPagesParams) == 20
    assert ctypes.sizeof(Bd.CovspecRotaryScaling) == 40 and Bd.CovspecRotaryScaling.base.offset == 8
    assert ctypes.sizeof(Bd.CovspecRotaryParams) == 72 and Bd.CovspecRotaryParams.magnitude.offset == 36 and Bd.CovspecRotaryParams.q_pitch.offset == 40
    assert ctypes.sizeof(Bd.CovspecSparseParams) == 96 and Bd.CovspecSparseParams.top.offset == 80


def test_pages_are_checked():
    lib = C.load_library()
    good = dict(n_seq=4, n_tokens=36, page_size=16, n_pages=50, max_pages=9)
    args = lambda n=None, by=None: [None if i == n and by is None else FAKE + by if i == n else FAKE for i in range(13)] + [BIG, None]     # noqa: E731
    for kw, status in [(dict(n_seq=0), Bd.INVALID_ARG), (dict(n_tokens=-1), Bd.INVALID_ARG), (dict(page_size=0), Bd.INVALID_ARG), (dict(n_pages=0), Bd.INVALID_ARG),
                       (dict(max_pages=0), Bd.INVALID_ARG), (dict(page_size=8), Bd.UNSUPPORTED), (dict(page_size=24), Bd.UNSUPPORTED), (dict(page_size=2048), Bd.UNSUPPORTED),
                       (dict(n_seq=65537), Bd.UNSUPPORTED), (dict(n_seq=65536, max_pages=1 << 14), Bd.UNSUPPORTED), (dict(n_tokens=1 << 30), Bd.UNSUPPORTED),
                       (dict(max_pages=1 << 26), Bd.UNSUPPORTED), (dict(n_pages=1 << 30), Bd.UNSUPPORTED)]:
        p = C.PagesParams(**{**good, **kw})
        assert C.pages_workspace_size(p) == 0, kw
        assert lib.covspec_pages_step(ctypes.byref(p.c_struct()), *args()) == status, kw
    p = C.PagesParams(**good)
    need, cs = C.pages_workspace_size(p), p.c_struct()
    # want rows pages held borrowed free n_free start length outcome slots positions workspace
    for i in range(13):
        if i not in (10, 11):
            assert lib.covspec_pages_step(ctypes.byref(cs), *args(i)) == Bd.INVALID_ARG, i
        assert lib.covspec_pages_step(ctypes.byref(cs), *args(i, 4 if i == 10 else 128 if i == 12 else 2)) == Bd.INVALID_ARG, i
    assert lib.covspec_pages_step(ctypes.byref(cs), *[FAKE] * 13, need - 1, None) == Bd.WORKSPACE_TOO_SMALL
    assert lib.covspec_pages_step(None, *args()) == Bd.INVALID_ARG


SCALINGS = [("plain", C.ROTARY_PLAIN, {}), ("linear", C.ROTARY_LINEAR, dict(factor=4.0)), ("base", C.ROTARY_BASE, dict(factor=7.0)),
            ("bands", C.ROTARY_BANDS, dict(factor=8.0, original=8192, low=1.0, high=4.0)), ("ramp", C.ROTARY_RAMP, dict(factor=16.0, original=4096, low=1.0, high=32.0)),
            ("ramp", C.ROTARY_RAMP, dict(factor=2.0, original=64, low=1e-9, high=40.0))]


@pytest.mark.parametrize("name,kind,kw", SCALINGS)
@pytest.mark.parametrize("R,base", [(64, 10000.0), (96, 500000.0), (128, 1e6), (16, 100.0), (2, 10000.0)])
def test_steps_are_those_of_the_formula(name, kind, kw, R, base):
    if name == "base" and R == 2:
        with pytest.raises(C.CovspecError):
            C.rotary_steps(R, base, kind, device="cpu", **kw)
        return
    got = C.rotary_steps(R, base, kind, device="cpu", **kw).tolist()
    for i, (a, want) in enumerate(zip(got, SO.rotary_turns(R, base, name, **kw))):
        # 64 bits of significand, some 20 roundings, exponents of up to 20 in the powers
        want = want * (1 << 64)
        assert abs((a % (1 << 64)) - want) <= 1 + float(want) * 2.0 ** -57, i
    if R == 64 and name == "plain":         # whole turns are left out
        fast = C.rotary_steps(R, 1e-4, device="cpu").tolist()
        for a, want in zip(fast, SO.rotary_turns(R, 1e-4)):
            diff = (a - int(want * (1 << 64))) % (1 << 64)
            assert min(diff, (1 << 64) - diff) <= 1 + float(want) * 2.0 ** 7


def test_scalings_are_checked():
    ok = dict(kind=C.ROTARY_BANDS, original_len=100, base=1e4, factor=2.0, low=1.0, high=4.0)
    out = (ctypes.c_uint64 * 32)()
    call = lambda R=64, **kw: C.load_library().covspec_rotary_steps(ctypes.byref(Bd.CovspecRotaryScaling(*{**ok, **kw}.values())), R, out)      # noqa: E731
    assert call() == Bd.OK and call(kind=C.ROTARY_RAMP) == Bd.OK
    inf, nan = float("inf"), float("nan")
    for kw in (dict(kind=-1), dict(kind=5), dict(base=0.0), dict(base=-1.0), dict(base=inf), dict(base=nan), dict(factor=0.0), dict(factor=nan), dict(original_len=0),
               dict(low=4.0), dict(low=nan), dict(high=inf), dict(kind=C.ROTARY_RAMP, low=0.0), dict(kind=C.ROTARY_RAMP, base=1.0), dict(R=0), dict(R=63), dict(R=-2)):
        assert call(**kw) == Bd.INVALID_ARG, kw
    assert call(kind=C.ROTARY_PLAIN, factor=nan, original_len=0, low=nan) == Bd.OK           # not looked at
    s = Bd.CovspecRotaryScaling(*ok.values())
    assert C.load_library().covspec_rotary_steps(None, 64, out) == Bd.INVALID_ARG and C.load_library().covspec_rotary_steps(ctypes.byref(s), 64, None) == Bd.INVALID_ARG


def test_rotations_are_checked():
    lib = C.load_library()
    good = dict(n_seq=3, n_tokens=24, n_heads=16, n_kv_heads=8, head_dim=128)
    a = lambda **kw: [kw.get(n, FAKE) for n in ("q", "k", "steps", "positions", "axis", "start", "length", "qo", "ko")] + [None]        # noqa: E731
    w = lambda **kw: [kw.get(n, FAKE) for n in ("q", "k", "v", "steps", "positions", "axis", "start", "length", "pages", "qo", "kc", "vc", "ks", "vs")] + [None]     # noqa: E731
    cc = _cache(cache_dtype=C.INT8).c_struct()
    for kw, status in [(dict(n_seq=0), Bd.INVALID_ARG), (dict(n_tokens=0), Bd.INVALID_ARG), (dict(n_heads=0), Bd.INVALID_ARG), (dict(n_kv_heads=0), Bd.INVALID_ARG),
                       (dict(head_dim=-1), Bd.INVALID_ARG), (dict(rotary_dim=-16), Bd.INVALID_ARG), (dict(rotary_dim=144), Bd.INVALID_ARG), (dict(n_axes=0), Bd.INVALID_ARG),
                       (dict(dtype=C.FP32), Bd.INVALID_ARG), (dict(dtype=C.INT8), Bd.INVALID_ARG), (dict(magnitude=float("nan")), Bd.INVALID_ARG),
                       (dict(magnitude=float("inf")), Bd.INVALID_ARG), (dict(interleaved=2), Bd.INVALID_ARG), (dict(head_dim=80), Bd.UNSUPPORTED), (dict(head_dim=256), Bd.UNSUPPORTED),
                       (dict(rotary_dim=24), Bd.UNSUPPORTED), (dict(n_axes=5), Bd.UNSUPPORTED), (dict(n_tokens=1 << 26), Bd.UNSUPPORTED), (dict(n_tokens=-(-(1 << 28) // 24)), Bd.UNSUPPORTED), (dict(n_seq=1 << 30), Bd.UNSUPPORTED)]:
        cs = C.RotaryParams(**{**good, **kw}).c_struct()
        assert lib.covspec_rotate(ctypes.byref(cs), *a()) == status, kw
        assert lib.covspec_rotate_write(ctypes.byref(cs), ctypes.byref(cc), *w()) == status, kw
    for pitch in ((8, 0, 0, 0), (0, 0, 4100, 0), (0, -8, 0, 0), (0, 0, 0, 1028)):
        cs = C.RotaryParams(**good).c_struct(*pitch)
        assert lib.covspec_rotate(ctypes.byref(cs), *a()) == Bd.INVALID_ARG, pitch
    cs = C.RotaryParams(**good).c_struct(0, (1 << 32) + 8)
    assert lib.covspec_rotate(ctypes.byref(cs), *a()) == Bd.UNSUPPORTED
    cs = C.RotaryParams(**good).c_struct()
    for kw in (dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(q=None, k=None, qo=None, ko=None), dict(steps=None), dict(start=None), dict(length=None),
               dict(start=None, length=None, positions=None), dict(q=FAKE + 8), dict(ko=FAKE + 8), dict(steps=FAKE + 4), dict(positions=FAKE + 2), dict(axis=FAKE + 2),
               dict(start=FAKE + 1), dict(length=FAKE + 2)):
        assert lib.covspec_rotate(ctypes.byref(cs), *a(**kw)) == Bd.INVALID_ARG, kw
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(steps=None), dict(start=None), dict(length=None), dict(pages=None), dict(qo=None), dict(kc=None),
               dict(vc=None), dict(ks=None), dict(vs=None), dict(q=FAKE + 8), dict(v=FAKE + 8), dict(qo=FAKE + 8), dict(kc=FAKE + 8), dict(steps=FAKE + 4)):
        assert lib.covspec_rotate_write(ctypes.byref(cs), ctypes.byref(cc), *w(**kw)) == Bd.INVALID_ARG, kw
    # in place only with rows on rows
    p = C.RotaryParams(**good).c_struct(16 * 128, 0, 32 * 128, 0)
    assert lib.covspec_rotate(ctypes.byref(p), *a()) == Bd.INVALID_ARG
    assert lib.covspec_rotate_write(ctypes.byref(p), ctypes.byref(cc), *w()) == Bd.INVALID_ARG
    for kw in (dict(n_seq=4), dict(n_tokens=23), dict(n_kv_heads=4), dict(head_dim=64), dict(dtype=C.FP16, cache_dtype=C.INT8)):
        assert lib.covspec_rotate_write(ctypes.byref(cs), ctypes.byref(_cache(**kw).c_struct()), *w()) == Bd.INVALID_ARG, kw
    assert lib.covspec_rotate_write(ctypes.byref(cs), ctypes.byref(_cache(page_size=8).c_struct()), *w()) == Bd.UNSUPPORTED
    assert lib.covspec_rotate_write(ctypes.byref(cs), None, *w()) == Bd.INVALID_ARG and lib.covspec_rotate(None, *a()) == Bd.INVALID_ARG


def test_summaries_and_sparse_attention_are_checked():
    lib = C.load_library()
    cs = _cache(cache_dtype=C.E4M3).c_struct()
    for i in range(7):
        args = [FAKE] * 7
        for bad in (None, FAKE + (8 if i in (3, 5) else 2)):
            args[i] = bad
            assert lib.covspec_block_summary(ctypes.byref(cs), *args, None) == Bd.INVALID_ARG, i
    assert lib.covspec_block_summary(None, *[FAKE] * 7, None) == Bd.INVALID_ARG
    assert lib.covspec_block_summary(ctypes.byref(_cache(head_dim=80).c_struct()), *[FAKE] * 7, None) == Bd.UNSUPPORTED
    assert lib.covspec_block_summary(ctypes.byref(_cache(n_seq=1 << 27, n_tokens=(1 << 27) - 1, n_kv_heads=1).c_struct()), *[FAKE] * 7, None) == Bd.UNSUPPORTED
    ok = dict(cache=_cache(), n_heads=64, max_len=1024, scale=0.1)
    args = lambda **kw: [kw.get(n, FAKE) for n in ("q", "start", "length", "pages", "kc", "vc", "ks", "vs", "summary", "scales")] + [       # noqa: E731
        kw.get("visible"), kw.get("blocks", FAKE), kw.get("out", FAKE), kw.get("lse"), kw.get("ws", FAKE), kw.get("bytes", BIG), None]
    for kw, mine, status in [(dict(n_heads=12), {}, Bd.INVALID_ARG), (dict(max_len=1025), {}, Bd.INVALID_ARG), (dict(window=5), {}, Bd.INVALID_ARG),
                             (dict(scale=float("nan")), {}, Bd.INVALID_ARG), (dict(n_heads=8 * 65), {}, Bd.UNSUPPORTED), ({}, dict(top=0), Bd.INVALID_ARG),
                             ({}, dict(first=-1), Bd.INVALID_ARG), ({}, dict(recent=-1), Bd.INVALID_ARG), ({}, dict(first=5, recent=4), Bd.INVALID_ARG),
                             ({}, dict(first=(1 << 31) - 1, recent=(1 << 31) - 1), Bd.INVALID_ARG), ({}, dict(top=1025), Bd.UNSUPPORTED),
                             (dict(cache=_cache(page_size=16, max_pages=40000), max_len=16 * 32769), {}, Bd.UNSUPPORTED),
                             (dict(cache=_cache(n_tokens=1 << 23)), {}, Bd.UNSUPPORTED)]:
        p = C.SparseParams(**{**dict(attend=C.AttendParams(**{**ok, **kw}), top=8, first=1, recent=2), **mine})
        assert C.sparse_workspace_size(p) == 0, (kw, mine)
        assert lib.covspec_sparse_attend(ctypes.byref(p.c_struct()), *args()) == status, (kw, mine)
    p = C.SparseParams(C.AttendParams(**ok), 8, 1, 2)
    need, cs = C.sparse_workspace_size(p), p.c_struct()
    for n in ("q", "start", "length", "pages", "kc", "vc", "summary", "scales", "blocks", "out", "ws"):
        assert lib.covspec_sparse_attend(ctypes.byref(cs), *args(**{n: None})) == Bd.INVALID_ARG, n
    for n, by in (("q", 8), ("out", 8), ("kc", 8), ("ws", 128), ("visible", 4), ("lse", 2), ("summary", 8), ("scales", 2), ("blocks", 2)):
        assert lib.covspec_sparse_attend(ctypes.byref(cs), *args(**{n: FAKE + by})) == Bd.INVALID_ARG, n
    assert lib.covspec_sparse_attend(ctypes.byref(cs), *args(bytes=need - 1)) == Bd.WORKSPACE_TOO_SMALL
    assert lib.covspec_sparse_attend(None, *args()) == Bd.INVALID_ARG
    given = p.c_struct(given=True)
    assert 0 < C.sparse_workspace_size(p, given=True) <= need
    assert lib.covspec_sparse_attend(ctypes.byref(given), *args(blocks=None, summary=None, scales=None)) == Bd.INVALID_ARG
    given.given = 2
    assert lib.covspec_sparse_attend(ctypes.byref(given), *args()) == Bd.INVALID_ARG
    cs = C.SparseParams(C.AttendParams(**{**ok, "cache": _cache(cache_dtype=C.E4M3)}), 8).c_struct()
    assert lib.covspec_sparse_attend(ctypes.byref(cs), *args(vs=None)) == Bd.INVALID_ARG


def test_the_binding_refuses_tensors_that_do_not_fit():
    import torch
    p = _cache(n_seq=1, n_tokens=2, n_pages=2, max_pages=2)
    host, i = torch.zeros(2, 8, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        C.pages_step(C.PagesParams(2, 4, 16, 3, 3), C.pages_alloc(C.PagesParams(2, 4, 16, 3, 3), "cpu"), i, i)
    with pytest.raises(ValueError):
        C.rotate(C.RotaryParams(1, 2, 8, 8, 128), host, host, torch.zeros(64, dtype=torch.int64), i, i[:1])
    with pytest.raises(ValueError):
        C.block_summary(p, i, i[:1], i.view(1, 2), (host, host, None, None), C.block_alloc(p, "cpu"))
    sp = C.SparseParams(C.AttendParams(p, 8, 100, 0.1), 4)
    with pytest.raises(ValueError):
        C.sparse_attend(sp, host, i, i[:1], i.view(1, 2), (host, host, None, None), None)
    with pytest.raises(ValueError):
        C.sparse_attend(sp, host, i, i[:1], i.view(1, 2), (host, host, None, None), None, blocks=i, blocks_out=i)
