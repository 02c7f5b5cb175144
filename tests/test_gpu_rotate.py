"""GPU parity of covspec_rotate and covspec_rotate_write with oracle/sparse_oracle.py (angles exact, the rest fp64).

Tolerance of an element, with u = half a step of its 16-bit type and X = magnitude (|x1| + |x2|) of its pair: cosine and sine are off by 2^-23 as the
header has it, their products with the magnitude, with x and the sum are four fp32 roundings: E = (2^-23 + 4 2^-24) X; then u |y| for the result's own rounding (of y
off by E: u E more, below 2^-30 X), and 2^-25, half the fixed step of fp16 near zero.  In 8 bits: the scale is off by what the largest element is, E / Q, and two roundings;
a code by half its step (integers 1/2; e4m3 2^-4 of the value, 2^-10 below 2^-6), the value it stands for by E and three roundings of the value more."""
import math

import numpy as np
import pytest

from oracle import sparse_oracle as SO
from round_util import HALF_STEP, Batch, pool_of, rounded, torch_dtype

pytestmark = pytest.mark.gpu

E = 2.0 ** -23 + 4 * 2.0 ** -24
Q = {"int8": 127.0, "e4m3": 448.0}


def steps_of(R, base=10000.0, kind="plain", **kw):
    """Whole numbers for the oracle, and the tensor for the call: the library's own, which a test on the host holds against the formula."""
    import paper_2605_02218_amd as C
    kinds = dict(plain=C.ROTARY_PLAIN, linear=C.ROTARY_LINEAR, base=C.ROTARY_BASE, bands=C.ROTARY_BANDS, ramp=C.ROTARY_RAMP)
    t = C.rotary_steps(R, base, kinds[kind], **kw)
    return [v % (1 << 64) for v in t.tolist()], t


def want_rows(x, positions, steps, interleaved, magnitude):
    """x [T, H, D] fp64, positions [T][R / 2]: turned rows and the magnitudes of their roundings."""
    y, size = np.array(x), np.zeros_like(x)
    for t in range(len(x)):
        if positions[t] is None:
            continue
        for h in range(x.shape[1]):
            y[t, h], size[t, h] = SO.turned(x[t, h], positions[t], steps, interleaved, magnitude)
    return y, size


def near(got, y, size, dtype, where):
    tol = HALF_STEP[dtype] * np.abs(y) + E * (1 + 2.0 ** -8) * size + 2.0 ** -25 * (size > 0)
    err = np.abs(got - y) - tol
    assert np.all(err <= 0), "%s: off by %g beyond the tolerance" % (where, err.max())


def batch_positions(b, half):
    out = [None] * b.T
    for s in range(b.S):
        n = b.new[s]
        for i in range(n):
            out[int(b.start[s]) + i] = [b.length[s] - n + i] * half
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R,heads,H", [(64, 64, 4, 1), (96, 96, 3, 3), (128, 128, 10, 2), (128, 16, 1, 1), (96, 48, 5, 1), (64, 32, 7, 7), (128, 112, 2, 2)])
def test_rows_equal_the_oracle(dtype, interleaved, D, R, heads, H):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(D + R)
    b = Batch(rng, [5, 0, 1, 9, 1], [5, 30, 131072, 1000003, 1], 1024, pad=3)
    steps, t_steps = steps_of(R, 500000.0, "bands", factor=8.0, original=8192, low=1.0, high=4.0)
    (q, q32), (k, k32) = (rounded(rng.standard_normal((b.T, n, D)) * np.exp(rng.standard_normal((b.T, n, 1))), dtype) for n in (heads, H))
    p = C.RotaryParams(b.S, b.T, heads, H, D, R, interleaved, dtype={"bf16": C.BF16, "fp16": C.FP16}[dtype], magnitude=1.25)
    start, length, _ = b.device()
    wide = torch.full((b.T, heads + H + 1, D), 7.0, dtype=torch_dtype(dtype), device="cuda")
    fused = torch.cat([q, k], 1).cuda()
    C.rotate(p, fused[:, :heads], fused[:, heads:], t_steps, start, length, q_out=wide[:, :heads], k_out=wide[:, heads:heads + H])
    torch.cuda.synchronize()
    pos, got = batch_positions(b, R // 2), wide.double().cpu().numpy()
    y, size = want_rows(np.concatenate([q32, k32], 1).astype(np.float64), pos, steps, interleaved, 1.25)
    n = int(b.start[-1])
    near(got[:n, :heads + H], y[:n], size[:n], dtype, "rows")
    assert np.array_equal(got[:n, :heads + H, R:], y[:n, :, R:])                    # what is not turned, to the bit
    assert np.all(got[n:] == 7.0) and np.all(got[:, heads + H:] == 7.0)             # padding, and what lies beside the rows
    # in place, and one of the two alone, gives the same bits
    same = fused.clone()
    C.rotate(p, same[:, :heads], same[:, heads:], t_steps, start, length, q_out=same[:, :heads], k_out=same[:, heads:])
    assert torch.equal(same[:n], wide[:n, :heads + H]) and torch.equal(same[n:], fused[n:])
    q1, none = C.rotate(p, fused[:, :heads], None, t_steps, start, length)
    none2, k1 = C.rotate(p, None, fused[:, heads:], t_steps, start, length)
    assert none is None and none2 is None and torch.equal(q1[:n], wide[:n, :heads]) and torch.equal(k1[:n], wide[:n, heads:heads + H])


@pytest.mark.parametrize("axes", [1, 2, 3, 4])
@pytest.mark.parametrize("with_batch", [False, True])
def test_positions_of_their_own(axes, with_batch):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(axes)
    T, heads, H, D, R = 37, 4, 2, 128, 96
    steps, t_steps = steps_of(R)
    (q, q32), (k, k32) = (rounded(rng.standard_normal((T, n, D)), "bf16") for n in (heads, H))
    positions = rng.choice([0, 1, 77, -5, 4095, -100000, 2 ** 31 - 1, -2 ** 31], (axes, T)).astype(np.int32)
    axis = rng.integers(-2, axes + 2, R // 2).astype(np.int32)                      # a value outside is the nearest axis
    p = C.RotaryParams(2, T, heads, H, D, R, True, axes)
    batch = (torch.tensor([0, 20, 30], dtype=torch.int32, device="cuda"), torch.tensor([20, 10], dtype=torch.int32, device="cuda")) if with_batch else (None, None)
    n = 30 if with_batch else T
    outs = [torch.full((T, m, D), 7.0, dtype=torch.bfloat16, device="cuda") for m in (heads, H)]
    for ax in ([axis] if axes > 1 else [axis, None]):
        a = np.clip(axis, 0, axes - 1) if ax is not None else np.zeros(R // 2, dtype=int)
        C.rotate(p, q.cuda(), k.cuda(), t_steps, *batch, positions=torch.from_numpy(positions).cuda(), axis=None if ax is None else torch.from_numpy(ax).cuda(), q_out=outs[0], k_out=outs[1])
        torch.cuda.synchronize()
        for got, x in zip(outs, (q32, k32)):
            y, size = want_rows(x[:n].astype(np.float64), [[int(positions[a[i], t]) for i in range(R // 2)] for t in range(n)], steps, True, 1.0)
            near(got[:n].double().cpu().numpy(), y, size, "bf16", "axes")
            assert bool((got[n:] == 7.0).all())


def test_the_gradient_is_the_call_with_negated_positions():
    """Of sum w y by x, against differences of the oracle's forward pass: y is linear, so they are exact but for fp64."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(9)
    T, D = 3, 64
    steps, t_steps = steps_of(D)
    positions = rng.integers(0, 1 << 20, T)
    w, w32 = rounded(rng.standard_normal((T, 1, D)), "bf16")
    p = C.RotaryParams(1, T, 1, 1, D, magnitude=1.5)
    got, _ = C.rotate(p, w.cuda(), None, t_steps, positions=torch.from_numpy(-positions.astype(np.int32)).cuda().view(1, T))
    x = rng.standard_normal((T, D))
    f = lambda x, t: float((SO.turned(x, [int(positions[t])] * (D // 2), steps, False, 1.5)[0] * w32[t, 0].astype(np.float64)).sum())        # noqa: E731
    for t in range(T):
        _, size = SO.turned(w32[t, 0].astype(np.float64), [0] * (D // 2), steps, False, 1.5)
        for d in range(0, D, 5):
            h = np.zeros(D)
            h[d] = 0.5
            slope = f(x[t] + h, t) - f(x[t] - h, t)
            assert abs(float(got[t, 0, d]) - slope) <= HALF_STEP["bf16"] * abs(slope) + E * 1.01 * size[d] + 1e-12


def test_angles_over_the_whole_range_of_positions():
    """Cosine and sine themselves: rows of (1, 0), fp16 outputs of both signs, positions from one to 2^31 - 1."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(2)
    D, T = 128, 400
    steps, t_steps = steps_of(D, 1e6)
    positions = np.unique(np.concatenate([np.arange(130), (2.0 ** rng.uniform(0, 31, T)).astype(np.int64), [2 ** 31 - 1]]))[:T]
    positions = np.concatenate([positions, [2 ** 31 - 1] * (T - len(positions))])
    x = torch.zeros(T, 1, D, dtype=torch.float16)
    x[..., :D // 2] = 1.0
    got, _ = C.rotate(C.RotaryParams(1, T, 1, 1, D, dtype=C.FP16), x.cuda(), None, t_steps, positions=torch.from_numpy(positions.astype(np.int32)).cuda().view(1, T))
    got = got.double().cpu().numpy()[:, 0]
    for t in range(T):
        for i in range(D // 2):
            c, s = SO.cos_sin(positions[t], steps[i])
            for v, w in ((got[t, i], c), (got[t, i + D // 2], s)):
                assert abs(v - w) <= 2.0 ** -11 * abs(w) + E + 2.0 ** -25


KINDS = [("bf16", "bf16"), ("bf16", "int8"), ("bf16", "e4m3"), ("fp16", "fp16"), ("fp16", "int8"), ("fp16", "e4m3")]


@pytest.mark.parametrize("dtype,kept", KINDS)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R,heads,H,page", [(64, 64, 8, 2, 16), (96, 32, 2, 2, 32), (128, 128, 8, 8, 64), (128, 48, 5, 1, 1024)])
def test_written_rows(dtype, kept, interleaved, D, R, heads, H, page):
    """The whole pool: 16 bits what rotating and writing leave, to the bit; codes against the oracle; v and places beside the rows to the bit."""
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(D * 3 + R)
    b = Batch(rng, [5, 0, 1, 40, 3], [5, 30, 77, 131, 2], page, pad=3)              # a row in front of the last sequence
    steps, t_steps = steps_of(R)
    wide, w32 = rounded(rng.standard_normal((b.T, heads + 2 * H, D)) * np.exp(rng.standard_normal((b.T, heads + 2 * H, 1))), dtype)
    wide[0, heads], wide[1, heads, 3], wide[2, heads + H, 5], wide[3, heads, 1] = 0.0, float("inf"), float("nan"), -float("inf")
    w32 = wide.float().numpy()
    wide = wide.cuda()
    q, k, v = wide[:, :heads], wide[:, heads:heads + H], wide[:, heads + H:]
    cp = b.params(H, D, dtype, kept)
    p = C.RotaryParams(b.S, b.T, heads, H, D, R, interleaved, dtype=cp.dtype)
    pools = [C.cache_alloc(cp) for _ in range(2)]
    for pool in pools:
        for t in pool:
            if t is not None:
                t.view(torch.uint8).fill_(0x5A)
    start, length, pages = b.device()
    q_out = torch.full((b.T, heads, D), 7.0, dtype=torch_dtype(dtype), device="cuda")
    C.rotate_write(p, cp, q, k, v, t_steps, start, length, pages, pools[0], q_out=q_out)
    q2, k2 = C.rotate(p, q, k, t_steps, start, length)
    C.cache_write(cp, k2, v.contiguous(), start, length, pages, pools[1])
    torch.cuda.synchronize()
    n = int(b.start[-1])
    assert torch.equal(q_out[:n], q2[:n]) and bool((q_out[n:] == 7.0).all())
    raw = lambda t: t.contiguous().view(torch.uint8)        # noqa: E731
    if kept == dtype:
        assert torch.equal(raw(pools[0][0]), raw(pools[1][0]))
    assert torch.equal(raw(pools[0][1]), raw(pools[1][1]))
    if kept != dtype:
        assert torch.equal(raw(pools[0][3]), raw(pools[1][3]))
        pos = batch_positions(b, R // 2)
        codes, scales = pools[0][0].float().cpu().numpy().astype(np.float64), pools[0][2].cpu().numpy().astype(np.float64)
        touched = np.zeros(codes.shape[:3], dtype=bool)
        for t, at in enumerate(b.places()):
            if at is None or at == "padding":
                continue
            for h in range(H):
                touched[at[0], h, at[1]] = True
                c, sc, x = codes[at[0], h, at[1]], scales[at[0], h, at[1]], w32[t, heads + h].astype(np.float64)
                if not np.isfinite(x).all():
                    assert math.isnan(sc) and not c.any()
                    continue
                y, size = SO.turned(x, pos[t], steps, interleaved)
                top, worst = np.abs(y).max(), E * size.max()
                assert abs(sc - top / Q[kept]) <= (worst + 2 * 2.0 ** -24 * top) / Q[kept]
                if top == 0:
                    assert sc == 0 and not c.any()
                    continue
                value = c * sc
                half = 0.5 if kept == "int8" else np.maximum(2.0 ** -4 * np.abs(y) / sc, 2.0 ** -10)
                tol = sc * half * (1 + 2.0 ** -20) + 2 * worst + 4 * 2.0 ** -24 * np.abs(y)
                assert np.all(np.abs(value - y) <= tol), (t, h)
        assert bool((raw(pools[0][0]).view(*codes.shape).cpu()[torch.from_numpy(~touched)] == 0x5A).all())


def test_many_tokens_and_heads():
    """Lanes that take several heads each, against lanes with one: the same bits as tokens on their own."""
    import torch
    import paper_2605_02218_amd as C
    g = torch.Generator(device="cuda").manual_seed(3)
    T, heads, H, D = 9000, 40, 8, 128
    x = torch.randn(T, heads + 2 * H, D, generator=g, device="cuda").to(torch.bfloat16)
    steps = C.rotary_steps(D)
    start, length = torch.tensor([0, 4000, T], dtype=torch.int32, device="cuda"), torch.tensor([4000, 5007], dtype=torch.int32, device="cuda")
    q, k = C.rotate(C.RotaryParams(2, T, heads, H, D), x[:, :heads], x[:, heads:heads + H], steps, start, length)
    pos = torch.cat([torch.arange(4000), torch.arange(7, 5007)]).to(torch.int32).cuda()
    for t in (0, 1, 3999, 4000, 8999):
        q1, k1 = C.rotate(C.RotaryParams(1, 1, heads, H, D), x[t:t + 1, :heads], x[t:t + 1, heads:heads + H], steps, positions=pos[t:t + 1].view(1, 1))
        assert torch.equal(q1[0], q[t]) and torch.equal(k1[0], k[t])
    for kept in (C.BF16, C.E4M3):
        cp = C.CacheParams(2, T, H, D, 64, 200, 100, C.BF16, kept)
        pages = torch.arange(200, dtype=torch.int32, device="cuda").view(2, 100)
        pool = C.cache_alloc(cp)
        q2 = C.rotate_write(C.RotaryParams(2, T, heads, H, D), cp, x[:, :heads], x[:, heads:heads + H], x[:, heads + H:], steps, start, length, pages, pool)
        assert torch.equal(q2, q)
        k3, v3 = C.cache_read(cp, pool, start, length, pages)
        if kept == C.BF16:
            assert torch.equal(k3, k) and torch.equal(v3, x[:, heads + H:])
        else:
            # |k3 - k| <= |k3 - z| + |z - y| + |y - k|: y the turned value in fp32, z = code scale.  |z - y| is half a step of e4m3, 2^-4 |y|, or 2^-10 scale below
            # 2^-6 scale, scale = amax / 448: 2^-18 amax; the other two are the roundings to bf16, 2^-8 |z| and 2^-8 |y| with |z| <= (1 + 2^-4) |y| + 2^-18 amax,
            # |y| <= |k| / (1 - 2^-8); amax of y is at most 1 / (1 - 2^-8) of that of k; what fp32 adds is below 2^-18 of both.
            y, amax = k.float().abs() / (1 - 2.0 ** -8), k.float().abs().amax(-1, keepdim=True) / (1 - 2.0 ** -8)
            tol = (2.0 ** -4 + 2.0 ** -8 * (2 + 2.0 ** -4) + 2.0 ** -18) * y + (2.0 ** -18 * (1 + 2.0 ** -8) + 2.0 ** -18) * amax
            assert bool(((k3.float() - k.float()).abs() <= tol).all())
