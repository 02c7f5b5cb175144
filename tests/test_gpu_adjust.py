"""GPU parity of covspec_adjust_logits with oracle/round_oracle.py (fp64).

Tolerance: half a step of the output's type, plus eight fp32 roundings (1 / r, 1 / T, product, product, two sums, sum, product) of at most 2^-24 of the
largest magnitude they are taken of, which the oracle returns.  Masked words are exactly -infinity.
"""
import numpy as np
import pytest

from oracle import round_oracle as RO

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -134, "fp16": 2.0 ** -25, "fp32": 2.0 ** -150}


def case(S, L, V, dtype, seed, history=200, prompts=True, drafted=True, biased=20, masked=True, stray=True, in_place=False, inf=False):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(seed)
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[dtype]
    z = torch.from_numpy((rng.standard_normal((S, L, V)) * 3).astype(np.float32)).to(dt)
    if inf:
        z[..., 1], z[..., 2], z[..., 3] = -float("inf"), float("inf"), torch.finfo(dt).min / 4
    counts = [0] + [int(x) for x in rng.integers(0, history + 1, S - 1)] if S > 1 else [history]
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    lo, hi = (-5, V + 5) if stray else (0, V)
    words = np.where(rng.random(start[-1]) < 0.5, rng.integers(0, 12, start[-1]), rng.integers(lo, hi, start[-1])).astype(np.int32)
    prompt = rng.integers(0, history // 2 + 1, S).astype(np.int32) if prompts else None
    d = np.where(rng.random((S, L)) < 0.6, rng.integers(0, 12, (S, L)), rng.integers(lo, hi, (S, L))).astype(np.int32) if drafted else None
    pen = np.stack([1 + rng.random(S), rng.random(S) - 0.3, 0.5 * rng.random(S), 0.4 + rng.random(S)], 1).astype(np.float32)
    pen[0] = (1, 0, 0, 1)
    if S > 1:
        pen[1, 3] = 0.0
    bias = None
    if biased:
        bs = np.arange(0, S * biased + 1, biased).astype(np.int32)
        bw = rng.integers(lo, min(hi, 60), S * biased).astype(np.int32)            # some words more than once: the last counts
        bv = (rng.standard_normal(S * biased) * 4).astype(np.float32)
        bias = (bs, bw, bv)
    bits = rng.integers(0, 1 << 32, (S, L, (V + 31) // 32), dtype=np.uint64).astype(np.uint32) if masked else None
    if masked:
        bits[0, 0] = 0                                                             # a state in which nothing is allowed
    dev = lambda a: None if a is None else torch.from_numpy(a.view(np.int32) if a.dtype == np.uint32 else a).cuda()  # noqa: E731
    p = C.LogitsParams(S, L, V, {"bf16": C.BF16, "fp16": C.FP16, "fp32": C.FP32}[dtype])
    zd = z.cuda()
    args = dict(prompt_len=dev(prompt), drafted=dev(d), bias=None if bias is None else tuple(dev(x) for x in bias), allowed=dev(bits))
    out = C.adjust_logits(p, zd, dev(words), dev(start), dev(pen), out=zd if in_place else None, **args)
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(zd.view(torch.uint8).cpu(), z.view(torch.uint8))
    got, z64 = out.float().cpu().numpy().astype(np.float64), z.double().numpy()
    for s in range(S):
        w = words[start[s]:start[s + 1]]
        cut = int(prompt[s]) if prompts else 0
        b = {}
        if bias is not None:
            for x, y in zip(bias[1][s * biased:(s + 1) * biased], bias[2][s * biased:(s + 1) * biased]):
                b[int(x)] = float(y)
        for t in range(L):
            ok = None
            if masked:
                i = np.arange(V)
                ok = (bits[s, t, i // 32] >> (i % 32).astype(np.uint32) & 1).astype(bool)
            with np.errstate(invalid="ignore"):
                x, size = RO.adjust_row(z64[s, t], w[:cut], list(w[cut:]) + (list(d[s, :t]) if drafted else []), pen[s], b, ok)
            inf_ = ~np.isfinite(x)
            np.testing.assert_array_equal(got[s, t][inf_], x[inf_])
            err = np.abs(got[s, t][~inf_] - x[~inf_])
            tol = HALF[dtype] * np.abs(x[~inf_]) + 8 * 2.0 ** -24 * size[~inf_] + TINY[dtype]
            assert np.all(err <= tol), (s, t, (err - tol).max())
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("S,L,V", [(1, 1, 8), (1, 5, 4096), (3, 8, 4104), (5, 2, 20008), (2, 64, 520)])
def test_adjusted_logits_equal_the_oracle(dtype, S, L, V):
    case(S, L, V, dtype, seed=S * 100 + L)


@pytest.mark.parametrize("kw", [dict(masked=False), dict(biased=0), dict(prompts=False), dict(drafted=False), dict(history=0), dict(in_place=True), dict(inf=True),
                                dict(history=9000, biased=700), dict(masked=False, biased=0, drafted=False, prompts=False)])
def test_parts_that_are_left_out(kw):
    case(3, 4, 8200, "bf16", seed=9, **kw)
    case(2, 3, 4100, "fp32", seed=10, **kw)


def test_nothing_to_do_changes_no_bit():
    import torch
    import paper_2605_02218_amd as C
    z = torch.randn(2, 3, 4096, device="cuda").to(torch.bfloat16)
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    pen = torch.tensor([[1.0, 0, 0, 1]] * 2, device="cuda")
    out = C.adjust_logits(C.LogitsParams(2, 3, 4096), z, none[:0], none, pen)
    assert torch.equal(out, z)


def test_a_captured_call_serves_other_histories():
    import torch
    import paper_2605_02218_amd as C
    S, L, V = 2, 3, 8192
    p = C.LogitsParams(S, L, V)
    z = torch.randn(S, L, V, device="cuda").to(torch.bfloat16)
    words = torch.randint(0, V, (500,), device="cuda", dtype=torch.int32)
    start = torch.tensor([0, 100, 300], dtype=torch.int32, device="cuda")
    drafted = torch.randint(0, V, (S, L), device="cuda", dtype=torch.int32)
    pen = torch.tensor([[1.2, 0.3, 0.1, 0.8]] * S, device="cuda")
    out = torch.empty_like(z)
    C.adjust_logits(p, z, words, start, pen, drafted=drafted, out=out)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            C.adjust_logits(p, z, words, start, pen, drafted=drafted, out=out)
    for ends in ([0, 100, 300], [0, 0, 500], [0, 250, 250]):
        start.copy_(torch.tensor(ends, dtype=torch.int32))
        words.random_(0, V)
        z.normal_()
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, C.adjust_logits(p, z, words, start, pen, drafted=drafted))
