"""What covspec_rotate is with positions negated: with the same magnitude twice the rotation's rows are magnitude^2 of what they were, with its reciprocal they are as before.

Tolerance, u and E as in test_gpu_rotate: the first call leaves each of a pair's y off by e = u |y| + E m (|x1| + |x2|) + 2^-25; the second, of magnitude m', m' (e1 + e2) from those
(a turn adds each at most once), then u |z| + E m' (|y1| + |y2|) + 2^-25 of its own, 1 % for e in |y| and |z|, and 2^-23 for m' itself."""
import numpy as np
import pytest

from round_util import HALF_STEP, rounded
from test_gpu_rotate import E, steps_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("magnitude", [1.0, 1.2772589, 0.3])
def test_negated_positions_with_the_same_magnitude_and_its_reciprocal(dtype, interleaved, magnitude):
    import torch
    import paper_2605_02218_amd as C
    rng = np.random.default_rng(17)
    T, D, R, u = 40, 128, 96, HALF_STEP[dtype]
    x, x32 = rounded(rng.standard_normal((T, 2, D)), dtype)
    _, steps = steps_of(R)
    positions = torch.from_numpy(rng.integers(-2 ** 31 + 1, 2 ** 31, (1, T)).astype(np.int32)).cuda()
    params = lambda m: C.RotaryParams(1, T, 2, 1, D, R, interleaved, dtype={"bf16": C.BF16, "fp16": C.FP16}[dtype], magnitude=m)        # noqa: E731
    y, _ = C.rotate(params(magnitude), x.cuda(), None, steps, positions=positions)
    i = np.arange(R // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    x64, y64, m = x32.astype(np.float64), y.double().cpu().numpy(), magnitude
    pair = lambda v: np.abs(v[..., a]) + np.abs(v[..., b])        # noqa: E731
    both = u * pair(y64) + 2 * (E * m * pair(x64) + 2.0 ** -25)
    for other in (m, 1.0 / m):
        z, _ = C.rotate(params(other), y, None, steps, positions=-positions)
        z64 = z.double().cpu().numpy()
        for at in (a, b):
            want = x64[..., at] * (m * other)
            tol = 1.01 * (other * both + u * np.abs(want) + E * other * pair(y64)) + 2.0 ** -23 * np.abs(want) + 2.0 ** -25
            assert np.all(np.abs(z64[..., at] - want) <= tol)
        assert np.array_equal(z64[..., R:], x64[..., R:])
