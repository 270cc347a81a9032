"""How often norm and rotation round in fp32: inputs on which each rounding shows by itself.

x / sqrt(mean(x^2) + eps): with small whole numbers, a power of two of them and eps = 0 the mean is exact, so only the quotient rounds:
half a step, 2^-24 of it (what the two-part reciprocal leaves is below 2^-44).  Cosine and sine: the pair (1, 0) turns into (cos, sin).
Near a quarter or half turn the function is small and its slope 1, so a rounding of the angle there - up to 2^-25 pi = 9.4e-8 of it - would
show beside 4 steps of the function's own value, 2^-21 |value| (its implementation's), and the reference's angles, below 1e-9
(10^6 radians in 64 bits)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import paper_2508_06526_amd as pk  # noqa: E402

DEV = "cuda:0"


@pytest.mark.parametrize("D", [16, 32, 64, 128])
def test_a_normed_value_is_rounded_once(D):
    rng = np.random.default_rng(D)
    x = rng.integers(-40, 41, (300, 3, D)).astype(np.float64)
    w = torch.ones(D, device=DEV)
    out = [torch.zeros((300, h, D), device=DEV) for h in (2, 1)]
    pk.pikv_norm_rope(torch.from_numpy(x).float().to(DEV), 300, 3 * D, 2, 1, D, w, w, 0.0, None, None, 0, False, *out)
    want = x / np.sqrt((x * x).mean(-1, keepdims=True))
    got = torch.cat(out, 1).double().cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -24 * (1 + 2.0 ** -16) * np.abs(want)).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_angle_is_not_rounded(interleaved):
    D, T = 128, 3000
    rng = np.random.default_rng(1)
    positions = rng.integers(0, 10 ** 6, T).astype(np.int32)
    freq = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)
    first = np.arange(D // 2) * (2 if interleaved else 1)
    second = first + (1 if interleaved else D // 2)
    x = torch.zeros((T, 1, D), device=DEV)
    x[:, :, torch.from_numpy(first).to(DEV)] = 1.0
    q = torch.zeros_like(x)
    pk.pikv_norm_rope(x, T, D, 1, 0, D, None, None, 0.0, torch.from_numpy(positions).to(DEV), torch.from_numpy(freq).to(DEV), D, interleaved, q, None)
    got = q[:, 0].double().cpu().numpy()
    angle = positions.astype(np.float64)[:, None] * freq.astype(np.float64)
    cos, sin = np.cos(angle), np.sin(angle)
    for value, mine, near in ((sin, got[:, second], (np.abs(sin) < 2.0 ** -6) & (cos < 0)), (cos, got[:, first], np.abs(cos) < 2.0 ** -6)):
        assert near.sum() > 500
        assert (np.abs(mine - value)[near] <= 2.0 ** -21 * np.abs(value)[near] + 1e-9).all()
