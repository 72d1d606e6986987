"""Layer norm of points whose channels are all the same, far from zero, with a small eps: their variance is what rounding leaves, of either
sign, and must not become a root of something negative.

Tolerance (u = 2^-24, n the longest chain of additions over channels, 64 at most).  The mean of equal values v is off by (n / 2 + 2) u v,
which is what the deviations d are; their own mean is off by (n + 2) u d, and rstd is at most 1 / sqrt(eps).  So xh, which is zero, is within
(n + 2) (n / 2 + 2) u^2 v / sqrt(eps), and y within gamma times that of beta, with two roundings of beta."""
import numpy as np
import pytest

from test_gpu_layer_norm import U, Layer


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [1e-5, 1e-12, 1e-30])
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("c", [3, 8, 12, 16, 20, 24, 27, 32, 64, 100, 128, 256, 300, 512, 1000, 1024, 4096, 16384])
def test_equal_channels_far_from_zero(c, layout, eps):
    if layout == "first" and c > 1024:
        c //= 16
    n = Layer(1, c, 1500, layout, "f32", "identity", eps=eps, seed=c)
    rng = np.random.default_rng(c)
    v = (10.0 ** rng.uniform(2, 8, 1500) * rng.choice([-1, 1], 1500)).astype(np.float32)
    n.x[:] = v
    y, (gx, gg, gb) = n.forward(), n.backward()
    chain = min(c, 64)
    most = (chain + 2) * (chain / 2 + 2) * U * U * np.abs(v.astype(np.float64)) / np.sqrt(eps)
    gamma, beta = (np.abs(t.astype(np.float64))[:, None] for t in (n.gamma, n.beta))
    assert np.all(np.abs(y[0] - n.beta[:, None]) <= gamma * most + 2 * U * beta + 1e-30)
    assert np.all(np.isfinite(gg)) and np.all(np.isfinite(gb))
    # gx grows with xh^2 rstd: (n^2 / 2 u^2 v)^2 eps^-1.5 is past the floats with an eps of 1e-30
    assert eps < 1e-20 or np.all(np.isfinite(gx))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("c", [20, 32, 100, 1000])
def test_a_nan_still_stays_with_its_point(c, layout):
    """Beside points of equal channels: what keeps a variance from falling below zero keeps no NaN from the results."""
    n = Layer(1, c, 200, layout, "f32", "identity", eps=1e-12, seed=c)
    n.x[:, :, ::2] = np.float32(1e5) * (1 + np.arange(100, dtype=np.float32))
    n.x[0, 0, 7], n.x[0, c - 1, 8], n.x[0, c // 2, 9] = np.nan, np.inf, -np.inf
    bad = np.isin(np.arange(200), (7, 8, 9))
    for t in (n.forward(), n.backward()[0]):
        assert np.array_equal(np.isnan(t), np.broadcast_to(bad, t.shape))
