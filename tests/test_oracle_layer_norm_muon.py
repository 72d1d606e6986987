"""Pins of the oracle's layer norm and Muon step: other routes to the same numbers, differences, and closed forms."""
import numpy as np
import pytest

from oracle import fno_oracle as O


def _case(seed=0, b=2, c=6, points=5):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((b, c, points)) * 1.3 + 0.4, 1 + 0.3 * rng.standard_normal(c), 0.2 * rng.standard_normal(c), 1e-3,
            rng.standard_normal((b, c, points)))


@pytest.mark.parametrize("act", ["identity", "gelu", "silu"])
def test_layer_norm_is_a_group_norm_of_every_point(act):
    x, ga, be, eps, gy = _case(1)
    rows = lambda t: np.moveaxis(t, 1, 2).reshape(-1, 6, 1)
    y, mean, rstd = O.group_norm_fwd(rows(x), ga, be, 1, eps, act)
    assert np.allclose(rows(O.layer_norm_fwd(x, ga, be, eps, act)), y, rtol=1e-13, atol=1e-14)
    ref = O.group_norm_bwd(rows(x), ga, be, mean, rstd, 1, rows(gy), act)
    got = O.layer_norm_bwd(x, ga, be, eps, gy, act)
    assert np.allclose(rows(got["gx"]), ref["gx"], rtol=1e-12, atol=1e-13)
    assert np.allclose(got["ggamma"], ref["ggamma"]) and np.allclose(got["gbeta"], ref["gbeta"])


@pytest.mark.parametrize("act", ["identity", "gelu", "silu"])
def test_layer_norm_gradients_match_central_differences(act):
    x, ga, be, eps, gy = _case()
    g = O.layer_norm_bwd(x, ga, be, eps, gy, act)

    def loss(x, ga, be):
        return float((gy * O.layer_norm_fwd(x, ga, be, eps, act)).sum())

    h = 1e-5
    for name, t, at in (("gx", x, [(0, 0, 0), (1, 3, 4), (0, 5, 2)]), ("ggamma", ga, [(0,), (4,)]), ("gbeta", be, [(1,), (5,)])):
        for i in at:
            up, down = t.copy(), t.copy()
            up[i] += h
            down[i] -= h
            args = [[(up if s is t else s) for s in (x, ga, be)], [(down if s is t else s) for s in (x, ga, be)]]
            diff = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            assert abs(diff - g[name][i]) < 1e-7 * max(1.0, abs(diff)), (name, i)


def test_layer_norm_closed_forms():
    # two channels: xh = +-1 wherever they lie; one channel: y = act(beta)
    x = np.array([[[3.0, -100.0], [5.0, 100.0]]])
    assert np.allclose(O.layer_norm_fwd(x, [2.0, 1.0], [0.0, 0.5], 0.0, "identity"), [[[-2, -2], [1.5, 1.5]]])
    assert np.allclose(O.layer_norm_fwd(np.full((2, 1, 3), 7.0), [3.0], [-1.0], 1e-5, "silu"), -1 / (1 + np.e))
    x, _, _, _, gy = _case(4)
    gx = O.layer_norm_bwd(x, None, None, 0.0, gy, "gelu")["gx"]
    assert np.allclose(gx.sum(1), 0) and np.allclose((gx * x).sum(1), 0)


def _polynomial(s, iterations, a=3.4445, b=-4.7750, c=2.0315):
    for _ in range(iterations):
        s = a * s + b * s ** 3 + c * s ** 5
    return s


@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (6, 4), (5, 5), (3, 20)])
@pytest.mark.parametrize("kind", ["real", "complex"])
def test_newton_schulz_acts_on_the_singular_values_alone(shape, kind):
    rng = np.random.default_rng(7)
    u = rng.standard_normal((3,) + shape) + (1j * rng.standard_normal((3,) + shape) if kind == "complex" else 0)
    for iterations in (0, 1, 5):
        left, s, right = np.linalg.svd(u, full_matrices=False)
        s = s / (np.sqrt((s ** 2).sum(1, keepdims=True)) + 1e-7)
        ref = (left * _polynomial(s, iterations)[:, None, :]) @ right
        assert np.allclose(O.newton_schulz(u, iterations), ref, rtol=1e-9, atol=1e-11)
    # all singular values of a matrix that is not far from orthogonal end between 0.68 and 1.14
    assert np.all(np.abs(_polynomial(np.linspace(0.1, 1.0, 1000), 5) - 0.91) < 0.24)


def test_newton_schulz_of_nothing_and_of_rank_one():
    assert np.array_equal(O.newton_schulz(np.zeros((2, 3, 4))), np.zeros((2, 3, 4)))
    u = np.outer([1.0, 2, 2], [3.0, 0, 4]) / 15
    assert np.allclose(O.newton_schulz(u, 5, eps=0.0), u * _polynomial(1.0, 5))


def test_muon_step_of_modes_is_that_of_every_matrix():
    rng = np.random.default_rng(2)
    p, g, m = (rng.standard_normal((4, 3, 2, 5)) + 1j * rng.standard_normal((4, 3, 2, 5)) for _ in range(3))
    got_p, got_m = O.muon_step(p, g, m, 0.1, 0.9, scale=1.5, weight_decay=0.2, grad_scale=0.5)
    assert np.allclose(got_m, 0.9 * m + 0.5 * g)
    for k in np.ndindex(2, 5):
        at = (slice(None), slice(None)) + k
        u = 0.5 * g[at] + 0.9 * got_m[at]
        assert np.allclose(got_p[at], p[at] * 0.98 - 0.15 * O.newton_schulz(u))
    real = O.muon_step(p.real[..., 0], g.real[..., 0], m.real[..., 0], 0.1, 0.9, nesterov=False)
    assert np.allclose(real[0][2], p.real[2, ..., 0] - 0.1 * O.newton_schulz(real[1][2]))


@pytest.mark.parametrize("is_complex", [False, True])
def test_tall_matrices_are_wide_ones_transposed(is_complex):
    rng = np.random.default_rng(21)
    u = rng.standard_normal((3, 9, 4)) + (1j * rng.standard_normal((3, 9, 4)) if is_complex else 0)
    x = O.newton_schulz(u)
    assert np.abs(x - np.conj(np.swapaxes(O.newton_schulz(np.conj(np.swapaxes(u, 1, 2))), 1, 2))).max() <= 1e-12
    for k in range(3):                                        # and as the formula has it, with the longer side's Gram matrix
        y = u[k] / (np.linalg.norm(u[k]) + 1e-7)
        for _ in range(5):
            A = y @ y.conj().T
            y = 3.4445 * y + (-4.7750 * A + 2.0315 * A @ A) @ y
        assert np.abs(x[k] - y).max() <= 1e-12
