"""Pins of the oracle's group norm, AdamW and 8-bit moments: closed forms, differences, and counts that do not go through
the formulas they check."""
import numpy as np
import pytest

from oracle import fno_oracle as O


def _case(act, seed=0, b=2, c=6, groups=3, points=5):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((b, c, points)) * 1.3 + 0.4, 1 + 0.3 * rng.standard_normal(c), 0.2 * rng.standard_normal(c), groups,
            1e-3, act, rng.standard_normal((b, c, points)))


@pytest.mark.parametrize("act", ["identity", "gelu", "silu"])
def test_group_norm_gradients_match_central_differences(act):
    x, ga, be, groups, eps, act, gy = _case(act)
    _, mean, rstd = O.group_norm_fwd(x, ga, be, groups, eps, act)
    g = O.group_norm_bwd(x, ga, be, mean, rstd, groups, gy, act)

    def loss(x, ga, be):
        return float((gy * O.group_norm_fwd(x, ga, be, groups, eps, act)[0]).sum())

    h = 1e-5
    for name, t, at in (("gx", x, [(0, 0, 0), (1, 3, 4), (0, 5, 2)]), ("ggamma", ga, [(0,), (4,)]), ("gbeta", be, [(1,), (5,)])):
        for i in at:
            up, down = t.copy(), t.copy()
            up[i] += h
            down[i] -= h
            args = [[(up if s is t else s) for s in (x, ga, be)], [(down if s is t else s) for s in (x, ga, be)]]
            diff = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            assert abs(diff - g[name][i]) < 1e-7 * max(1.0, abs(diff)), (name, i)


def test_group_norm_closed_forms():
    # two values per group: xh = +-1 for eps = 0; the second group's are far apart, which changes nothing
    x = np.array([[[3.0], [5.0], [-100.0], [100.0]]])
    y, mean, rstd = O.group_norm_fwd(x, None, None, 2, 0.0, "identity")
    assert np.allclose(y.ravel(), [-1, 1, -1, 1]) and np.allclose(mean, [[4, 0]]) and np.allclose(rstd, [[1, 0.01]])
    # a constant group: xh = 0, so y = act(beta), and its gradient through x is rstd (gz - mean gz)
    x = np.full((1, 2, 3), 7.0)
    y, mean, rstd = O.group_norm_fwd(x, [2.0, 3.0], [0.5, -1.0], 1, 1e-4, "silu")
    assert np.allclose(y[0, 0], 0.5 / (1 + np.exp(-0.5))) and np.allclose(y[0, 1], -1 / (1 + np.e)) and np.allclose(rstd, 100)
    g = O.group_norm_bwd(x, None, None, mean, rstd, 1, np.arange(6.0).reshape(1, 2, 3), "identity")
    assert np.allclose(g["gx"].ravel(), 100 * (np.arange(6) - 2.5)) and np.allclose(g["ggamma"], 0) and np.allclose(g["gbeta"], [3, 12])
    # adding a constant or scaling changes nothing but the statistics (eps = 0); groups of one channel see only their own
    rng = np.random.default_rng(3)
    x = rng.standard_normal((2, 4, 9))
    base = O.group_norm_fwd(x, None, None, 4, 0.0, "gelu")[0]
    moved = O.group_norm_fwd(x * np.array([1.0, 2, 3, 4])[None, :, None] + 5, None, None, 4, 0.0, "gelu")[0]
    assert np.allclose(base, moved)


def test_group_norm_gradient_is_orthogonal_to_shift_and_scale():
    x, ga, be, groups, _, act, gy = _case("gelu", 4)
    _, mean, rstd = O.group_norm_fwd(x, ga, be, groups, 0.0, act)
    gx = O.group_norm_bwd(x, ga, be, mean, rstd, groups, gy, act)["gx"].reshape(2, groups, -1)
    xg = x.reshape(2, groups, -1)
    assert np.allclose(gx.sum(2), 0) and np.allclose((gx * xg).sum(2), 0)


def test_silu_values():
    assert np.allclose(O.silu([0.0, 1.0, -1.0]), [0, 1 / (1 + np.exp(-1)), -1 / (1 + np.e)])
    assert O.silu(-1000.0) == 0.0 and O.silu(1000.0) == 1000.0
    z = np.linspace(-6, 6, 25)
    assert np.allclose(O.silu_prime(z), (O.silu(z + 1e-6) - O.silu(z - 1e-6)) / 2e-6, atol=1e-8)


def test_adamw_first_step_and_decay():
    # first step from zero moments: the move is lr sign(g), whatever the gradient's size; the decay is apart from it
    p, m, v = O.adamw_step([2.0, -2.0, 1.0], [1e-3, -5.0, 0.0], [0, 0, 0], [0, 0, 0], 1, lr=0.1, eps=0.0 + 1e-30, weight_decay=0.5)
    assert np.allclose(p, [2 - 0.1 - 0.1, -2 + 0.1 + 0.1, 1 - 0.05]) and np.allclose(m, [1e-4, -0.5, 0]) and np.allclose(v, [1e-9, 0.025, 0])
    q, _, _ = O.adamw_step([2.0], [4.0], [0.5], [0.25], 7, weight_decay=0.0, scale=0.25)
    r, _, _ = O.adam_step([2.0], [1.0], [0.5], [0.25], 7)
    assert q == r


@pytest.mark.parametrize("which", ["m", "v"])
def test_every_code_is_read_and_written_back(which):
    last = 127 if which == "m" else 255
    codes = np.concatenate([np.arange(last + 1), last - np.arange(O.CODE_BLOCK - last - 1)]).astype(np.uint8)
    vals = O.code_values(codes, [130], which)
    assert vals[0] == 0 and np.all(np.diff(vals[: last + 1]) > 0) and vals[last] == 1.875 * 8.0
    back, e = O.encode_moment(vals, np.full(vals.size, 0), which)
    assert e[0] == 130 and np.array_equal(back, codes)
    back, _ = O.encode_moment(vals, np.full(vals.size, 65535), which)
    assert np.array_equal(back, codes)                   # what a code stands for is never moved
    assert np.array_equal(vals.astype(np.float32).view(np.uint32) & 0xFFFF, np.zeros(vals.size))   # bf16 values
    if which == "m":
        neg, _ = O.encode_moment(-vals, np.full(vals.size, 9), which)
        assert np.array_equal(neg[1:] % 128, codes[1:]) and np.array_equal(O.code_values(neg, [130], "m"), -vals)


def test_random_rounding_keeps_the_mean_and_nearest_would_not():
    n, steps = 2560, 400
    v = np.full(n, 0.7)
    codes, e = O.encode_moment(v, O.code_bits(n, 5, 0, 0) >> 16, "v")
    for t in range(1, steps + 1):
        new = 0.999 * O.code_values(codes, e, "v")
        codes, e = O.encode_moment(new, O.code_bits(n, 5, t, 0) >> 16, "v")
    mean = O.code_values(codes, e, "v").mean()
    # a value moves by up to an eighth of a power of two a time: about 0.05 after 400 steps for one, 0.001 for the mean
    assert abs(mean - 0.7 * 0.999 ** steps) < 0.01
    held = O.code_values([200], [127], "v")              # to nearest (a half for the random part) it stays for ever
    assert O.code_values(*O.encode_moment(0.999 * held, np.array([32768]), "v"), "v") == held


def test_small_values_of_a_block():
    x = np.zeros(256)
    x[0], x[1], x[2], x[3] = 1.0, 1e-12, -3e-5, 2.0 ** -15
    codes, e = O.encode_moment(np.abs(x), np.zeros(256, int), "v")
    assert e[0] == 127 and codes[1] == 1 and codes[4] == 0          # v: what is not zero stays
    up, _ = O.encode_moment(x, np.zeros(256, int), "m")
    down, _ = O.encode_moment(x, np.full(256, 65535), "m")
    assert up[2] == 129 and down[2] == 128 and up[4] == down[4] == 0          # m: rounded to zero or the smallest code
    assert np.isnan(O.code_values(*O.encode_moment(np.where(np.arange(256) == 9, np.nan, x), np.zeros(256, int), "m"), "m")).all()
    assert np.isnan(O.code_values(*O.encode_moment(np.where(np.arange(256) == 9, np.inf, 1.0), np.zeros(256, int), "v"), "v")).all()


def test_random_bits_look_uniform_and_differ():
    r = O.code_bits(4096, 1, 2, 3)
    assert r.min() >= 0 and r.max() < 2 ** 32
    for half in (r & 0xFFFF, r >> 16):
        assert abs(half.mean() / 65536 - 0.5) < 0.02
    assert abs(np.corrcoef(r & 0xFFFF, r >> 16)[0, 1]) < 0.06
    for other in (O.code_bits(4096, 2, 2, 3), O.code_bits(4096, 1, 3, 3), O.code_bits(4096, 1, 2, 4)):
        assert (other == r).mean() < 0.01
