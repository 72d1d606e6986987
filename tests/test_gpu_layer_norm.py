"""Layer norm with an activation against the float64 oracle: layouts, types, channels and points on either side of every split,
values far from zero, infinities, in place, on a stream of its own, in a graph, and the refusals.

Tolerances, entry by entry, from the arithmetic (u = 2^-24).  With n the longest chain of additions over channels (64 at most),
the mean is off by n u times the mean deviation, which is at most 1 / rstd, and the variance by (n + 2) u of itself; a deviation x - mean
is rounded once, so that with e the error of xh

    e <= u (|xh| (n / 2 + 6) + n + 1 + n^2 u |mean| rstd),

z = gamma xh + beta adds two roundings, the activation is within 1e-6 (absolute) of its definition and has slopes up to 1.13.
The adjoint follows the same chain: the slope within 1e-6, its derivative at most 0.8, h = gamma gz, the two means over channels
off by n u of the mean size of their terms, and rstd by (n / 2 + 4) u.  A gradient of gamma or beta sums its terms' errors, and its
own roundings are at most m u of the terms' sizes, m = 512 being the longest chain of additions in float.  bf16 results: one
more rounding, 2^-8 of the value."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import fno_oracle as O
from paper_2204_01205_amd import binding as B

ACTS = {"identity": B.FNO_ACT_IDENTITY, "gelu": B.FNO_ACT_GELU, "silu": B.FNO_ACT_SILU}
U = 2.0 ** -24


def field(rng, b, c, p, offset=1.0):
    """float32 [b][c][p], every channel with a mean and a scale of its own, representable in bf16."""
    x = rng.standard_normal((b, c, p)) * (0.5 + rng.random((1, c, 1))) + offset * rng.random((1, c, 1))
    return torch.from_numpy(x.astype(np.float32)).bfloat16().float().numpy()


class Layer:
    def __init__(self, b, c, p, layout="first", dtype="f32", act="gelu", eps=1e-5, seed=0, offset=1.0, flags=0):
        rng = np.random.default_rng([seed, b, c, p])
        self.b, self.c, self.p, self.layout, self.act, self.eps = b, c, p, layout, act, eps
        self.torch_dtype = torch.float32 if dtype == "f32" else torch.bfloat16
        self.x, self.gy = field(rng, b, c, p, offset), field(rng, b, c, p, 0.3)
        self.gamma = (1 + 0.3 * rng.standard_normal(c)).astype(np.float32)
        self.beta = (0.3 * rng.standard_normal(c)).astype(np.float32)
        self.desc = B.make_layer_norm_desc(b, c, p, layout=B.FNO_LAYOUT_CHANNELS_FIRST if layout == "first" else B.FNO_LAYOUT_CHANNELS_LAST,
                                           dtype=B.FNO_DTYPE_F32 if dtype == "f32" else B.FNO_DTYPE_BF16, activation=ACTS[act],
                                           eps=eps, flags=flags)

    def dev(self, a):
        t = torch.from_numpy(np.ascontiguousarray(a if self.layout == "first" else a.transpose(0, 2, 1)))
        return t.to(self.torch_dtype).cuda()

    def host(self, t):
        a = t.float().cpu().numpy()
        return a if self.layout == "first" else a.transpose(0, 2, 1)

    def affine(self, on=True):
        return tuple(torch.from_numpy(t).cuda() if on else None for t in (self.gamma, self.beta))

    def forward(self, affine=True):
        x = self.dev(self.x)
        y = torch.empty_like(x)
        B.fno_layer_norm_fwd(self.desc, x, *self.affine(affine), y)
        torch.cuda.synchronize()
        return self.host(y)

    def backward(self, affine=True, start=7.0):
        x, gy, ws = self.dev(self.x), self.dev(self.gy), B.alloc_layer_norm_workspace(self.desc)
        ws.fill_(255)                                    # scratch holds NaN: nothing may be read before it is written
        gx = torch.empty_like(x)
        gg, gb = (torch.full((self.c,), start, device="cuda") for _ in range(2))
        B.fno_layer_norm_bwd(self.desc, x, *self.affine(affine), gy, gx, gg, gb, ws)
        torch.cuda.synchronize()
        return self.host(gx), gg.cpu().numpy(), gb.cpu().numpy()

    def parts(self, affine=True):
        """gamma, beta as [1][C][1], xh, rstd and the error of xh."""
        x = self.x.astype(np.float64)
        mean = x.mean(1, keepdims=True)
        rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + self.eps)
        xh, n = (x - mean) * rstd, min(self.c, 64)
        e = U * (np.abs(xh) * (n / 2 + 6) + n + 1 + n * n * U * np.abs(mean) * rstd)
        ga, be = (t.astype(np.float64)[None, :, None] if affine else d + np.zeros((1, self.c, 1)) for t, d in ((self.gamma, 1.0), (self.beta, 0.0)))
        return ga, be, xh, rstd, e, n

    def rounded(self, ref):
        return 2.0 ** -8 * np.abs(ref) + 2.0 ** -126 if self.torch_dtype == torch.bfloat16 else 0.0

    def check_forward(self, y, affine=True):
        ref = O.layer_norm_fwd(self.x, self.gamma if affine else None, self.beta if affine else None, self.eps, self.act)
        ga, be, xh, _, e, _ = self.parts(affine)
        tol = 1.2e-6 + 1.13 * (np.abs(ga) * e + 2 * U * (np.abs(ga * xh) + np.abs(be)))
        worst = np.abs(y - ref) - tol - self.rounded(ref)
        assert np.all(worst <= 0), (float(worst.max()), float(np.abs(y - ref).max()))

    def check_backward(self, gx, gg, gb, affine=True, start=0.0):
        ref = O.layer_norm_bwd(self.x, self.gamma if affine else None, self.beta if affine else None, self.eps, self.gy, self.act)
        ga, be, xh, rstd, e, n = self.parts(affine)
        gy = np.abs(self.gy.astype(np.float64))
        gz = gy * 1.13
        dz = gy * (1e-6 + 0.8 * (np.abs(ga) * e + 2 * U * (np.abs(ga * xh) + np.abs(be))) + 4 * U * 1.13)
        h, dh = np.abs(ga) * gz, np.abs(ga) * dz
        over = lambda t: t.mean(1, keepdims=True)
        m1, m2 = over(h), over(h * np.abs(xh))
        d1, d2 = over(dh) + n * U * m1, over(dh * np.abs(xh) + h * e) + n * U * m2
        tol = rstd * (dh + d1 + e * m2 + np.abs(xh) * d2 + 4 * U * (h + m1 + np.abs(xh) * m2)) + (n / 2 + 4) * U * np.abs(ref["gx"])
        worst = np.abs(gx - ref["gx"]) - tol - self.rounded(ref["gx"])
        assert np.all(worst <= 0), (float(worst.max()), float(np.abs(gx - ref["gx"]).max()))
        sums = lambda t: t.sum((0, 2))
        for got, name, terms, errors in ((gg, "ggamma", gz * np.abs(xh), dz * np.abs(xh) + gz * e), (gb, "gbeta", gz, dz)):
            bound = sums(errors) + 512 * U * sums(terms) + 4 * U * abs(start) + 1e-30
            worst = np.abs(got - start - ref[name]) - bound
            assert np.all(worst <= 0), (name, float(worst.max()), float(np.abs(got - start - ref[name]).max()))


CHANNELS = [1, 2, 3, 4, 5, 8, 9, 12, 13, 16, 20, 24, 27, 29, 32, 33, 64, 100, 128, 257, 320, 512, 513, 1000, 1024]
POINTS = [1, 7, 64, 65, 255, 257, 1031]


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", CHANNELS)
def test_channels(c, dtype, layout):
    for k, p in enumerate(POINTS if c <= 64 else (1, 66, 263)):
        n = Layer(1 + k % 3, c, p, layout, dtype, ("gelu", "silu", "identity")[(c + k) % 3], seed=c, eps=1e-5 if c > 2 else 1e-2)
        n.check_forward(n.forward())
        n.check_backward(*n.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [1025, 2000, 2048, 3001, 4096, 5003, 8192, 10000, 16383, 16384])
def test_wide_rows(c, dtype):
    n = Layer(2, c, 19, "last", dtype, "silu", seed=c)
    n.check_forward(n.forward())
    n.check_backward(*n.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["identity", "gelu", "silu"])
@pytest.mark.parametrize("layout", ["first", "last"])
def test_many_points(layout, act):
    """More tiles than blocks, so that blocks go over several; whole and odd numbers of points."""
    for b, c, p, dtype in ((1, 20, 262144, "f32"), (2, 12, 142883, "f32"), (3, 27, 40001, "bf16"), (1, 40, 70000, "bf16"), (1, 8, 500001, "f32")):
        n = Layer(b, c, p, layout, dtype, act, seed=3)
        n.check_forward(n.forward())
        n.check_backward(*n.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [13, 15, 16, 17, 19, 20, 21, 22, 24, 25])
def test_channels_of_many_points(c, dtype):
    """Channels first, where a lane takes all channels of a point only with enough points: that many, and one fewer."""
    for b, p in ((1, 2 ** 18), (1, 2 ** 18 - 1), (2, 2 ** 17 + 77)):
        n = Layer(b, c, p, "first", dtype, "identity", seed=c)
        n.check_forward(n.forward())
        n.check_backward(*n.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("layout,c,p,dtype", [("first", 20, 3400003, "f32"), ("first", 8, 8400001, "f32"), ("first", 16, 8500007, "bf16"),
                                              ("first", 64, 1050005, "f32"), ("last", 27, 5000001, "bf16"), ("last", 1024, 132001, "bf16"),
                                              ("last", 300, 224001, "f32")])
def test_fields_beyond_the_caches(layout, c, p, dtype):
    """More than 256 MB: sampled points against the oracle, the gradients of gamma and beta against sums in double over all."""
    n = Layer(1, c, 1, layout, dtype, "identity", seed=15)
    desc = B.make_layer_norm_desc(1, c, p, layout=n.desc.layout, dtype=n.desc.dtype, activation=B.FNO_ACT_IDENTITY)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(c)
    shape = (c, p) if layout == "first" else (p, c)
    x, gy = ((torch.randn(shape, device="cuda", generator=gen) + 0.5).to(n.torch_dtype) for _ in range(2))
    assert x.numel() * x.element_size() > 2 ** 28
    y, gx, ws = torch.empty_like(x), torch.empty_like(x), B.alloc_layer_norm_workspace(desc)
    ws.fill_(255)
    (ga, be), gg, gb = n.affine(), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    B.fno_layer_norm_fwd(desc, x, ga, be, y)
    B.fno_layer_norm_bwd(desc, x, ga, be, gy, gx, gg, gb, ws)
    torch.cuda.synchronize()
    by_point = lambda t: t if layout == "first" else t.t()                      # [c][p]
    at = torch.cat([torch.arange(700), torch.arange(p - 700, p), torch.randint(p, (3000,), generator=torch.Generator().manual_seed(1))]).cuda()
    n.x, n.gy, y, gx = (by_point(t)[:, at].float().cpu().numpy()[None] for t in (x, gy, y, gx))
    n.check_forward(y)
    sums = [torch.zeros(c, dtype=torch.float64, device="cuda") for _ in range(5)]
    for k in range(0, p, 200000):
        v, g = (by_point(t)[:, k:k + 200000].double() for t in (x, gy))
        mean = v.mean(0, keepdim=True)
        rstd = 1.0 / ((v - mean).square().mean(0, keepdim=True) + n.eps).sqrt()
        xh, m = (v - mean) * rstd, min(c, 64)
        e = U * (xh.abs() * (m / 2 + 6) + m + 1 + m * m * U * mean.abs() * rstd)
        for s, t in zip(sums, (g * xh, g, (g * xh).abs(), g.abs(), g.abs() * e)):
            s += t.sum(1)
    wg, wb, tg, tb, errors = (s.cpu().numpy() for s in sums)
    assert np.all(np.abs(gg.cpu().numpy() - wg) <= errors + 516 * U * tg) and np.all(np.abs(gb.cpu().numpy() - wb) <= 516 * U * tb)
    # of the sampled points, gx alone
    ref = O.layer_norm_bwd(n.x, n.gamma, n.beta, n.eps, n.gy, "identity")
    n.check_backward(gx, ref["ggamma"], ref["gbeta"])


@pytest.mark.gpu
@pytest.mark.parametrize("layout,b,c,p", [("first", 2, 20, 55000003), ("first", 3, 100, 7200001), ("last", 2, 27, 40000001), ("last", 1, 1000, 2200003)])
def test_offsets_past_32_bits(layout, b, c, p):
    """More than 2^31 values in bf16: sampled points of every batch entry against the oracle, in place."""
    n = Layer(1, c, 1, layout, "bf16", "gelu", seed=16)
    desc = B.make_layer_norm_desc(b, c, p, layout=n.desc.layout, dtype=n.desc.dtype, activation=B.FNO_ACT_GELU)
    shape = (b, c, p) if layout == "first" else (b, p, c)
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_()
    gy = torch.empty_like(x).normal_()
    assert x.numel() > 2 ** 31
    at = torch.cat([torch.arange(130), torch.arange(p // 2, p // 2 + 130), torch.arange(p - 130, p)]).cuda()
    pick = lambda t: (t[:, :, at] if layout == "first" else t[:, at].transpose(1, 2)).float().cpu().numpy()
    n.x, n.gy, (ga, be) = pick(x), pick(gy), n.affine()
    ws = B.alloc_layer_norm_workspace(desc)
    B.fno_layer_norm_bwd(desc, x, ga, be, gy, gy, None, None, ws)
    B.fno_layer_norm_fwd(desc, x, ga, be, x)
    torch.cuda.synchronize()
    n.check_forward(pick(x))
    ref = O.layer_norm_bwd(n.x, n.gamma, n.beta, n.eps, n.gy, "gelu")
    n.check_backward(pick(gy), ref["ggamma"], ref["gbeta"])


@pytest.mark.gpu
@pytest.mark.parametrize("c,p,layout,dtype", [(20, 777, "first", "f32"), (27, 500, "last", "bf16"), (48, 300, "first", "bf16"), (2048, 40, "last", "f32")])
def test_without_gamma_and_beta(c, p, layout, dtype):
    n = Layer(2, c, p, layout, dtype, "gelu", seed=9)
    n.check_forward(n.forward(affine=False), affine=False)
    n.check_backward(*n.backward(affine=False), affine=False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("b,c,p", [(65535, 8, 1), (65535, 20, 5), (4097, 20, 64), (3000, 40, 65), (700, 300, 3)])
def test_many_batch_entries_of_few_points(b, c, p, layout, dtype):
    n = Layer(b, c, p, layout, dtype, "identity", seed=17)
    n.check_forward(n.forward())
    n.check_backward(*n.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("c,p,layout", [(20, 300, "first"), (100, 70, "first"), (27, 300, "last"), (1000, 20, "last"), (5000, 9, "last")])
@pytest.mark.parametrize("there", ["gamma", "beta"])
def test_gamma_or_beta_alone(c, p, layout, there):
    """The one that is not there stands for ones or zeros."""
    n = Layer(2, c, p, layout, "f32", "gelu", seed=18)
    if there == "gamma":
        n.beta[:] = 0
    else:
        n.gamma[:] = 1
    n.affine = lambda on=True: tuple(torch.from_numpy(t).cuda() if name == there else None for name, t in (("gamma", n.gamma), ("beta", n.beta)))
    n.check_forward(n.forward())
    n.check_backward(*n.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("c,layout", [(20, "first"), (32, "first"), (1000, "first"), (32, "last"), (383, "last"), (16384, "last")])
def test_large_values(c, layout):
    """The largest that the header names: squares of deviations and their sums stay within float."""
    n = Layer(1, c, 70, layout, "f32", "identity", seed=19)
    plain = n.forward()
    size = np.float32(2.0 ** 59 if c <= 32 else 2.0 ** 55) / 2.0 ** np.ceil(np.log2(np.abs(n.x).max()))
    n.x = (n.x * size).astype(np.float32)
    assert np.abs(plain - n.forward()).max() <= 1e-4                # eps is gone beside them


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("c", [20, 100, 700])
def test_points_far_from_zero(layout, c):
    """Means of a thousand and a million beside deviations of about one: what is left of x - mean counts, not the mean."""
    for offset in (1e3, 1e6):
        n = Layer(2, c, 130, layout, "f32", "identity", seed=4)
        n.x = (n.x + np.float32(offset)).astype(np.float32)
        n.check_forward(n.forward())
        n.check_backward(*n.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("c", [20, 100, 700])
def test_one_channel_unlike_the_rest(layout, c):
    """An outlier in any place, the first and the last among them, does not carry its size into the others' errors."""
    for at in (0, 1, c // 2, c - 1):
        n = Layer(1, c, 70, layout, "f32", "identity", seed=5)
        n.x[:, at] = 1e4
        n.check_forward(n.forward())
        n.check_backward(*n.backward())


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("c", [5, 20, 64, 1000])
def test_a_nan_or_an_infinity_stays_with_its_point(layout, c):
    n = Layer(2, c, 140, layout, "f32", "silu", seed=6)
    n.x[0, c // 2, 3], n.x[1, 0, 139], n.x[1, c - 1, 64] = np.nan, np.inf, -np.inf
    y = n.forward()
    gx = n.backward()[0]
    bad = np.zeros((2, 140), bool)
    bad[0, 3] = bad[1, 139] = bad[1, 64] = True
    for t in (y, gx):
        assert np.array_equal(np.isnan(t), np.broadcast_to(bad[:, None], t.shape))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("c", [8, 20, 600])
def test_points_of_equal_channels(layout, c):
    n = Layer(1, c, 50, layout, "f32", "identity", seed=7)
    n.x[:, :, 10:20] = np.float32(0.3)
    y = n.forward()
    # deviations of at most an ulp of 0.3, 2^-25, over sqrt(eps), times gamma, which is below 2.5
    assert np.allclose(y[0, :, 10:20], n.beta[:, None], rtol=1e-6, atol=2.5 * 2.0 ** -25 / np.sqrt(1e-5))
    n.x[:, :, 10:20] = 0.0
    assert np.array_equal(n.forward()[0, :, 10:20], np.broadcast_to(n.beta[:, None], (c, 10)))


@pytest.mark.gpu
@pytest.mark.parametrize("c,p,layout,dtype", [(20, 5001, "first", "f32"), (27, 3001, "last", "bf16"), (300, 500, "first", "f32"), (1500, 60, "last", "bf16")])
def test_in_place(c, p, layout, dtype):
    n = Layer(2, c, p, layout, dtype, "gelu", seed=8)
    apart = n.forward()
    x = n.dev(n.x)
    B.fno_layer_norm_fwd(n.desc, x, *n.affine(), x)
    assert np.array_equal(n.host(x), apart)
    gx = n.backward()[0]
    for over in ("gy", "x"):
        x, gy, ws = n.dev(n.x), n.dev(n.gy), B.alloc_layer_norm_workspace(n.desc)
        out = gy if over == "gy" else x
        gg, gb = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        B.fno_layer_norm_bwd(n.desc, x, *n.affine(), gy, out, gg, gb, ws)
        assert np.array_equal(n.host(out), gx)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("c", [20, 200, 2000])
def test_outputs_that_are_not_asked_for(layout, c):
    if layout == "first" and c > 1024:
        c = 1000
    n = Layer(2, c, 300, layout, "f32", "gelu", seed=10)
    gx, gg, gb = n.backward()
    x, gy, ws = n.dev(n.x), n.dev(n.gy), B.alloc_layer_norm_workspace(n.desc)
    for which in range(1, 8):
        out = torch.full_like(x, 3.0), torch.full((c,), 3.0, device="cuda"), torch.full((c,), 3.0, device="cuda")
        B.fno_layer_norm_bwd(n.desc, x, *n.affine(), gy, *(t if which >> k & 1 else None for k, t in enumerate(out)), ws)
        for k, (t, ref) in enumerate(zip(out, (gx, gg, gb))):
            got = n.host(t) if k == 0 else t.cpu().numpy()
            assert np.array_equal(got, ref) if which >> k & 1 else np.all(got == 3.0), (which, k)


@pytest.mark.gpu
@pytest.mark.parametrize("layout,c", [("first", 20), ("last", 27), ("last", 1200), ("first", 90)])
def test_gradients_that_are_added_to(layout, c):
    n = Layer(2, c, 400, layout, "f32", "silu", seed=11, flags=B.FNO_FLAG_ACCUMULATE_GRADS)
    n.check_backward(*n.backward(start=0.5), start=0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
def test_a_backward_pass_against_differences_of_the_forward_pass(layout):
    n = Layer(2, 12, 90, layout, "f32", "gelu", seed=12)
    gx, gg, gb = n.backward()
    rng, h = np.random.default_rng(0), 2.0 ** -6
    direction = rng.standard_normal(n.x.shape).astype(np.float32)
    base = n.x.copy()

    def loss(step):
        n.x = (base + np.float32(step) * direction).astype(np.float32)
        return float((n.gy.astype(np.float64) * n.forward()).sum())

    # fourth order in h: the rest is h^4 of the fifth derivative, about 1e-7 of 100; rounding of the sums 1e-6 / h
    diff = (8 * (loss(h) - loss(-h)) - (loss(2 * h) - loss(-2 * h))) / (12 * h)
    assert abs(diff - float((gx * direction).sum())) <= 5e-3 * np.abs(gx * direction).sum() / np.sqrt(gx.size) + 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("layout,c,p,dtype", [("first", 20, 20000, "f32"), ("last", 27, 9000, "bf16"), ("last", 1024, 500, "bf16"), ("first", 64, 3000, "f32")])
def test_the_same_bits_on_every_run_and_on_another_stream(layout, c, p, dtype):
    n = Layer(2, c, p, layout, dtype, "gelu", seed=13)
    first = (n.forward(),) + n.backward()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = (n.forward(),) + n.backward()
    for a, b in zip(first, again):
        assert np.array_equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("layout,c,p,dtype", [("first", 20, 20000, "f32"), ("last", 27, 9000, "bf16"), ("last", 1024, 500, "bf16"), ("first", 64, 3000, "f32")])
def test_replays_of_a_graph(layout, c, p, dtype):
    n = Layer(2, c, p, layout, dtype, "gelu", seed=14)
    x, gy, ws, (ga, be) = n.dev(n.x), n.dev(n.gy), B.alloc_layer_norm_workspace(n.desc), n.affine()
    y, gx = torch.empty_like(x), torch.empty_like(x)
    gg, gb = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")

    def both():
        B.fno_layer_norm_fwd(n.desc, x, ga, be, y)
        B.fno_layer_norm_bwd(n.desc, x, ga, be, gy, gx, gg, gb, ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(4):
        x.copy_(n.dev(n.x * (1 + k)))
        both()
        eager = [t.clone() for t in (y, gx, gg, gb)]
        for t in (y, gx, gg, gb):
            t.fill_(-1)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for t, ref in zip((y, gx, gg, gb), eager):
            assert torch.equal(t, ref), k


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
def test_no_points(layout):
    n = Layer(2, 20, 0, layout)
    empty = torch.empty(0, device="cuda")
    B.fno_layer_norm_fwd(n.desc, empty, *n.affine(), empty)
    gx, gg, gb = n.backward()
    assert gx.size == 0 and np.all(gg == 0) and np.all(gb == 0)
    n.desc.flags = B.FNO_FLAG_ACCUMULATE_GRADS
    assert all(np.all(t == 2.5) for t in n.backward(start=2.5)[1:])


@pytest.mark.gpu
@pytest.mark.parametrize("layout,c,p,dtype", [("first", 20, 1031, "f32"), ("first", 9, 517, "bf16"), ("last", 27, 333, "bf16"), ("last", 1500, 7, "f32"), ("first", 77, 131, "bf16")])
def test_nothing_is_written_past_the_end(layout, c, p, dtype):
    n = Layer(1, c, p, layout, dtype, "gelu", seed=15)
    x, gy, ws = n.dev(n.x).reshape(-1), n.dev(n.gy).reshape(-1), B.alloc_layer_norm_workspace(n.desc)
    need = B.fno_layer_norm_workspace_bytes(n.desc)
    guarded = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    out = [torch.full((c * p + 64,), 3.0, device="cuda", dtype=n.torch_dtype) for _ in range(2)]
    small = [torch.full((c + 64,), 3.0, device="cuda") for _ in range(2)]
    B.fno_layer_norm_fwd(n.desc, x, *n.affine(), out[0][: c * p])
    B.fno_layer_norm_bwd(n.desc, x, *n.affine(), gy, out[1][: c * p], small[0][:c], small[1][:c], guarded[:need])
    torch.cuda.synchronize()
    assert all(torch.all(t[c * p:] == 3.0) for t in out) and all(torch.all(t[c:] == 3.0) for t in small)
    assert torch.all(guarded[need:] == 77)


# ------------------------------------------------------------------------------------------ refusals, without a device

def _status(call, desc, *args):
    return getattr(B.lib(), call)(ctypes.byref(desc) if desc is not None else None, *args)


BAD = [(dict(batch=0), B.FNO_EINVAL), (dict(channels=0), B.FNO_EINVAL), (dict(npoints=-1), B.FNO_EINVAL), (dict(layout=2), B.FNO_EINVAL),
       (dict(dtype=2), B.FNO_EINVAL), (dict(activation=3), B.FNO_EINVAL), (dict(flags=1), B.FNO_EINVAL), (dict(eps=-1e-9), B.FNO_EINVAL),
       (dict(eps=float("nan")), B.FNO_EINVAL), (dict(eps=float("inf")), B.FNO_EINVAL), (dict(channels=1025), B.FNO_EUNSUPPORTED),
       (dict(channels=16385, layout=1), B.FNO_EUNSUPPORTED), (dict(batch=65536), B.FNO_EUNSUPPORTED),
       (dict(npoints=2 ** 41), B.FNO_EUNSUPPORTED), (dict(npoints=2 ** 40, channels=20), B.FNO_EUNSUPPORTED)]


@pytest.mark.parametrize("change,status", BAD)
def test_descriptors_that_are_refused(change, status):
    desc = B.make_layer_norm_desc(**{**dict(batch=2, channels=20, npoints=100), **change})
    p, size = 1 << 20, 1 << 40
    n = ctypes.c_size_t(0)
    assert _status("fno_layer_norm_workspace_bytes", desc, ctypes.byref(n)) == status
    assert _status("fno_layer_norm_fwd", desc, p, p, p, p, None) == status
    assert _status("fno_layer_norm_bwd", desc, p, p, p, p, p, p, p, p, size, None) == status


def test_pointers_and_workspaces_that_are_refused():
    desc, p, size = B.make_layer_norm_desc(2, 20, 100), 1 << 20, 1 << 40
    need = B.fno_layer_norm_workspace_bytes(desc)
    fwd = lambda *a: _status("fno_layer_norm_fwd", desc, *a, None)
    bwd = lambda *a: _status("fno_layer_norm_bwd", desc, *a, None)
    assert _status("fno_layer_norm_fwd", None, p, p, p, p, None) == B.FNO_EINVAL
    assert _status("fno_layer_norm_workspace_bytes", desc, None) == B.FNO_EINVAL
    assert fwd(None, p, p, p) == fwd(p, p, p, None) == fwd(p + 4, p, p, p) == fwd(p, p, p, p + 8) == B.FNO_EINVAL
    assert bwd(None, p, p, p, p, p, p, p, size) == bwd(p, p, p, None, p, p, p, p, size) == B.FNO_EINVAL
    assert bwd(p, p, p, p + 4, p, p, p, p, size) == bwd(p, p, p, p, p + 4, p, p, p, size) == B.FNO_EINVAL
    assert bwd(p, p, p, p, p, p, p, None, size) == B.FNO_EINVAL
    assert bwd(p, p, p, p, p, p, p, p + 16, size) == bwd(p, p, p, p, p, p, p, p, need - 1) == B.FNO_ENOSPC
    assert bwd(p, p, p, p, None, None, None, p, size) == B.FNO_OK       # nothing asked for


def test_the_binding_refuses_tensors_that_do_not_fit():
    desc = B.make_layer_norm_desc(1, 4, 8)
    with pytest.raises(ValueError):
        B.fno_layer_norm_fwd(desc, torch.zeros(32), None, None, torch.zeros(32))


@pytest.mark.gpu
def test_the_binding_refuses_wrong_sizes_types_and_strides():
    desc = B.make_layer_norm_desc(1, 4, 8)
    x, v = torch.zeros(1, 4, 8, device="cuda"), torch.zeros(4, device="cuda")
    ws = B.alloc_layer_norm_workspace(desc)
    for bad in (torch.zeros(1, 4, 9, device="cuda"), x.bfloat16(), torch.zeros(8, 4, device="cuda").t(), torch.zeros(1, 4, 8)):
        with pytest.raises(ValueError):
            B.fno_layer_norm_fwd(desc, bad, v, v, x)
        with pytest.raises(ValueError):
            B.fno_layer_norm_fwd(desc, x, v, v, bad)
        with pytest.raises(ValueError):
            B.fno_layer_norm_bwd(desc, x, v, v, bad, x, v, v, ws)
    for bad in (torch.zeros(5, device="cuda"), torch.zeros(4), torch.zeros(4, device="cuda").double()):
        with pytest.raises(ValueError):
            B.fno_layer_norm_fwd(desc, x, bad, v, torch.empty_like(x))
