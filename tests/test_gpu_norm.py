"""Group norm with an activation against the float64 oracle: layouts, types, sizes on either side of every split, empty and
constant groups, infinities, in place, on a stream of its own, in a graph, and the refusals.

Tolerances, entry by entry, from the arithmetic (u = 2^-24).  Forward: x - mean is exact to u |x - mean|, three roundings up
to z, the activation within 1e-6 (absolute) of its definition: 1.2e-6 + 6 u (|gamma xh| + |beta|), slopes being at most
1.13.  bf16 results: one more rounding, 2^-8 of the value (8 significant bits).  Backward: xh is off by 3 u |xh| + u |mean| rstd (the saved mean is a
float), the slope by 1e-6, and its derivative is at most 0.8; with every factor's error next to the terms of
gx = rstd (gamma gz - m1 - xh m2): the sum of the terms' sizes, with gy in gz's place, times 2e-6 plus the mean's rounding.
Sums are in double from products of floats: their error is at most that of their terms."""
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


class Norm:
    def __init__(self, b, c, groups, p, layout="first", dtype="f32", act="gelu", eps=1e-5, seed=0, offset=1.0, flags=0):
        rng = np.random.default_rng([seed, b, c, groups, p])
        self.b, self.c, self.groups, self.p, self.layout, self.act, self.eps = b, c, groups, p, layout, act, eps
        self.torch_dtype = torch.float32 if dtype == "f32" else torch.bfloat16
        self.x, self.gy = field(rng, b, c, p, offset), field(rng, b, c, p, 0.3)
        self.gamma = (1 + 0.3 * rng.standard_normal(c)).astype(np.float32)
        self.beta = (0.3 * rng.standard_normal(c)).astype(np.float32)
        self.desc = B.make_norm_desc(b, c, groups, p,
                                     layout=B.FNO_LAYOUT_CHANNELS_FIRST if layout == "first" else B.FNO_LAYOUT_CHANNELS_LAST,
                                     dtype=B.FNO_DTYPE_F32 if dtype == "f32" else B.FNO_DTYPE_BF16, activation=ACTS[act], eps=eps,
                                     flags=flags)

    def dev(self, a):
        t = torch.from_numpy(np.ascontiguousarray(a if self.layout == "first" else a.transpose(0, 2, 1)))
        return t.to(self.torch_dtype).cuda()

    def host(self, t):
        a = t.float().cpu().numpy()
        return a if self.layout == "first" else a.transpose(0, 2, 1)

    def stats(self):
        return torch.empty(self.b, self.groups, device="cuda"), torch.empty(self.b, self.groups, device="cuda")

    def forward(self, affine=True):
        x, ws = self.dev(self.x), B.alloc_norm_workspace(self.desc)
        y, (mean, rstd) = torch.empty_like(x), self.stats()
        ga, be = (torch.from_numpy(t).cuda() if affine else None for t in (self.gamma, self.beta))
        B.fno_group_norm_fwd(self.desc, x, ga, be, y, mean, rstd, ws)
        torch.cuda.synchronize()
        return self.host(y), mean.cpu().numpy(), rstd.cpu().numpy()

    def backward(self, mean, rstd, affine=True, start=None):
        x, gy, ws = self.dev(self.x), self.dev(self.gy), B.alloc_norm_workspace(self.desc)
        gx = torch.empty_like(x)
        gg, gb = (torch.full((self.c,), 7.0 if start is None else start, device="cuda") for _ in range(2))
        ga, be = (torch.from_numpy(t).cuda() if affine else None for t in (self.gamma, self.beta))
        B.fno_group_norm_bwd(self.desc, x, ga, be, torch.from_numpy(mean).cuda(), torch.from_numpy(rstd).cuda(), gy, gx, gg, gb, ws)
        torch.cuda.synchronize()
        return self.host(gx), gg.cpu().numpy(), gb.cpu().numpy()

    def check_forward(self, y, mean, rstd, affine=True):
        ga, be = (self.gamma, self.beta) if affine else (None, None)
        ry, rm, rr = O.group_norm_fwd(self.x, ga, be, self.groups, self.eps, self.act)
        scale = np.sqrt(1.0 / rr ** 2)                   # sqrt(var + eps)
        assert np.all(np.abs(mean - rm) <= 2 * U * np.abs(rm) + 1e-9 * scale)
        assert np.all(np.abs(rstd - rr) <= 4 * U * rr)
        d = self.c // self.groups
        per = lambda t: np.repeat(t, d, axis=1)[:, :, None]
        ga, be = (np.ones(self.c), np.zeros(self.c)) if ga is None else (ga, be)
        xh = (self.x.astype(np.float64) - per(rm)) * per(rr)
        tol = 1.2e-6 + 6 * U * (np.abs(ga[None, :, None] * xh) + np.abs(be)[None, :, None])
        if self.torch_dtype == torch.bfloat16:
            tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ry)
        assert np.all(np.abs(y - ry) <= tol), float((np.abs(y - ry) / tol).max())

    def check_backward(self, mean, rstd, gx, gg, gb, affine=True, add=0.0):
        ga, be = (self.gamma, self.beta) if affine else (None, None)
        ref = O.group_norm_bwd(self.x, ga, be, mean, rstd, self.groups, self.gy, self.act)
        d, n = self.c // self.groups, max(self.c // self.groups * self.p, 1)
        per = lambda t: np.repeat(np.asarray(t, np.float64), d, axis=1)[:, :, None]
        ga = np.ones(self.c) if ga is None else ga
        xh = (self.x.astype(np.float64) - per(mean)) * per(rstd)
        gz = np.abs(self.gy) * 1.13
        gh = gz * np.abs(ga)[None, :, None]
        eh = 3 * U * np.abs(xh) + U * np.abs(per(mean)) * per(rstd)          # error of xh
        egz = np.abs(self.gy) * (1e-6 + 0.8 * (eh * np.abs(ga)[None, :, None] + U)) + 2 * U * gz
        group = lambda t: np.repeat(t.reshape(self.b, self.groups, -1).sum(2) / n, d, axis=1)[:, :, None]
        egh = egz * np.abs(ga)[None, :, None] + U * gh
        tol = per(rstd) * (egh + group(egh) + np.abs(xh) * group(egh * np.abs(xh) + gh * eh) + eh * group(gh * np.abs(xh))
                           + 3 * U * (gh + group(gh) + np.abs(xh) * group(gh * np.abs(xh)))) * 1.05 + 1e-30
        if self.torch_dtype == torch.bfloat16:
            tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref["gx"])
        assert np.all(np.abs(gx - ref["gx"]) <= tol), float((np.abs(gx - ref["gx"]) / tol).max())
        for got, want, each in ((gg, ref["ggamma"], egz * np.abs(xh) + gz * eh), (gb, ref["gbeta"], egz)):
            t = each.sum((0, 2)) * 1.05 + 2 * U * np.abs(want) + 2 * U * abs(add) + 1e-30
            assert np.all(np.abs(got - (want + add)) <= t), float((np.abs(got - want - add) / t).max())


SIZES = [
    # b, c, groups, p
    (1, 1, 1, 1),                 # one value: variance 0
    (2, 3, 3, 1),                 # one value a group
    (1, 8, 2, 1),                 # a single point
    (5, 512, 32, 1),              # single points, many channels
    (1, 5, 1, 7),
    (3, 6, 2, 33),
    (2, 12, 3, 630),
    (4, 27, 9, 1344),             # odd everything
    (1, 20, 4, 4096),
    (2, 20, 5, 4097),
    (1, 8, 2, 8191),
    (1, 1, 1, 65537),
    (2, 1, 1, 100003),            # one channel
    (1, 1023, 11, 5),             # the most channels, odd
    (1, 1024, 1, 9),
    (2, 1024, 1024, 3),
    (7, 33, 11, 257),
    (1, 64, 2, 6000),
    (1, 20, 1, 120001),           # long rows
    (64, 16, 4, 64),              # many short rows
    (2, 64, 2, 600),              # groups past one block, of short rows
    (1, 96, 1, 1501),
    (1, 1000, 4, 211),
    (3, 1024, 2, 2050),           # rows just long enough for blocks of their own
    (300, 32, 8, 5),
    (1, 1023, 3, 100),            # the longest steps of the channels-last kernels
    (2, 1019, 1, 70),
]


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,c,groups,p", SIZES)
def test_forward_and_backward_match_the_oracle(b, c, groups, p, layout, dtype):
    act = ("gelu", "silu", "identity")[(b + c + p) % 3]
    n = Norm(b, c, groups, p, layout, dtype, act)
    y, mean, rstd = n.forward()
    n.check_forward(y, mean, rstd)
    n.check_backward(mean, rstd, *n.backward(mean, rstd))


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["gelu", "silu", "identity"])
@pytest.mark.parametrize("layout", ["first", "last"])
def test_without_affine_and_with_added_gradients(act, layout):
    n = Norm(2, 6, 3, 1001, layout, "f32", act, flags=B.FNO_FLAG_ACCUMULATE_GRADS)
    y, mean, rstd = n.forward(affine=False)
    n.check_forward(y, mean, rstd, affine=False)
    n.check_backward(mean, rstd, *n.backward(mean, rstd, affine=False, start=-3.0), affine=False, add=-3.0)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("b,c,groups,p", [(2, 12, 3, 630), (1, 20, 4, 70000), (1, 6, 2, 300000)])
def test_a_mean_far_from_zero_costs_nothing(layout, b, c, groups, p):
    """Values 1000 to 4000 standard deviations away from zero (exact in float32): the variance comes from sums that do not
    cancel, and x - mean is formed before it is scaled."""
    n = Norm(b, c, groups, p, layout)
    rng = np.random.default_rng(1)
    n.x = (np.round(rng.standard_normal((b, c, p)) * 256) / 256 + 2048).astype(np.float32)
    y, mean, rstd = n.forward()
    n.check_forward(y, mean, rstd)
    n.check_backward(mean, rstd, *n.backward(mean, rstd))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("p", [3, 5000, 90001])
def test_constant_groups_and_eps(layout, p):
    n = Norm(1, 4, 2, p, layout, eps=1e-4)
    n.x[:, 2:] = 0.1
    y, mean, rstd = n.forward()
    n.check_forward(y, mean, rstd)
    n.check_backward(mean, rstd, *n.backward(mean, rstd))
    zero = Norm(1, 4, 2, p, layout, eps=0.0)
    zero.x[:, 2:] = 0.5
    y, mean, rstd = zero.forward()
    assert np.isinf(rstd[0, 1]) and np.isnan(y[0, 2:]).all() and np.isfinite(y[0, :2]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("p", [50, 40000])
def test_what_is_not_finite_stays_in_its_group(layout, bad, p):
    n = Norm(2, 6, 3, p, layout)
    clean = n.forward()
    n.x[1, 2, p // 2] = bad                              # batch entry 1, group 1
    y, mean, rstd = n.forward()
    assert np.isnan(y[1, 2:4]).all() and np.isnan(rstd[1, 1]) and not np.isfinite(mean[1, 1])
    mask = np.ones((2, 6), bool)
    mask[1, 2:4] = False
    assert np.array_equal(y[mask], clean[0][mask])
    n.x[1, 2, p // 2] = 0.0
    n.gy[0, 5, p // 3] = bad                             # a cotangent: its channel's gradients and its group's gx
    gx, gg, gb = n.backward(clean[1], clean[2])
    assert not np.isfinite(gx[0, 4:]).any() and np.isfinite(gx[1]).all() and np.isfinite(gx[0, :4]).all()
    assert not np.isfinite(gg[5]) and not np.isfinite(gb[5]) and np.isfinite(gg[:5]).all() and np.isfinite(gb[:5]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
def test_no_points(layout):
    n = Norm(2, 4, 2, 0, layout, eps=0.25)
    empty, stats = torch.empty(0, device="cuda"), n.stats()
    ws = B.alloc_norm_workspace(n.desc)
    # an empty tensor has no address: any aligned one stands for it
    some = torch.empty(64, device="cuda")
    ptr = ctypes.c_void_p(some.data_ptr())
    zero = ctypes.c_void_p(0)
    st = [ctypes.c_void_p(t.data_ptr()) for t in stats]
    w, wn = B._ws(ws)
    B._check(B.lib().fno_group_norm_fwd(ctypes.byref(n.desc), ptr, zero, zero, ptr, st[0], st[1], w, wn, B._stream()))
    g = torch.full((4,), 7.0, device="cuda")
    B._check(B.lib().fno_group_norm_bwd(ctypes.byref(n.desc), ptr, zero, zero, st[0], st[1], ptr, ptr, ctypes.c_void_p(g.data_ptr()),
                                        zero, w, wn, B._stream()))
    assert empty.numel() == 0 and stats[0].eq(0).all() and stats[1].eq(2).all() and g.eq(0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,c,groups,p", [(2, 6, 2, 100), (3, 20, 4, 30001)])
def test_in_place_on_another_stream_and_again(layout, dtype, b, c, groups, p):
    n = Norm(b, c, groups, p, layout, dtype)
    y, mean, rstd = n.forward()
    gx, gg, gb = n.backward(mean, rstd)
    ga, be = torch.from_numpy(n.gamma).cuda(), torch.from_numpy(n.beta).cuda()
    for over in ("x", "gy"):
        side = torch.cuda.Stream()
        x, gy, ws = n.dev(n.x), n.dev(n.gy), B.alloc_norm_workspace(n.desc)
        m, r = n.stats()
        g2, b2 = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            target = x.clone() if over == "x" else gy
            B.fno_group_norm_bwd(n.desc, target if over == "x" else x, ga, be, torch.from_numpy(mean).cuda(),
                                 torch.from_numpy(rstd).cuda(), gy, target, g2, b2, ws)
            B.fno_group_norm_fwd(n.desc, x, ga, be, x, m, r, ws)
        side.synchronize()
        assert np.array_equal(n.host(x), y) and np.array_equal(n.host(target), gx)
        assert np.array_equal(g2.cpu().numpy(), gg) and np.array_equal(b2.cpu().numpy(), gb)
        assert np.array_equal(m.cpu().numpy(), mean) and np.array_equal(r.cpu().numpy(), rstd)


@pytest.mark.gpu
def test_each_output_alone_has_the_same_bits():
    for p in (200, 50000):
        n = Norm(2, 6, 3, p)
        y, mean, rstd = n.forward()
        gx, gg, gb = n.backward(mean, rstd)
        x, gy, ws = n.dev(n.x), n.dev(n.gy), B.alloc_norm_workspace(n.desc)
        ga, be, m, r = (torch.from_numpy(t).cuda() for t in (n.gamma, n.beta, mean, rstd))
        out, a, b_ = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
        B.fno_group_norm_fwd(n.desc, x, ga, be, out, None, None, ws)
        assert np.array_equal(n.host(out), y)
        B.fno_group_norm_bwd(n.desc, x, ga, be, m, r, gy, out, None, None, ws)
        B.fno_group_norm_bwd(n.desc, x, ga, be, m, r, gy, None, a, None, ws)
        B.fno_group_norm_bwd(n.desc, x, ga, be, m, r, gy, None, None, b_, ws)
        assert np.array_equal(n.host(out), gx) and np.array_equal(a.cpu().numpy(), gg) and np.array_equal(b_.cpu().numpy(), gb)


@pytest.mark.gpu
@pytest.mark.parametrize("p", [500, 60000])
def test_replays_of_a_graph_have_the_bits_of_eager_calls(p):
    n = Norm(2, 8, 2, p)
    x, gy, ws = n.dev(n.x), n.dev(n.gy), B.alloc_norm_workspace(n.desc)
    ga, be = torch.from_numpy(n.gamma).cuda(), torch.from_numpy(n.beta).cuda()
    y, gx, (m, r) = torch.empty_like(x), torch.empty_like(x), n.stats()
    gg, gb = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")

    def call():
        B.fno_group_norm_fwd(n.desc, x, ga, be, y, m, r, ws)
        B.fno_group_norm_bwd(n.desc, x, ga, be, m, r, gy, gx, gg, gb, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        x.copy_(n.dev(n.x + np.float32(k)))
        call()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, gx, m, r, gg, gb)]
        for t in (y, gx, m, r, gg, gb):
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b_) for a, b_ in zip(want, (y, gx, m, r, gg, gb)))


@pytest.mark.gpu
@pytest.mark.parametrize("b,c,groups,p,layout", [(1, 10, 5, 5000011, "first"), (5, 10, 2, 1000003, "last"), (1, 3, 1, 16000001, "last")])
def test_fields_larger_than_the_caches(b, c, groups, p, layout):
    """200 MB: taken in shares of groups or batch entries, the last share smaller, or in one that is read backwards."""
    n = Norm(b, c, groups, p, layout, act="silu")
    y, mean, rstd = n.forward()
    n.check_forward(y, mean, rstd)
    n.check_backward(mean, rstd, *n.backward(mean, rstd))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
def test_offsets_past_32_bits(layout):
    """Two channels of 2^31 + 20 bf16 points: the values repeat, so that the statistics are known; groups of one channel."""
    period, p = 1024, 2 ** 31 + 1024 * 20
    rng = np.random.default_rng(0)
    pat = torch.from_numpy(rng.standard_normal((2, period)).astype(np.float32)).bfloat16()
    small = pat.float().numpy()[None]
    ref, mean, rstd = O.group_norm_fwd(small, None, None, 2, 1e-5, "gelu")
    desc = B.make_norm_desc(1, 2, 2, p, layout=B.FNO_LAYOUT_CHANNELS_FIRST if layout == "first" else B.FNO_LAYOUT_CHANNELS_LAST,
                            dtype=B.FNO_DTYPE_BF16, activation=B.FNO_ACT_GELU)
    x = (pat.cuda()[:, None].expand(2, p // period, period) if layout == "first" else
         pat.cuda().t()[None].expand(p // period, period, 2)).contiguous()
    ws, (m, r) = B.alloc_norm_workspace(desc), (torch.empty(2, device="cuda") for _ in range(2))
    gy = x.clone()
    y = torch.empty_like(x)
    B.fno_group_norm_fwd(desc, x, None, None, y, m, r, ws)
    g = O.group_norm_bwd(small, None, None, mean, rstd, 2, small, "gelu")
    gg, gb = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    B.fno_group_norm_bwd(desc, x, None, None, m, r, gy, gy, gg, gb, ws)
    torch.cuda.synchronize()
    assert np.allclose(m.cpu().numpy(), mean[0], rtol=1e-6, atol=1e-8) and np.allclose(r.cpu().numpy(), rstd[0], rtol=1e-6)
    blocks = p // period
    for t, want in ((y, ref), (gy, g["gx"])):
        got = t.view(2, blocks, period) if layout == "first" else t.view(blocks, period, 2)
        got = got if layout == "first" else got.permute(2, 0, 1)
        for q in (0, 1, blocks // 2, blocks - 1):
            a = got[:, q].float().cpu().numpy()
            assert np.all(np.abs(a - want[0]) <= 2.0 ** -8 * np.abs(want[0]) + 1e-5)
        assert torch.equal(got[:, 0], got[:, blocks - 1]) and torch.equal(got[:, 5], got[:, blocks // 2 + 1])
    scale = np.abs(small[0]).sum(1) * blocks
    assert np.all(np.abs(gg.cpu().numpy() - g["ggamma"] * blocks) <= 1e-5 * scale)
    assert np.all(np.abs(gb.cpu().numpy() - g["gbeta"] * blocks) <= 1e-5 * scale)


def test_refusals_without_a_device():
    lib, n = B.lib(), ctypes.c_size_t(0)
    good = B.make_norm_desc(1, 8, 2, 100)
    assert lib.fno_group_norm_workspace_bytes(ctypes.byref(good), ctypes.byref(n)) == B.FNO_OK and n.value >= 256
    assert lib.fno_group_norm_workspace_bytes(ctypes.byref(good), None) == B.FNO_EINVAL
    assert lib.fno_group_norm_workspace_bytes(None, ctypes.byref(n)) == B.FNO_EINVAL
    bad = [dict(batch=0), dict(channels=0), dict(groups=0), dict(groups=3), dict(npoints=-1), dict(layout=2), dict(dtype=2),
           dict(activation=3), dict(flags=1), dict(flags=4), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))]
    for change in bad:
        d = B.make_norm_desc(**{**dict(batch=1, channels=8, groups=2, npoints=100), **change})
        assert lib.fno_group_norm_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == B.FNO_EINVAL, change
        assert B.fno_status_string(B.FNO_EINVAL)
    for change in (dict(channels=1026), dict(batch=65536), dict(npoints=2 ** 41), dict(npoints=2 ** 40, channels=32),
                   dict(batch=60000, channels=256)):
        d = B.make_norm_desc(**{**dict(batch=1, channels=8, groups=2, npoints=100), **change})
        assert lib.fno_group_norm_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == B.FNO_EUNSUPPORTED, change
    p, z, odd = ctypes.c_void_p(4096), ctypes.c_void_p(0), ctypes.c_void_p(4100)
    size, d = ctypes.c_size_t(1 << 40), ctypes.byref(good)
    assert lib.fno_group_norm_fwd(d, z, p, p, p, p, p, p, size, z) == B.FNO_EINVAL
    assert lib.fno_group_norm_fwd(d, p, p, p, z, p, p, p, size, z) == B.FNO_EINVAL
    assert lib.fno_group_norm_fwd(d, odd, p, p, p, p, p, p, size, z) == B.FNO_EINVAL
    assert lib.fno_group_norm_fwd(d, p, p, p, p, p, p, z, size, z) == B.FNO_EINVAL
    assert lib.fno_group_norm_fwd(d, p, p, p, p, p, p, odd, size, z) == B.FNO_ENOSPC
    assert lib.fno_group_norm_fwd(d, p, p, p, p, p, p, p, ctypes.c_size_t(8), z) == B.FNO_ENOSPC
    for drop in range(9):
        args = [p] * 9                                   # x, gamma, beta, mean, rstd, gy, gx, ggamma, gbeta
        args[drop] = z
        required = drop in (0, 3, 4, 5)
        if required:
            assert lib.fno_group_norm_bwd(d, *args, p, size, z) == B.FNO_EINVAL
    assert lib.fno_group_norm_bwd(d, p, p, p, p, p, odd, p, p, p, p, size, z) == B.FNO_EINVAL
    assert lib.fno_group_norm_bwd(d, p, p, p, p, p, p, p, p, p, p, ctypes.c_size_t(8), z) == B.FNO_ENOSPC
    assert lib.fno_group_norm_bwd(d, p, p, p, p, p, p, z, z, z, p, size, z) == B.FNO_OK          # nothing asked for
    # the blocks know two activations
    layer = B.make_desc(1, 4, 4, (8, 8, 8, 8), (2, 2, 2, 3), 0, B.FNO_ACT_SILU)
    assert lib.fno_workspace_bytes(ctypes.byref(layer), B.FNO_OP_BLOCK_FWD, ctypes.byref(n)) == B.FNO_EINVAL


@pytest.mark.gpu
def test_binding_refuses_tensors_that_do_not_fit():
    desc = B.make_norm_desc(2, 4, 2, 10)
    x, c, s = torch.zeros(2, 4, 10, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(2, 2, device="cuda")
    ws = B.alloc_norm_workspace(desc)
    for bad in (x[:, :, :9].contiguous(), x.bfloat16(), x.transpose(1, 2), x.cpu(), torch.zeros(2, 4, 5, dtype=torch.complex64, device="cuda")):
        with pytest.raises(ValueError):
            B.fno_group_norm_fwd(desc, bad, c, c, x, s, s, ws)
    with pytest.raises(ValueError):
        B.fno_group_norm_fwd(desc, x, c[:3], c, x, s, s, ws)
    with pytest.raises(ValueError):
        B.fno_group_norm_fwd(desc, x, c, c, x, s[:1], s, ws)
    with pytest.raises(ValueError):
        B.fno_group_norm_bwd(desc, x, c, c, s, s, x, x, c.double(), c, ws)
    with pytest.raises(B.FnoError):
        B.fno_group_norm_fwd(desc, x, c, c, x, s, s, ws[:8])
