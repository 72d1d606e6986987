"""AdamW over lists of tensors, moments in 32 and 8 bits, and the norm of all gradients, against the float64 oracle.

Tolerances (u = 2^-24): m and v are two products and a sum of floats (and one product with the scale): 4 u of the sum of the
terms' sizes.  The parameter moves by at most lr (|m'| / (sqrt(v') + eps)) with a handful of roundings, and the move and the
decay are rounded to the parameter: 3 u |param| + 10 u |move|.  The norm is a sum in double: 2 u of it.  8-bit codes are
compared bit for bit with codes of the oracle for moments formed in the same order in 32 bits (numpy), where no clipping
rounds the gradient before."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import fno_oracle as O
from paper_2204_01205_amd import binding as B

U = 2.0 ** -24
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)


def offset_view(a, skip, dtype=torch.float32):
    """A device copy of `a` that starts `skip` elements into its allocation: aligned to one element only."""
    t = torch.empty(a.size + skip, dtype=dtype, device="cuda")
    t[skip:] = torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype).reshape(-1)
    return t[skip:]


class Tensors:
    def __init__(self, sizes, bits=32, seed=0, skip=0, scale=1e-2):
        rng = np.random.default_rng([seed, len(sizes)])
        f = lambda n, s: (s * rng.standard_normal(n)).astype(np.float32)
        self.sizes, self.bits = sizes, bits
        self.p = [f(n, 0.5) for n in sizes]
        # gradients over five powers of ten, some zero
        self.g = [(f(n, scale) * 10.0 ** rng.uniform(-4, 1, n) * (rng.random(n) > 0.05)).astype(np.float32) for n in sizes]
        m = [f(n, 0.3 * scale) for n in sizes]
        v = [(f(n, scale) ** 2 + 1e-10).astype(np.float32) for n in sizes]
        self.decay = [0.0 if k % 3 == 1 else 0.05 for k in range(len(sizes))]
        self.exps = None
        if bits == 8:
            self.m, self.v, self.exps = [], [], []
            for k, n in enumerate(sizes):
                r = O.code_bits(n, 99, 0, k)
                cm, em = O.encode_moment(m[k], r & 0xFFFF, "m")
                cv, ev = O.encode_moment(v[k], r >> 16, "v")
                self.m.append(cm)
                self.v.append(cv)
                self.exps.append(np.stack([em, ev], 1))
        else:
            self.m, self.v = m, v
        kind = torch.float32 if bits == 32 else torch.uint8
        self.dp, self.dg = [offset_view(t, skip) for t in self.p], [offset_view(t, skip) for t in self.g]
        self.dm, self.dv = ([offset_view(t, 4 * skip if bits == 8 else skip, kind) for t in s] for s in (self.m, self.v))
        self.de = None if bits == 32 else [torch.from_numpy(e.copy()).cuda() for e in self.exps]
        self.list = B.make_adamw_tensors(self.dp, self.dg, self.dm, self.dv, self.de, self.decay)

    def norm(self):
        out = torch.empty(1, device="cuda")
        B.fno_grad_norm(self.list, out, B.alloc_grad_norm_workspace(self.list))
        return out

    def exact_norm(self):
        return float(np.sqrt(sum((g.astype(np.float64) ** 2).sum() for g in self.g)))

    def moments(self, k):
        """What the state of tensor k stands for, before the step."""
        if self.bits == 32:
            return self.m[k], self.v[k]
        return (O.code_values(self.m[k], self.exps[k][:, 0], "m").astype(np.float32),
                O.code_values(self.v[k], self.exps[k][:, 1], "v").astype(np.float32))

    def check_params(self, step, scale=1.0, hyper=HYPER):
        for k in range(len(self.sizes)):
            m, v = self.moments(k)
            with np.errstate(all="ignore"):
                p, rm, rv = O.adamw_step(self.p[k], self.g[k], m, v, step, weight_decay=self.decay[k], scale=scale, **hyper)
            move = np.abs(p - self.p[k])
            terms = 0.9 * np.abs(m) + 0.1 * np.abs(self.g[k] * scale)        # m's error against its terms moves with them
            denom = np.sqrt(rv / (1 - hyper["beta2"] ** step)) + hyper["eps"]
            tol = 3 * U * np.abs(self.p[k]) + 10 * U * move + 6 * U * hyper["lr"] * terms / (1 - hyper["beta1"] ** step) / denom
            got = self.dp[k].cpu().numpy()
            assert np.all(np.abs(got - p) <= tol), (k, float((np.abs(got - p) / tol).max()))
            if self.bits == 32:
                assert np.all(np.abs(self.dm[k].cpu().numpy() - rm) <= 4 * U * terms + 1e-44)
                assert np.all(np.abs(self.dv[k].cpu().numpy() - rv) <= 6 * U * rv + 1e-44)

    def check_codes(self, step, seed, hyper=HYPER):
        """Codes bit for bit, from moments formed in 32 bits in the order of the definition."""
        f = np.float32
        for k, n in enumerate(self.sizes):
            m, v = self.moments(k)
            m = f(hyper["beta1"]) * m + f(1 - hyper["beta1"]) * self.g[k]
            v = f(hyper["beta2"]) * v + f(1 - hyper["beta2"]) * (self.g[k] * self.g[k])
            r = O.code_bits(n, seed, step, k)
            for got, e, x, part, which in ((self.dm[k], self.de[k][:, 0], m, r & 0xFFFF, "m"), (self.dv[k], self.de[k][:, 1], v, r >> 16, "v")):
                codes, exps = O.encode_moment(x, part, which)
                assert np.array_equal(e.cpu().numpy(), exps), (k, which)
                assert np.array_equal(got.cpu().numpy(), codes), (k, which)


SIZES = [[1], [2, 3, 1, 5], [255, 256, 257], [4095, 4096, 4097, 7], [1023, 1024, 1025, 2047, 2048, 2049], [100003, 1, 20, 400, 8193],
         [(37 * k) % 700 for k in range(150)]]           # more than one launch's tensors, some empty


@pytest.mark.gpu
@pytest.mark.parametrize("skip", [0, 1, 3])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_a_step_matches_the_oracle(sizes, bits, skip):
    t = Tensors(sizes, bits, skip=skip)
    B.fno_adamw_step(t.list, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], 7, seed=11)
    t.check_params(7)
    if bits == 8:
        t.check_codes(7, 11)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 1e-15, 1e-12, 3e-12, 1e-3])
def test_eps_of_any_size(bits, eps):
    """Down to zero, with gradients whose squares are tiny (of 1e-15) or subnormal (of 3e-19, where v has few bits left and
    the parameters are only asked to be finite): the quotient is then m over the root of v alone."""
    for tiny in (1.0, 1e-15, 3e-19):
        t = Tensors([700, 5000], bits)
        for k, n in enumerate(t.sizes):
            g = (tiny * np.sign(t.p[k]) * (0.5 + np.abs(t.p[k]) % 1.0)).astype(np.float32)       # 0.5 to 1.5 times `tiny`
            t.g[k] = g
            t.dg[k].copy_(torch.from_numpy(g))
            for s in (t.m[k], t.v[k]) + (() if bits == 32 else (t.exps[k],)):
                s[:] = 0
            for s in (t.dm[k], t.dv[k]) + (() if bits == 32 else (t.de[k],)):
                s.zero_()
        B.fno_adamw_step(t.list, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], eps, 1, seed=2)
        if tiny > 1e-18:
            t.check_params(1, hyper=dict(HYPER, eps=eps))
        assert all(torch.isfinite(p).all() for p in t.dp) or (eps == 0.0 and tiny < 1e-18)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_clipping_by_the_norm_of_all_gradients(bits, max_norm):
    t = Tensors([5000, 3, 70000, 1], bits)
    norm = t.norm()
    exact = t.exact_norm()
    assert abs(float(norm) - exact) <= 2 * U * exact and exact > 1.0
    B.fno_adamw_step(t.list, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], 3, grad_norm=norm, max_norm=max_norm, seed=5)
    t.check_params(3, scale=min(1.0, max_norm / exact))
    if bits == 8 and max_norm > exact:
        t.check_codes(3, 5)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES + [[3000000], [1 << 20, 5, 1 << 19, 12345]], ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("skip", [0, 1])
def test_gradient_norm(sizes, skip):
    t = Tensors(sizes, skip=skip)
    norm = t.norm()
    exact = t.exact_norm()
    assert abs(float(norm) - exact) <= 2 * U * exact
    assert float(t.norm()) == float(norm)


@pytest.mark.gpu
def test_gradient_norm_of_huge_and_tiny_values_and_of_nothing():
    for scale, n in ((1e30, 1000), (1e-30, 1000)):
        t = Tensors([n])
        t.dg[0].copy_(torch.full((n,), scale))
        assert abs(float(t.norm()) / (scale * n ** 0.5) - 1) < 1e-6
    empty = B.make_adamw_tensors([], [], [], [])
    out = torch.full((1,), 5.0, device="cuda")
    B.fno_grad_norm(empty, out, B.alloc_grad_norm_workspace(empty))
    assert float(out) == 0.0
    B.fno_adamw_step(empty, 1e-3, 0.9, 0.999, 1e-8, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_norm_that_is_not_finite_leaves_everything_as_it_was(bits, bad):
    t = Tensors([300, 5000], bits)
    before = [x.clone() for x in t.dp + t.dm + t.dv + (t.de or [])]
    t.dg[1][4321] = bad
    norm = t.norm()
    assert not np.isfinite(float(norm))
    B.fno_adamw_step(t.list, 1e-3, 0.9, 0.999, 1e-8, 4, grad_norm=norm, max_norm=1.0)
    assert all(torch.equal(a, b) for a, b in zip(before, t.dp + t.dm + t.dv + (t.de or [])))


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_finite_shows_without_a_norm(bad):
    t = Tensors([1000], 32)
    t.dg[0][3] = bad
    B.fno_adamw_step(t.list, 1e-3, 0.9, 0.999, 1e-8, 4)
    finite = np.isfinite(t.dp[0].cpu().numpy())
    assert not finite[3] and finite.sum() == 999
    t = Tensors([1000], 8)
    t.dg[0][300] = bad                                   # the second block of 256
    B.fno_adamw_step(t.list, 1e-3, 0.9, 0.999, 1e-8, 4)
    assert t.de[0].cpu().numpy()[:, 0].tolist().count(255) == 1 and t.de[0][1].cpu().tolist() == [255, 255]
    m, v = (torch.empty(1000, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.fno_adamw_state_read(t.list, [m], [v])
    for x in (m, v):
        nan = np.isnan(x.float().cpu().numpy())
        assert nan[256:512].all() and nan.sum() == 256
    t.dg[0][300] = 0.0                                   # and from then on
    B.fno_adamw_step(t.list, 1e-3, 0.9, 0.999, 1e-8, 5)
    nan = np.isnan(t.dp[0].cpu().numpy())
    assert nan[256:512].all() and nan.sum() == 256 and t.de[0][1].cpu().tolist() == [255, 255]


@pytest.mark.gpu
@pytest.mark.parametrize("skip", [0, 1])
def test_state_read_gives_what_the_codes_stand_for(skip):
    t = Tensors([1, 255, 256, 4097, 0, 10000] + [3] * 70, 8, skip=skip)
    m = [torch.empty(n + 2 * skip, dtype=torch.bfloat16, device="cuda")[2 * skip:] for n in t.sizes]
    v = [torch.empty(n + 2 * skip, dtype=torch.bfloat16, device="cuda")[2 * skip:] for n in t.sizes]
    B.fno_adamw_state_read(t.list, m, v)
    for k in range(len(t.sizes)):
        rm, rv = t.moments(k)
        assert np.array_equal(m[k].float().cpu().numpy(), rm) and np.array_equal(v[k].float().cpu().numpy(), rv)


@pytest.mark.gpu
def test_extreme_moments_in_8_bits():
    """The ends of the exponents: squares that underflow, the largest floats, blocks of zeros."""
    n = 256 * 6
    t = Tensors([n], 8)
    for x in (t.dm[0], t.dv[0], t.de[0]):
        x.zero_()
    t.m[0][:], t.v[0][:], t.exps[0][:] = 0, 0, 0
    g = np.zeros(n, np.float32)
    g[256:512] = np.float32(1e-25) * np.arange(256)      # squares are subnormal or zero
    g[512:768] = np.float32(3e18) * (np.arange(256) - 100)   # squares near the largest float
    g[768:1024] = np.float32(1e-3)
    g[1024:1280] = 10.0 ** np.linspace(-19, 0, 256)
    g[1280:] = np.where(np.arange(256) % 7 == 0, 1.0, 0.0)
    t.g[0] = g
    t.dg[0].copy_(torch.from_numpy(g))
    B.fno_adamw_step(t.list, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], 1, seed=3)
    t.check_codes(1, 3)
    assert torch.isfinite(t.dp[0]).all()


@pytest.mark.gpu
def test_steps_in_8_bits_follow_those_in_32():
    """200 steps on a quadratic whose curvatures lie between 1 and 1e4, with noise in the gradients: both end near the
    minimum, at about the same loss (the moments' steps are a sixteenth of a value, unbiased)."""
    n, losses = 4096, {}
    for bits in (32, 8):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(3)
        curve = torch.logspace(0, 4, n, device="cuda")
        p = torch.randn(n, device="cuda", generator=gen)
        g = torch.empty_like(p)
        kind = torch.float32 if bits == 32 else torch.uint8
        m, v = torch.zeros(n, dtype=kind, device="cuda"), torch.zeros(n, dtype=kind, device="cuda")
        e = None if bits == 32 else [torch.zeros(B.adamw_exps_shape(n), dtype=torch.uint8, device="cuda")]
        lst = B.make_adamw_tensors([p], [g], [m], [v], e)
        start = float((p.square()).mean())
        for step in range(1, 201):
            g.copy_(curve * (p + 0.1 * torch.randn(n, device="cuda", generator=gen)))
            B.fno_adamw_step(lst, 2e-2, 0.9, 0.999, 1e-8, step, seed=1)
        losses[bits] = float((p.square()).mean())
    assert losses[32] < 0.02 * start and abs(losses[8] / losses[32] - 1) < 0.25, losses


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_streams_graphs_and_repeats_give_the_same_bits(bits):
    sizes = [5000, 3, 70000, 1, 256]

    def outputs(t):
        return [x.clone() for x in t.dp + t.dm + t.dv + (t.de or [])]

    def call(t, norm, ws):
        B.fno_grad_norm(t.list, norm, ws)
        B.fno_adamw_step(t.list, 1e-3, 0.9, 0.999, 1e-8, 6, grad_norm=norm, max_norm=0.5, seed=2)

    results = []
    for way in ("eager", "again", "stream", "graph"):
        t = Tensors(sizes, bits)
        norm, ws = torch.empty(1, device="cuda"), B.alloc_grad_norm_workspace(t.list)
        first = outputs(t)
        if way == "graph":
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                call(t, norm, ws)
            torch.cuda.current_stream().wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call(t, norm, ws)
            for _ in range(3):
                for x, y in zip(t.dp + t.dm + t.dv + (t.de or []), first):
                    x.copy_(y)
                graph.replay()
                torch.cuda.synchronize()
                results.append(outputs(t) + [norm.clone()])
            continue
        if way == "stream":
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                call(t, norm, ws)
            side.synchronize()
        else:
            call(t, norm, ws)
        torch.cuda.synchronize()
        results.append(outputs(t) + [norm.clone()])
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], r))


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """2^32 + 777 values: the last ones, moved with moments of zero, and every block's own random bits."""
    n = 2 ** 32 + 777
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 0.5, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    e = torch.zeros(B.adamw_exps_shape(n), dtype=torch.uint8, device="cuda")
    lst = B.make_adamw_tensors([p], [g], [m], [v], [e])
    norm = torch.empty(1, device="cuda")
    B.fno_grad_norm(lst, norm, B.alloc_grad_norm_workspace(lst))
    assert abs(float(norm) / (0.5 * n ** 0.5) - 1) < 1e-6
    B.fno_adamw_step(lst, 1e-2, 0.9, 0.999, 1e-8, 1, seed=9)
    assert p.min().item() == p.max().item() and abs(p[0].item() + 1e-2) < 1e-8
    f = np.float32
    rv = f(1 - 0.999) * f(0.25)
    for at in (0, 2 ** 32 - 1000, n - 777):
        at = at // 256 * 256
        r = _bits_from(at, min(n - at, 1000), 9, 1, 0)
        codes, _ = O.encode_moment(np.full(r.size, rv, np.float32), r >> 16, "v")
        assert np.array_equal(v[at: at + r.size].cpu().numpy(), codes)
    del p, g, m, v, e


def _bits_from(at, count, seed, step, tensor):
    """O.code_bits of values at .. at + count - 1 (at a multiple of 256) without the ones before."""
    def mix(x):
        x &= 0xFFFFFFFF
        x ^= x >> 16
        x = (x * 0xCB4F2D3B) & 0xFFFFFFFF
        x ^= x >> 13
        x = (x * 0xFDB6A5C3) & 0xFFFFFFFF
        return x ^ (x >> 16)

    key = mix(mix(mix(seed) ^ step) ^ tensor)
    out = []
    for i in range(at, at + count):
        q = i // 256
        out.append(mix(mix(mix(q + key) + (q >> 32)) + (i % 256) * 0x9E3779B1))
    return np.array(out, np.int64)


def test_bits_from_agrees_with_the_oracle():
    assert np.array_equal(_bits_from(512, 300, 9, 1, 4), O.code_bits(812, 9, 1, 4)[512:])


def test_refusals_without_a_device():
    lib, n = B.lib(), ctypes.c_size_t(0)
    d, i32 = ctypes.c_double, ctypes.c_int32

    def step(count=1, tensors=None, bits=32, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, t=1, norm=0, max_norm=1.0):
        return lib.fno_adamw_step(i32(count), tensors, i32(bits), d(lr), d(b1), d(b2), d(eps), i32(t), ctypes.c_void_p(norm),
                                  d(max_norm), ctypes.c_uint32(0), None)

    def one(param=4096, grad=4096, m=4096, v=4096, exps=4096, size=8, decay=0.0):
        return (B.FnoAdamwTensor * 1)(B.FnoAdamwTensor(param, grad, m, v, exps, size, decay))

    assert step(0) == B.FNO_OK and step(1, one(0, 0, 0, 0, 0, 0)) == B.FNO_OK        # nothing to do
    assert step(-1) == B.FNO_EINVAL and step(1, None) == B.FNO_EINVAL
    for bad in (one(param=0), one(grad=0), one(m=0), one(v=0), one(param=4098), one(grad=4097), one(m=4098), one(v=4099), one(size=-1),
                one(size=2 ** 41), one(decay=float("nan"))):
        assert step(1, bad) == B.FNO_EINVAL and B.fno_status_string(B.FNO_EINVAL)
    assert step(1, one(exps=0), bits=8) == B.FNO_EINVAL and step(1, one(exps=4097), bits=8) == B.FNO_EINVAL
    for kw in (dict(bits=16), dict(t=0), dict(b1=1.0), dict(b2=-0.1), dict(b1=float("nan")), dict(lr=float("inf")), dict(eps=-1e-8),
               dict(eps=float("nan")), dict(norm=4096, max_norm=0.0), dict(norm=4096, max_norm=float("nan"))):
        assert step(1, one(), **kw) == B.FNO_EINVAL, kw
    assert lib.fno_grad_norm_workspace_bytes(i32(1), one(0, 0, 0, 0, 0, 10 ** 6), ctypes.byref(n)) == B.FNO_OK and n.value >= 8
    assert lib.fno_grad_norm_workspace_bytes(i32(1), one(), None) == B.FNO_EINVAL
    need, p = n.value, ctypes.c_void_p(4096)
    big = one(size=10 ** 6)
    assert lib.fno_grad_norm(i32(1), big, None, p, ctypes.c_size_t(need), None) == B.FNO_EINVAL
    assert lib.fno_grad_norm(i32(1), big, p, None, ctypes.c_size_t(need), None) == B.FNO_EINVAL
    assert lib.fno_grad_norm(i32(1), big, p, ctypes.c_void_p(4100), ctypes.c_size_t(need), None) == B.FNO_EINVAL
    assert lib.fno_grad_norm(i32(1), big, p, p, ctypes.c_size_t(need - 1), None) == B.FNO_ENOSPC
    assert lib.fno_grad_norm(i32(1), one(grad=0), p, p, ctypes.c_size_t(need), None) == B.FNO_EINVAL
    outs = (ctypes.c_void_p * 1)(0)
    assert lib.fno_adamw_state_read(i32(1), one(), None, None, None) == B.FNO_EINVAL
    assert lib.fno_adamw_state_read(i32(1), one(), outs, outs, None) == B.FNO_EINVAL
    outs[0] = 4098
    assert lib.fno_adamw_state_read(i32(1), one(), outs, outs, None) == B.FNO_EINVAL
    assert lib.fno_adamw_state_read(i32(0), None, None, None, None) == B.FNO_OK


@pytest.mark.gpu
def test_binding_refuses_tensors_that_do_not_fit():
    f = lambda n: torch.zeros(n, device="cuda")
    u = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        B.make_adamw_tensors([f(5)], [f(4)], [f(5)], [f(5)])
    with pytest.raises(ValueError):
        B.make_adamw_tensors([f(5)], [f(5)], [f(5)], [f(5)], weight_decay=[0.1, 0.2])
    with pytest.raises(ValueError):
        B.make_adamw_tensors([f(5)], [f(5)], [u(5)], [u(5)])
    with pytest.raises(ValueError):
        B.make_adamw_tensors([f(300)], [f(300)], [u(300)], [u(300)], [u(1, 2)])
    with pytest.raises(ValueError):
        B.make_adamw_tensors([f(5)], [f(5).cpu()], [f(5)], [f(5)])
    lst = B.make_adamw_tensors([f(5)], [f(5)], [f(5)], [f(5)])
    with pytest.raises(ValueError):
        B.fno_adamw_step(lst, 1e-3, 0.9, 0.999, 1e-8, 1, grad_norm=f(2))
    with pytest.raises(ValueError):
        B.fno_adamw_state_read(lst, [f(5)], [f(5)])
    c = torch.zeros(4, dtype=torch.complex64, device="cuda")
    assert B.make_adamw_tensors([c], [c.clone()], [f(8)], [f(8)]).sizes == [8]
