"""AdamW, gradient norm and read of 8-bit moments over lists that the memory-side cache does not hold (their kernels read and write
with the nontemporal hint), on stretches of every tensor: its first values, its last ones, and some between.  Codes after
clipping, and v at the upper end of the floats.  Bounds: those of test_gpu_adamw.py, derived there."""
import numpy as np
import pytest
import torch

from oracle import fno_oracle as O
from paper_2204_01205_amd import binding as B
from test_gpu_adamw import HYPER, Tensors

U = 2.0 ** -24


def bits_at(at, n, seed, step, tensor):
    """O.code_bits of the n values from `at` (a multiple of 256) on."""
    def mix(x):
        x = np.asarray(x, np.uint64) & np.uint64(0xFFFFFFFF)
        for shift, factor in ((16, 0xCB4F2D3B), (13, 0xFDB6A5C3)):
            x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xFFFFFFFF)
        return x ^ (x >> np.uint64(16))

    key = mix(mix(mix(seed) ^ np.uint64(step)) ^ np.uint64(tensor))
    i = np.arange(at, at + n, dtype=np.uint64)
    q = i // np.uint64(256)
    return mix(mix(mix(q + key) + (q >> np.uint64(32))) + (i % np.uint64(256)) * np.uint64(0x9E3779B1)).astype(np.int64)


def test_bits_at_agree_with_the_oracle():
    assert np.array_equal(bits_at(1024, 700, 9, 1, 4), O.code_bits(1724, 9, 1, 4)[1024:])


def stretches(n, length=6144):
    """(start, count): whole blocks of 256, but for the last one of a tensor."""
    if n <= 3 * length:
        return [(0, n)] if n else []
    middle, last = n // 2 // 4096 * 4096 - 1024, (n - length) // 256 * 256
    return [(0, length), (middle, length), (last, n - last)]


class Large:
    """Lists made on the device; 4-byte aligned views of their allocations."""

    def __init__(self, sizes, bits, seed=1):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def view(n, dtype=torch.float32):
            skip = 4 if dtype == torch.uint8 else 1
            return torch.empty(n + skip, dtype=dtype, device="cuda")[skip:]

        def normal(n, scale):
            return view(n).copy_(torch.randn(n, device="cuda", generator=gen)).mul_(scale)

        self.sizes, self.bits = sizes, bits
        self.p, self.g = [normal(n, 0.5) for n in sizes], [normal(n, 1e-2) for n in sizes]
        for g in self.g:                                 # over four powers of ten, some zero
            g.mul_(10.0 ** (4 * torch.rand(g.numel(), device="cuda", generator=gen) - 3))
            g.mul_(torch.rand(g.numel(), device="cuda", generator=gen) > 0.05)
        self.e = None
        if bits == 32:
            self.m, self.v = [normal(n, 3e-3) for n in sizes], [normal(n, 1e-2).square_().add_(1e-10) for n in sizes]
        else:
            def codes(n):
                return view(n, torch.uint8).copy_(torch.randint(0, 256, (n,), device="cuda", generator=gen, dtype=torch.uint8))

            self.m, self.v = [codes(n) for n in sizes], [codes(n) for n in sizes]
            self.e = []
            for n in sizes:                              # the largest of a block: m 2^-11 to 2^-8, v 2^-18 to 2^-13
                e = torch.empty(B.adamw_exps_shape(n), dtype=torch.uint8, device="cuda")
                e[:, 0] = torch.randint(116, 120, (e.shape[0],), device="cuda", generator=gen).to(torch.uint8)
                e[:, 1] = torch.randint(109, 115, (e.shape[0],), device="cuda", generator=gen).to(torch.uint8)
                self.e.append(e)
        self.decay = [0.0 if k % 3 == 1 else 0.05 for k in range(len(sizes))]
        self.list = B.make_adamw_tensors(self.p, self.g, self.m, self.v, self.e, self.decay)

    def take(self):
        """The stretches of everything, on the host."""
        out = {}
        for k, n in enumerate(self.sizes):
            for at, count in stretches(n):
                part = {name: t[k][at: at + count].cpu().numpy() for name, t in (("p", self.p), ("g", self.g), ("m", self.m), ("v", self.v))}
                if self.e is not None:
                    part["e"] = self.e[k][at // 256: -(-(at + count) // 256)].cpu().numpy()
                out[k, at] = part
        return out


def check(large, before, step, seed, hyper, scale=np.float32(1)):
    after = large.take()
    f = np.float32
    for (k, at), old in before.items():
        new = after[k, at]
        g = old["g"] * f(scale)
        if large.bits == 8:
            m, v = (O.code_values(old[name], old["e"][:, j], name).astype(f) for j, name in enumerate("mv"))
        else:
            m, v = old["m"], old["v"]
        p, rm, rv = O.adamw_step(old["p"], old["g"], m, v, step, weight_decay=large.decay[k], scale=float(scale), **hyper)
        move = np.abs(p - old["p"])
        terms = 0.9 * np.abs(m) + 0.1 * np.abs(g)
        denom = np.sqrt(rv / (1 - hyper["beta2"] ** step)) + hyper["eps"]
        tol = 3 * U * np.abs(old["p"]) + 10 * U * move + 6 * U * hyper["lr"] * terms / (1 - hyper["beta1"] ** step) / denom
        assert np.all(np.abs(new["p"] - p) <= tol), (k, at, float((np.abs(new["p"] - p) / tol).max()))
        assert np.array_equal(new["g"], old["g"])
        if large.bits == 32:
            assert np.all(np.abs(new["m"] - rm) <= 4 * U * terms + 1e-44) and np.all(np.abs(new["v"] - rv) <= 6 * U * rv + 1e-44), (k, at)
            continue
        m = f(hyper["beta1"]) * m + f(1 - hyper["beta1"]) * g
        v = f(hyper["beta2"]) * v + f(1 - hyper["beta2"]) * (g * g)
        r = bits_at(at, g.size, seed, step, k)
        for j, (name, x, part) in enumerate((("m", m, r & 0xFFFF), ("v", v, r >> 16))):
            codes, exps = O.encode_moment(x, part, name)
            assert np.array_equal(new["e"][:, j], exps) and np.array_equal(new[name], codes), (k, at, name)


MILLION = 1 << 20
LISTS = {32: [17 * MILLION + 3, 5, 4097, 0, 70001, 2 * MILLION], 8: [27 * MILLION + 255, 5, 4097, 0, 70001, 18 * MILLION + 1]}


@pytest.mark.gpu
@pytest.mark.parametrize("bits,eps", [(32, 1e-8), (8, 1e-8), (8, 1e-12)])
@pytest.mark.parametrize("clip", [False, True])
def test_a_step_over_a_list_larger_than_the_cache(bits, eps, clip):
    hyper = dict(HYPER, eps=eps)
    large = Large(LISTS[bits], bits)
    before = large.take()
    norm, scale = None, np.float32(1)
    if clip:
        norm = torch.empty(1, device="cuda")
        B.fno_grad_norm(large.list, norm, B.alloc_grad_norm_workspace(large.list))
        assert float(norm) > 1.0
        scale = np.float32(0.75) / np.float32(norm.item())
    B.fno_adamw_step(large.list, hyper["lr"], hyper["beta1"], hyper["beta2"], eps, 40, grad_norm=norm, max_norm=0.75, seed=6)
    check(large, before, 40, 6, hyper, scale)


@pytest.mark.gpu
def test_a_read_of_a_list_larger_than_the_cache():
    large = Large(LISTS[8], 8)
    m, v = ([torch.empty(n + 2, dtype=torch.bfloat16, device="cuda")[2:] for n in large.sizes] for _ in range(2))
    B.fno_adamw_state_read(large.list, m, v)
    for (k, at), old in large.take().items():
        for j, (name, out) in enumerate((("m", m), ("v", v))):
            want = O.code_values(old[name], old["e"][:, j], name)
            assert np.array_equal(out[k][at: at + want.size].float().cpu().numpy(), want), (k, at, name)


@pytest.mark.gpu
def test_the_norm_of_a_list_larger_than_the_cache():
    sizes = [50 * MILLION + 3, 0, 7, 19 * MILLION + 1, 4097]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    g = [torch.empty(n + 1, device="cuda")[1:].copy_(torch.randn(n, device="cuda", generator=gen)) for n in sizes]
    lst = B.make_adamw_tensors(g, g, g, g)
    norm, ws = torch.empty(2, device="cuda"), B.alloc_grad_norm_workspace(lst)
    for k in range(2):
        B.fno_grad_norm(lst, norm[k:k + 1], ws)
    exact = np.sqrt(sum(np.square(t.cpu().numpy().astype(np.float64)).sum() for t in g))
    assert abs(norm[0].item() - exact) <= 2 * U * exact and norm[0].item() == norm[1].item()


@pytest.mark.gpu
@pytest.mark.parametrize("max_norm", [1e-3, 0.5])
def test_codes_of_clipped_steps(max_norm):
    t = Tensors([5000, 3, 70000, 1, 256], 8)
    norm = t.norm()
    scale = np.float32(max_norm) / np.float32(norm.item())
    assert scale < 1
    B.fno_adamw_step(t.list, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], 3, grad_norm=norm, max_norm=max_norm, seed=5)
    t.check_params(3, scale=float(scale))
    t.g = [g * scale for g in t.g]                       # in float32, as the kernel does
    t.check_codes(3, 5)


@pytest.mark.gpu
def test_the_largest_v_that_8_bits_hold():
    """1.875 x 2^127, the last code of the last exponent: values above it, as squares of finite gradients make, stay there."""
    n, step = 256 * 4, 100000                            # (so late that v is not scaled up)
    t = Tensors([n], 8)
    t.m[0][:], t.v[0][:], t.exps[0][:] = 0, 255, (16, 254)
    g = np.zeros(n, np.float32)
    g[:256] = 1.84e19                                    # v grows past the last code
    g[256:512] = np.linspace(0, 1.84e19, 256)
    g[768:] = 1.9e19                                     # the square is infinite: the block is lost
    t.g[0] = g
    for d, s in ((t.dm[0], t.m[0]), (t.dv[0], t.v[0]), (t.de[0], t.exps[0]), (t.dg[0], g)):
        d.copy_(torch.from_numpy(s))
    B.fno_adamw_step(t.list, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], step, seed=3)
    with np.errstate(over="ignore"):
        t.check_codes(step, 3)
    e, v = t.de[0].cpu().numpy()[:, 1], t.dv[0].cpu().numpy()
    assert e.tolist() == [254, 254, 254, 255] and (v[:256] == 255).all() and (v[256:768] >= 254).all() and (v[512:768] == 255).any()
    assert torch.isfinite(t.dp[0]).all()
    m, out = (torch.empty(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.fno_adamw_state_read(t.list, [m], [out])
    out = out.float().cpu().numpy()
    assert (out[:256] == np.float32(1.875 * 2.0 ** 127)).all() and np.isnan(out[768:]).all()
