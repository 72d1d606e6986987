"""The Muon step against the float64 oracle: real matrices of any shape, spectral weights mode by mode, lists, clipping, and the
refusals.

With parameters of zero, lr = 1, scale = -1 and no decay the new parameters are X itself.  Its tolerance, from the arithmetic
(u = 2^-24; 2^-21 where products run on pairs of 16-bit parts, which carry 22 bits of a value, and 2^-22 is the size of the
product that is left out): the polynomial of a matrix amplifies an error of X by at most a = 3.4445 an iteration (its
derivative on [0, 1.2], the range of the singular values, and the difference quotients that the rotations between singular
directions see).  An iteration's own error: sums of n + m products whose roundings are independent grow with the root of their
number (Higham & Mary 2019), 2 sqrt(n + m) + 8 units of the terms a |X|, 2 |b| |A X| and 3 |c| |A A X|, with singular values up to
1.2: 3.4 + 2 * 4.8 * 1.44 + 3 * 2.03 * 2.07 = 30 at most, of X's norm |X|_F <= 1.2 sqrt(m).  The start X = u / |u| is off by 4 u.
So |error|_F <= u (4 a^k + 30 (2 sqrt(n + m) + 8) sum_j a^j max_j |X_j|_F).  Rounding up all of these at once is far from
what happens: it is the bound, and a second one, with a fiftieth of the iterations' part, is asked of the mean over the matrices of a
tensor.  (The start's part stays whole: its 4 u are three or four roundings of up to u each, not a sum of many.)

Momenta: three roundings of their terms."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import fno_oracle as O
from paper_2204_01205_amd import binding as B

U = 2.0 ** -24
A = 3.4445


def draw(rng, shape, is_complex, size=1.0):
    t = size * rng.standard_normal(shape + ((2,) if is_complex else ()))
    t = t.astype(np.float32)
    return t.view(np.complex64)[..., 0] if is_complex else t


def stack(t):
    """[matrices][rows][cols]"""
    if np.iscomplexobj(t):
        return np.moveaxis(t.reshape(t.shape[:2] + (-1,)), 2, 0)
    return t.reshape((-1,) + t.shape[-2:])


def bounds(u, iterations, share=1.0):
    """Bound of |error|_F for every matrix, with this share of the iterations' part; u: (matrices, rows, cols) before the
    products."""
    m, n = min(u.shape[1:]), max(u.shape[1:])
    unit = U if m <= 32 or np.iscomplexobj(u) else 8 * U
    x, most = O.newton_schulz(u, 0), np.zeros(len(u))
    for k in range(iterations + 1):
        most = np.maximum(most, np.sqrt((np.abs(x) ** 2).sum((1, 2))))
        if k < iterations:
            x = O.newton_schulz(u, k + 1)
    total = sum(A ** j for j in range(iterations))
    return unit * (4 * A ** iterations + share * 30 * (2 * np.sqrt(n + m) + 8) * total * most) + 1e-30


class Muon:
    """A list of tensors, on both sides."""

    def __init__(self, shapes, seed=0, size=1.0):
        rng = np.random.default_rng(seed)
        self.params, self.grads, self.momentum = ([draw(rng, s, c, k * size) for s, c in shapes] for k in (1.0, 0.3, 1.0))

    def run(self, lr=1.0, mu=0.9, scale=-1.0, decay=0.0, zero=True, norm=None, ws_fill=255, **kw):
        dev = lambda ts: [torch.from_numpy(t.copy()).cuda() for t in ts]
        self.dp, self.dg, self.dm = dev([np.zeros_like(p) for p in self.params] if zero else self.params), dev(self.grads), dev(self.momentum)
        self.list = B.make_muon_tensors(self.dp, self.dg, self.dm, scale=scale, weight_decay=decay)
        ws = B.alloc_muon_workspace(self.list)
        ws.fill_(ws_fill)                                  # scratch holds NaN
        gn = None if norm is None else torch.tensor([norm], device="cuda")
        B.fno_muon_step(self.list, lr, mu, ws, grad_norm=gn, **kw)
        torch.cuda.synchronize()
        return [t.cpu().numpy() for t in self.dp], [t.cpu().numpy() for t in self.dm]

    def check(self, mu=0.9, nesterov=True, iterations=5, s=1.0, **kw):
        """X and the momenta, entry by entry of the list."""
        got_p, got_m = self.run(mu=mu, nesterov=nesterov, iterations=iterations, **kw)
        for k, (p, m) in enumerate(zip(got_p, got_m)):
            if p.size == 0:
                continue
            x, ref_m = O.muon_step(np.zeros_like(self.params[k]), self.grads[k], self.momentum[k], 1.0, mu, scale=-1.0, nesterov=nesterov,
                                   iterations=iterations, grad_scale=s)
            size = mu * np.abs(self.momentum[k]) + s * np.abs(self.grads[k])
            assert np.all(np.abs(m - ref_m) <= 4 * U * size), k
            g = s * self.grads[k].astype(ref_m.dtype)
            u = stack(g + mu * ref_m if nesterov else ref_m)
            error = np.sqrt((np.abs(stack(p) - stack(x)) ** 2).sum((1, 2)))
            bound, typical = bounds(u, iterations), bounds(u, iterations, 0.02)
            assert np.all(error <= bound), (k, p.shape, float((error / bound).max()))
            assert error.mean() <= typical.mean(), (k, p.shape, float(error.mean() / typical.mean()))


REAL = [(1, 1), (1, 2), (2, 1), (1, 128), (128, 1), (3, 5), (4, 4), (5, 20), (20, 5), (20, 20), (16, 16), (17, 13), (31, 32), (32, 32), (128, 20),
        (20, 200), (32, 1000), (1000, 31), (7, 4099), (32, 32768)]
DENSE = [(33, 33), (33, 40), (48, 200), (64, 64), (65, 64), (96, 130), (127, 129), (128, 128), (129, 128), (200, 333), (256, 256), (37, 512),
         (1000, 36), (257, 600), (512, 384)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", REAL + DENSE, ids=lambda s: f"{s[0]}x{s[1]}")
def test_real_matrices(shape):
    Muon([(shape, False)], seed=shape[0] * 7 + shape[1]).check()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(70, 3, 5), (33, 20, 20), (3, 128, 20), (5, 64, 64), (3, 100, 250), (2, 300, 129), (600, 2, 2), (1, 40, 40)])
def test_stacks_of_real_matrices(shape):
    Muon([(shape, False)], seed=1).check()


@pytest.mark.gpu
@pytest.mark.parametrize("ci", [1, 2, 3, 4, 5, 8, 9, 12, 13, 16, 20, 23, 24, 27, 28, 32])
def test_modes(ci):
    """Every number of tiles on the shorter side, with more, fewer and as many on the other, and modes around 16."""
    for co in sorted({1, ci, 20, 32, max(1, ci - 3), min(32, ci + 1)}):
        for modes in ((1,), (15,), (16,), (17, 3)):
            Muon([((ci, co) + modes, True)], seed=co).check()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(32, 512), (32, 513), (513, 32), (512, 31), (31, 528), (31, 529), (1, 16384), (16385, 1), (16384, 1), (2, 8191), (8192, 2), (4, 4096),
                                   (3, 5461), (5, 3276), (3276, 5), (8, 2048), (7, 2341), (9, 1820), (16, 1024), (1024, 16), (17, 963), (4, 128), (4, 129), (8, 64),
                                   (8, 65), (65, 6), (3, 200)], ids=lambda s: f"{s[0]}x{s[1]}")
def test_the_largest_matrices_of_a_block_and_folded_ones(shape):
    Muon([(shape, False)], seed=shape[0]).check()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 8, 65536), (8, 8, 65537), (5, 8, 65540), (7, 6, 70001)])
def test_many_modes_of_few_channels(shape):
    Muon([(shape, True)], seed=2).check()


@pytest.mark.gpu
@pytest.mark.parametrize("shape,is_complex", [((20, 20, 1270001), True), ((20, 20, 1350003), True), ((32, 32, 1100003), True), ((8, 7, 20000003), True),
                                              ((2200001, 32, 32), False), ((300007, 90, 100), False)])
def test_offsets_past_32_bits(shape, is_complex):
    """Tensors of some 2^32 bytes and of more: sampled matrices against the oracle."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(shape[0])
    dtype = torch.complex64 if is_complex else torch.float32
    draws = [torch.randn(shape, dtype=dtype, device="cuda", generator=gen) for _ in range(2)]
    params, (grads, momentum) = torch.zeros_like(draws[0]), draws
    size = params.numel() * params.element_size()
    assert size > 0.94 * 2 ** 32
    count = shape[-1] if is_complex else shape[0]
    at = torch.tensor([0, 1, 5, count // 3, count // 2 + 1, count - 17, count - 3, count - 2, count - 1], device="cuda")
    pick = lambda t: np.ascontiguousarray(stack((t[..., at] if is_complex else t[at]).cpu().numpy()))
    u = 0.9 * (pick(grads) + 0.9 * pick(momentum).astype(np.complex128 if is_complex else np.float64)) + pick(grads)
    tensors = B.make_muon_tensors([params], [grads], [momentum], scale=-1.0)
    B.fno_muon_step(tensors, 1.0, 0.9, B.alloc_muon_workspace(tensors))
    torch.cuda.synchronize()
    error = np.sqrt((np.abs(pick(params) - O.newton_schulz(u)) ** 2).sum((1, 2)))
    assert np.all(error <= bounds(u, 5)), (error / bounds(u, 5)).max()


@pytest.mark.gpu
@pytest.mark.parametrize("iterations", [0, 1, 2, 5, 8])
@pytest.mark.parametrize("nesterov", [True, False])
def test_iterations(iterations, nesterov):
    Muon([((20, 20, 50), True), ((20, 5), False), ((70, 90), False), ((64, 300), False)], seed=2).check(iterations=iterations, nesterov=nesterov)


NETWORK = [((20, 5), False), ((128, 20), False), ((1, 128), False)] + 2 * [((20, 20, 6, 5, 4, 3), True), ((20, 20), False)]


@pytest.mark.gpu
def test_a_list_of_all_kinds():
    Muon(NETWORK + [((0, 5), False), ((150, 70), False), ((4, 3, 0), True), ((2, 64, 65), False), ((13, 9, 77), True)], seed=3).check()


@pytest.mark.gpu
def test_a_list_longer_than_a_launch_takes():
    Muon([((3 + k % 5, 4, 7), True) for k in range(70)] + [((k % 37 + 1, k % 11 + 1), False) for k in range(150)]
         + [((40 + k, 50), False) for k in range(40)], seed=4).check()


@pytest.mark.gpu
def test_steps_of_parameters_with_decay_and_a_scale_of_their_own():
    net = Muon(NETWORK + [((90, 40), False)], seed=5)
    count = len(net.params)
    scale, decay = [0.5 + 0.1 * k for k in range(count)], [0.1 * k for k in range(count)]
    got, _ = net.run(lr=0.05, mu=0.95, scale=scale, decay=decay, zero=False)
    for k, p in enumerate(got):
        ref, m = O.muon_step(net.params[k], net.grads[k], net.momentum[k], 0.05, 0.95, scale[k], decay[k])
        u = stack(net.grads[k] + 0.95 * m)
        bound = 0.05 * scale[k] * np.sqrt((bounds(u, 5) ** 2).sum()) + 4 * U * np.sqrt((np.abs(net.params[k]) ** 2).sum())
        assert np.sqrt((np.abs(p - ref) ** 2).sum()) <= bound, k


@pytest.mark.gpu
@pytest.mark.parametrize("coefficients", [(2.0, -1.5, 0.5), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375)])
def test_other_coefficients_make_a_matrix_orthogonal(coefficients):
    """Convergent polynomials: twelve iterations take singular values from 0.2 on (of the norm) to one."""
    rng = np.random.default_rng(6)
    shapes = [((20, 64), False), ((64, 20), False), ((20, 20, 3), True), ((80, 70), False)]
    net = Muon(shapes, seed=6)
    for k, (shape, is_complex) in enumerate(shapes):
        q = rng.standard_normal((3 if is_complex else 1,) + shape[:2]) + (1j * rng.standard_normal((3,) + shape[:2]) if is_complex else 0)
        left, s, right = np.linalg.svd(q, full_matrices=False)
        q = (left * np.linspace(1, 2, s.shape[1])[None, None, :]) @ right
        net.momentum[k] = (np.moveaxis(q, 0, 2) if is_complex else q[0]).astype(net.momentum[k].dtype)
        net.grads[k] = np.zeros_like(net.grads[k])
    got, _ = net.run(iterations=20, coefficients=coefficients)
    for p in got:
        x = stack(p).astype(np.complex128)
        if x.shape[1] > x.shape[2]:
            x = np.swapaxes(x, 1, 2)
        # an error e of X leaves |X X^H - 1|_F = 2 e sqrt(m) at most; the last iteration's own error is what remains
        gram = x @ np.conj(np.swapaxes(x, 1, 2))
        assert np.abs(gram - np.eye(x.shape[1])).max() <= 2e-5


@pytest.mark.gpu
def test_clipping_by_the_norm_of_all_gradients():
    net = Muon(NETWORK + [((50, 60), False)], seed=7)
    net.check(norm=0.5)                                  # below the limit: no scale
    net.check(norm=8.0, max_norm=2.0, s=0.25)


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [float("nan"), float("inf")])
def test_a_norm_that_is_not_finite_writes_nothing(norm):
    net = Muon(NETWORK + [((50, 60), False), ((300, 200), False)], seed=8)
    p, m = net.run(zero=False, norm=norm)
    assert all(np.array_equal(a, b) for a, b in zip(p + m, net.params + net.momentum))


@pytest.mark.gpu
def test_zeros_nans_and_sizes_stay_with_their_matrix():
    shapes = [((20, 20, 40), True), ((5, 20, 7), False), ((4, 70, 50), False), ((20, 32), False)]
    net = Muon(shapes, seed=9)
    clean, _ = net.run()
    for t in (net.grads, net.momentum):
        t[0][..., 17] = 0
        t[1][2] = 0
        t[2][1] = 0
    net.grads[0][3, 4, 20], net.momentum[0][0, 0, 21], net.grads[1][3, 1, 1], net.grads[2][2, 69, 49] = np.nan, np.inf, -np.inf, np.nan
    for t in (net.grads, net.momentum):                   # 1e15 and 1e-15 (of which eps is much), and 1e30: squares beyond floats
        t[0][..., 22] *= np.float32(1e15)
        t[0][..., 23] *= np.float32(1e-15)
        t[0][..., 24] *= np.float32(1e30)
        t[1][4] *= np.float32(1e30)
        t[2][3] *= np.float32(1e30)
        t[3] *= np.float32(1e-4)
    got, _ = net.run()
    assert np.all(got[0][..., 17] == 0) and np.all(got[1][2] == 0) and np.all(got[2][1] == 0)
    assert np.all(np.isnan(got[0][..., 20].real)) and np.all(np.isnan(got[0][..., 21].real)) and np.all(np.isnan(got[1][3])) and np.all(np.isnan(got[2][2]))
    for k, at in ((0, (Ellipsis, 22)), (0, (Ellipsis, 24)), (1, (4,)), (2, (3,)), (3, ())):
        assert np.linalg.norm(got[k][at] - clean[k][at]) <= 1e-3 * np.linalg.norm(clean[k][at]), (k, at)
    assert np.all(np.abs(got[0][..., 23]) < 1e-4)            # 485 |u| / eps
    keep = [n for n in range(40) if n not in (17, 20, 21, 22, 23, 24)]
    assert np.array_equal(got[0][..., keep], clean[0][..., keep])
    assert np.array_equal(got[1][:2], clean[1][:2]) and np.array_equal(got[2][0], clean[2][0])


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", [[((20, 20, 900), True), ((20, 5), False)], [((300, 200), False), ((2, 64, 64), False), ((40, 700), False)]])
def test_the_same_bits_on_every_run_and_on_another_stream_and_in_a_graph(shapes):
    net = Muon(shapes, seed=10)
    first = sum(net.run(zero=False, lr=0.1), [])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert all(np.array_equal(a, b) for a, b in zip(sum(net.run(zero=False, lr=0.1, ws_fill=0), []), first))
    ws = B.alloc_muon_workspace(net.list)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.fno_muon_step(net.list, 0.1, 0.9, ws)
    start = [torch.from_numpy(t.copy()).cuda() for t in net.params + net.momentum]
    for k in range(4):
        for g in net.dg:
            g.mul_(1.0 + k)
        results = []
        for go in (lambda: B.fno_muon_step(net.list, 0.1, 0.9, ws), graph.replay):
            for t, s in zip(net.dp + net.dm, start):
                t.copy_(s)
            ws.fill_(255)
            go()
            torch.cuda.synchronize()
            results.append([t.clone() for t in net.dp + net.dm])
        assert all(torch.equal(a, b) for a, b in zip(*results)), k


@pytest.mark.gpu
def test_nothing_is_written_past_a_tensor():
    for shape, is_complex in (((13, 9, 21), True), ((70, 41), False), ((3, 19, 7), False), ((20, 20, 16), True)):
        net = Muon([(shape, is_complex)], seed=11)
        n = net.params[0].size
        flat = [torch.full((n + 64,), 3.0, device="cuda", dtype=torch.complex64 if is_complex else torch.float32) for _ in range(3)]
        for t, src in zip(flat, (net.params[0], net.grads[0], net.momentum[0])):
            t[:n] = torch.from_numpy(src.copy()).reshape(-1).cuda()
        views = [[t[:n].view(shape)] for t in flat]
        tensors = B.make_muon_tensors(*views)
        need = B.fno_muon_workspace_bytes(tensors)
        ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
        B.fno_muon_step(tensors, 0.1, 0.9, ws[: max(need, 256)])
        torch.cuda.synchronize()
        assert all(torch.all(t[n:] == 3.0) for t in flat) and torch.all(ws[max(need, 256):] == 77)
        assert torch.equal(flat[1][:n].cpu(), torch.from_numpy(net.grads[0].copy()).reshape(-1))


@pytest.mark.gpu
def test_tensors_at_odd_addresses():
    """Four bytes (complex: eight) are all the alignment that the call asks for."""
    for shape in ((50, 70), (20, 20), (3, 64, 64), (129, 300)):
        net = Muon([(shape, False)], seed=12)
        aligned = net.run(zero=False)
        n = net.params[0].size
        flat = [torch.zeros(n + 3, device="cuda") for _ in range(3)]
        views = []
        for off, t, src in zip((1, 2, 3), flat, (net.params[0], net.grads[0], net.momentum[0])):
            v = t[off:off + n] if off + n <= n + 3 else None
            v.copy_(torch.from_numpy(src.copy()).reshape(-1))
            views.append([v.view(shape)])
        tensors = B.make_muon_tensors(*views, scale=-1.0)
        B.fno_muon_step(tensors, 1.0, 0.9, B.alloc_muon_workspace(tensors))
        torch.cuda.synchronize()
        assert np.array_equal(views[0][0].cpu().numpy(), aligned[0][0]) and np.array_equal(views[2][0].cpu().numpy(), aligned[1][0])


@pytest.mark.gpu
def test_gradients_alone_for_the_norm():
    net = Muon(NETWORK, seed=13)
    grads = [torch.from_numpy(g.copy()).cuda() for g in net.grads]
    tensors = B.make_grad_tensors(grads)
    out, ws = torch.empty(1, device="cuda"), B.alloc_grad_norm_workspace(tensors)
    B.fno_grad_norm(tensors, out, ws)
    ref = np.sqrt(sum(float((np.abs(g.astype(np.complex128)) ** 2).sum()) for g in net.grads))
    assert abs(float(out) - ref) <= 2 * U * ref
    with pytest.raises(B.FnoError):                         # no parameters to move
        B.fno_adamw_step(tensors, 1e-3, 0.9, 0.999, 1e-8, 1)


# ------------------------------------------------------------------------------------------ refusals, without a device

def _tensor(**kw):
    d = dict(param=1 << 20, grad=1 << 21, momentum=1 << 22, batch=3, rows=20, cols=20, kind=0, scale=1.0, weight_decay=0.0)
    d.update(kw)
    return B.FnoMuonTensor(*(d[k] for k in ("param", "grad", "momentum", "batch", "rows", "cols", "kind", "scale", "weight_decay")))


def _step(tensors, options=(), norm=None, max_norm=1.0, ws=1 << 30, size=1 << 50, count=None):
    o = dict(lr=0.1, momentum=0.9, eps=1e-7, a=3.4, b=-4.7, c=2.0, iterations=5, nesterov=1)
    o.update(options)
    opt = B.FnoMuonOptions(*(o[k] for k in ("lr", "momentum", "eps", "a", "b", "c", "iterations", "nesterov")))
    array = (B.FnoMuonTensor * max(len(tensors), 1))(*tensors)
    return B.lib().fno_muon_step(len(tensors) if count is None else count, array, ctypes.addressof(opt), norm, max_norm, ws, size, None)


NAN, INF = float("nan"), float("inf")
BAD = [(dict(batch=-1), B.FNO_EINVAL), (dict(rows=-2), B.FNO_EINVAL), (dict(cols=-2), B.FNO_EINVAL), (dict(kind=2), B.FNO_EINVAL),
       (dict(kind=-1), B.FNO_EINVAL), (dict(scale=NAN), B.FNO_EINVAL), (dict(weight_decay=INF), B.FNO_EINVAL), (dict(param=None), B.FNO_EINVAL),
       (dict(grad=None), B.FNO_EINVAL), (dict(momentum=None), B.FNO_EINVAL), (dict(param=(1 << 20) + 2), B.FNO_EINVAL),
       (dict(grad=(1 << 20) + 4, kind=1), B.FNO_EINVAL), (dict(rows=33, kind=1), B.FNO_EUNSUPPORTED), (dict(cols=33, kind=1), B.FNO_EUNSUPPORTED),
       (dict(rows=32769), B.FNO_EUNSUPPORTED), (dict(batch=2 ** 31), B.FNO_EUNSUPPORTED), (dict(batch=2 ** 30, rows=32768), B.FNO_EUNSUPPORTED)]


@pytest.mark.parametrize("change,status", BAD)
def test_tensors_that_are_refused(change, status):
    bad = _tensor(**change)
    assert _step([_tensor(), bad]) == status
    if change.keys() & {"batch", "rows", "cols", "kind", "scale", "weight_decay"} and not change.keys() & {"grad"}:
        n = ctypes.c_size_t(0)
        assert B.lib().fno_muon_workspace_bytes(ctypes.c_int32(1), (B.FnoMuonTensor * 1)(bad), ctypes.byref(n)) == status


@pytest.mark.parametrize("options", [dict(lr=NAN), dict(lr=INF), dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=NAN), dict(eps=-1.0), dict(eps=INF),
                                     dict(a=NAN), dict(b=INF), dict(c=NAN), dict(iterations=-1), dict(iterations=65), dict(nesterov=2)])
def test_options_that_are_refused(options):
    assert _step([_tensor()], options) == B.FNO_EINVAL


def test_calls_that_are_refused():
    big = _tensor(rows=300, cols=200)
    n = ctypes.c_size_t(0)
    assert B.lib().fno_muon_workspace_bytes(ctypes.c_int32(1), (B.FnoMuonTensor * 1)(big), ctypes.byref(n)) == B.FNO_OK and n.value > 0
    assert _step([big], ws=None) == B.FNO_EINVAL
    assert _step([big], ws=(1 << 30) + 128) == _step([big], size=n.value - 1) == B.FNO_ENOSPC
    assert _step([_tensor()], norm=1 << 23, max_norm=0.0) == _step([_tensor()], norm=1 << 23, max_norm=NAN) == B.FNO_EINVAL
    assert _step([], count=-1) == B.FNO_EINVAL
    assert B.lib().fno_muon_step(1, None, None, None, 1.0, None, 0, None) == B.FNO_EINVAL
    assert B.lib().fno_muon_workspace_bytes(ctypes.c_int32(0), None, None) == B.FNO_EINVAL
    assert _step([]) == B.FNO_OK and _step([_tensor(batch=0, param=None)]) == B.FNO_OK         # nothing to do
    assert _step([_tensor(rows=0, param=None), _tensor(cols=0, grad=None)], ws=None, size=0) == B.FNO_OK


@pytest.mark.gpu
def test_the_binding_refuses_tensors_that_do_not_fit():
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)
    good = z(4, 5)
    for p, g, m in ((z(5), z(5), z(5)), (z(2, 2, 2, 2), z(2, 2, 2, 2), z(2, 2, 2, 2)), (good, z(5, 4), good), (good, good, good.bfloat16()),
                    (z(4, 5, dtype=torch.complex64), good, good), (z(5, 4).t(), good, good), (good, good.cpu(), good),
                    (good.to(torch.float64), good.to(torch.float64), good.to(torch.float64))):
        with pytest.raises(ValueError):
            B.make_muon_tensors([p], [g], [m])
    with pytest.raises(ValueError):
        B.make_muon_tensors([good], [good], [])
    with pytest.raises(ValueError):
        B.make_muon_tensors([good], [z(4, 5)], [z(4, 5)], scale=[1.0, 2.0])
    tensors = B.make_muon_tensors([good], [z(4, 5)], [z(4, 5)])
    with pytest.raises(ValueError):
        B.fno_muon_step(tensors, 0.1, 0.9, B.alloc_muon_workspace(tensors), grad_norm=torch.zeros(2, device="cuda"))


@pytest.mark.gpu
def test_the_binding_refuses_a_tensor_twice_and_lazy_views():
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)
    p, other = z(4, 5), z(4, 5)
    for params, momentum in (([p, p], [z(4, 5), z(4, 5)]), ([p, other], [z(4, 5)] * 2), ([p, other], [z(4, 5), p])):
        with pytest.raises(ValueError, match="already"):
            B.make_muon_tensors(params, [z(4, 5), z(4, 5)], momentum)
    B.make_muon_tensors([z(0, 5), z(0, 5)], [z(0, 5)] * 2, [z(0, 5)] * 2)
    g = z(4, 5)
    B.make_muon_tensors([p, other], [g, g], [z(4, 5), z(4, 5)])                   # a gradient that is only read may be
    c = lambda: z(3, 4, 5, dtype=torch.complex64)
    for bad in (([c().conj()], [c()], [c()]), ([c()], [c().conj()], [c()]), ([c()], [c()], [c().conj()]), ([p], [torch._neg_view(g)], [other])):
        with pytest.raises(ValueError, match="view"):
            B.make_muon_tensors(*bad)


@pytest.mark.gpu
def test_graphs_of_kernels_that_ask_for_local_memory():
    """More than 64 KB a block is asked of the runtime by every call, a captured one too."""
    net = Muon([((32, 32, 40), True), ((32, 512), False), ((24, 31, 9), True)], seed=22)
    eager = net.run(zero=False, lr=0.1)
    for t, s in zip(net.dp + net.dm, net.params + net.momentum):
        t.copy_(torch.from_numpy(s))
    tensors = B.make_muon_tensors(net.dp, net.dg, net.dm, scale=-1.0)
    ws, graph = B.alloc_muon_workspace(tensors), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.fno_muon_step(tensors, 0.1, 0.9, ws)
    for _ in range(3):
        for t, s in zip(net.dp + net.dm, net.params + net.momentum):
            t.copy_(torch.from_numpy(s))
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(t.cpu().numpy(), r) for t, r in zip(net.dp + net.dm, eager[0] + eager[1]))
