"""The Muon step of larger real matrices, in tiles of 64 and of 128, as closely as its arithmetic allows.

The tolerance is the error of a plain program with the same roundings: X, A and B as sums of two fp16 values, three of the four
products of such pairs, sums in float 16 terms at a time.  It has every rounding that the kernels have; what differs is the order
within the 16 terms and where a split sum is put together, so signs and not sizes.  Both errors are norms over a thousand entries or more
of sums of independent roundings, which lie close to their root mean square: 4 times the program's error is out of their reach.  What a lost
second part or cross term makes of the result is far beyond the limit, in one of the three products alone too: the test without a device
asks for 30 limits.

Momenta: three roundings of their terms."""
import numpy as np
import pytest
import torch

from oracle import fno_oracle as O
from paper_2204_01205_amd import binding as B
from test_gpu_muon import Muon, U, bounds, stack

QUINTIC = (3.4445, -4.7750, 2.0315)
KX, KA, KB = 1024.0, 256.0, 64.0
MU = 0.9

# Tiles of 128: shorter sides above 192, and enough of them in the list; else tiles of 64.
WIDE = [((1000, 4100), False)]
TALL = [((4100, 1000), False)]
STACK = [((9, 1023, 1025), False)]
AT_LEAST = [((1024, 4000), False)]                       # 36 tiles of a symmetric product, 128 steps each
BELOW = [((1024, 3968), False)]                          # 124 steps
SQUARES = [((4, 1024, 1024), False), ((1000, 1536), False)]
ONE = [((1640, 1660), False)]                             # 169 tiles of the last product, whose sums are split too
MIXED = [((150, 700), False), ((1000, 4100), False), ((4, 64, 65), False), ((20, 20, 33), True), ((193, 257), False), ((192, 900), False),
         ((2, 300, 250), False), ((20, 128), False)]
IN_128 = dict(wide=WIDE, tall=TALL, stack=STACK, at_least=AT_LEAST, squares=SQUARES, one=ONE, mixed=MIXED)
IN_64 = [(33, 33), (33, 40), (48, 200), (64, 64), (65, 64), (96, 130), (129, 128), (200, 333), (256, 256), (37, 512), (1000, 36), (257, 600), (512, 384),
         (192, 1000)]


def is_dense(t):
    return not np.iscomplexobj(t) and (min(t.shape[-2:]) > 32 or t.shape[-2] * t.shape[-1] > 16384)


def what_is_orthogonalised(g, m, mu=MU):
    """In 64 bits, and in the kernels' float."""
    fine = g + mu * (mu * m.astype(np.float64) + g)
    mu = np.float64(np.float32(mu))
    new = (mu * m + g).astype(np.float32)
    return fine, (mu * new + g).astype(np.float32)


def same_roundings(u, iterations=5, coefficients=QUINTIC, eps=1e-7, lost="", where=(0, 1, 2)):
    """X of the matrix u (float32), rows no more than columns.  lost: a mistake to plant in the products `where`."""
    a, b, c = (float(np.float32(v)) for v in coefficients)

    def parts(v):
        first = v.half().float()
        return first, (v - first).half().float()

    def product(which, left, right):                     # left right^T
        out = torch.zeros(len(left[0]), len(right[0]))
        gone = lost if which in where else ""
        for k in range(0, left[0].shape[1], 16):
            lf, ls, rf, rs = (t[:, k:k + 16] for t in left + right)
            out += lf @ rf.t()
            if gone not in ("second parts", "right cross term"):
                out += lf @ rs.t()
            if gone not in ("second parts", "left cross term"):
                out += ls @ rf.t()
        return out

    u = torch.from_numpy(u.T.copy() if u.shape[0] > u.shape[1] else u)
    v = (u.double() / (u.double().square().sum().sqrt() + eps)).float() * KX
    for _ in range(iterations):
        x = parts(v)
        A = parts(product(0, x, x) * (KA / KX ** 2))
        B_ = parts((b * KB / KA) * (A[0] + A[1]) + (c * KB / KA ** 2) * product(1, A, A))
        v = a * (x[0] + x[1]) + product(2, B_, tuple(t.t().contiguous() for t in x)) * (1 / KB)
    return (v / KX).double().numpy()


def off(x, ref):
    return np.linalg.norm((x if x.shape == ref.shape else x.T) - ref)


def check(net, iterations=5, coefficients=QUINTIC):
    got_p, got_m = net.run(mu=MU, iterations=iterations, coefficients=coefficients)
    for k, (p, m) in enumerate(zip(got_p, got_m)):
        g, old = net.grads[k], net.momentum[k]
        wide = np.complex128 if np.iscomplexobj(m) else np.float64
        assert np.all(np.abs(m - (MU * old.astype(wide) + g)) <= 4 * U * (MU * np.abs(old) + np.abs(g))), k
        if not is_dense(p):
            u = stack(g + MU * (MU * old.astype(wide) + g))
            error = np.sqrt((np.abs(stack(p) - O.newton_schulz(u, iterations, coefficients)) ** 2).sum((1, 2)))
            assert np.all(error <= bounds(u, iterations)), k
            continue
        for j, (x, gj, mj) in enumerate(zip(stack(p), stack(g), stack(old))):
            fine, u = what_is_orthogonalised(gj, mj)
            ref = O.newton_schulz(fine, iterations, coefficients)
            error, limit = off(x, ref), 4 * off(same_roundings(u, iterations, coefficients), ref)
            assert error <= limit, (k, j, p.shape, error / limit)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", IN_64, ids=lambda s: f"{s[0]}x{s[1]}")
def test_tiles_of_64(shape):
    check(Muon([(shape, False)], seed=31 + shape[0]))


@pytest.mark.gpu
@pytest.mark.parametrize("which", sorted(IN_128))
def test_tiles_of_128(which):
    check(Muon(IN_128[which], seed=32))


@pytest.mark.gpu
def test_just_below_tiles_of_128():
    check(Muon(BELOW, seed=33))


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", [[((257, 600), False), ((512, 384), False), ((70, 90), False)], WIDE, TALL], ids=["64", "128 wide", "128 tall"])
def test_a_convergent_polynomial_makes_a_matrix_orthogonal(shapes):
    """Singular values from 1 to 2 (before they are divided by the norm) end at one: six doublings at most, and quadratic steps.  An error e
    of X leaves 2 e in its Gram matrix."""
    net = Muon(shapes, seed=34)
    rng = np.random.default_rng(34)
    for k, (shape, _) in enumerate(shapes):
        m, n = min(shape), max(shape)
        left, right = np.linalg.qr(rng.standard_normal((m, m)))[0], np.linalg.qr(rng.standard_normal((n, m)))[0]
        q = (left * np.linspace(1, 2, m)) @ right.T
        net.momentum[k] = np.ascontiguousarray(q if shape[0] <= shape[1] else q.T).astype(np.float32)
        net.grads[k] = np.zeros_like(net.grads[k])
    coefficients, iterations = (2.0, -1.5, 0.5), 18
    check(net, iterations, coefficients)
    for p in net.dp:
        x = p.cpu().numpy().astype(np.float64)
        x = x if x.shape[0] <= x.shape[1] else x.T
        gram = x @ x.T - np.eye(len(x))
        # of the last iteration: 3 n / 16 and 3 m / 16 additions to sums of at most 1, and a handful of values of at most 1 in 22 bits (4 U)
        assert np.abs(gram).max() <= 2 * U * (3 * sum(x.shape) / 16 + 16)


@pytest.mark.gpu
@pytest.mark.parametrize("nesterov", [True, False])
def test_no_iterations_in_tiles_of_128(nesterov):
    net = Muon(MIXED, seed=35)
    got, _ = net.run(mu=MU, iterations=0, nesterov=nesterov)
    for k, p in enumerate(got):
        g, m = stack(net.grads[k]), stack(net.momentum[k]).astype(np.complex128 if np.iscomplexobj(p) else np.float64)
        new = MU * m + g
        u = g + MU * new if nesterov else new
        size = np.abs(g) + np.abs(m) + np.abs(new)                     # the terms, of which u may be a small difference
        norm = np.sqrt((np.abs(u) ** 2).sum((1, 2), keepdims=True))
        # mu and two additions, twice, and the quotient; the squares of spectral weights are added in float, some 50 in a chain
        assert np.all(np.abs(stack(p) - u / (norm + 1e-7)) <= (8 if is_dense(net.params[k]) else 32) * U * size / norm), k


@pytest.mark.gpu
def test_zeros_nans_and_sizes_stay_with_their_matrix_in_tiles_of_128():
    net = Muon([((5, 1023, 1025), False), ((1, 200, 210), False)], seed=36)
    clean, _ = net.run()
    for t in (net.grads, net.momentum):
        t[0][1] = 0
        t[0][3] *= np.float32(1e30)                       # squares beyond floats
    net.grads[0][2, 1022, 1024] = np.nan
    got, _ = net.run()
    assert np.all(got[0][1] == 0) and np.all(np.isnan(got[0][2]))
    assert np.array_equal(got[0][0], clean[0][0]) and np.array_equal(got[0][4], clean[0][4]) and np.array_equal(got[1], clean[1])
    assert np.linalg.norm(got[0][3] - clean[0][3]) <= 1e-3 * np.linalg.norm(clean[0][3])


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", [MIXED, STACK], ids=["mixed", "stack"])
def test_the_same_bits_in_replays_of_a_graph_in_tiles_of_128(shapes):
    net = Muon(shapes, seed=37)
    first = sum(net.run(zero=False, lr=0.1), [])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert all(np.array_equal(a, b) for a, b in zip(sum(net.run(zero=False, lr=0.1, ws_fill=0), []), first))
    ws, graph = B.alloc_muon_workspace(net.list), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.fno_muon_step(net.list, 0.1, MU, ws)
    start = [torch.from_numpy(t.copy()).cuda() for t in net.params + net.momentum]
    for k in range(3):
        for g in net.dg:
            g.mul_(1.0 + k)
        results = []
        for go in (lambda: B.fno_muon_step(net.list, 0.1, MU, ws), graph.replay):
            for t, s in zip(net.dp + net.dm, start):
                t.copy_(s)
            ws.fill_(255)
            go()
            torch.cuda.synchronize()
            results.append([t.clone() for t in net.dp + net.dm])
        assert all(torch.equal(a, b) for a, b in zip(*results)), k


@pytest.mark.gpu
def test_clipping_and_norms_that_are_not_finite_in_tiles_of_128():
    net = Muon(WIDE + [((100, 70), False)], seed=38)
    plain, _ = net.run(zero=False, lr=0.1)
    same, _ = net.run(zero=False, lr=0.1, norm=0.5)
    assert all(np.array_equal(a, b) for a, b in zip(plain, same))
    clipped = sum(net.run(zero=False, norm=8.0, max_norm=2.0), [])
    p, m = net.run(zero=False, norm=float("inf"))
    net.grads = [0.25 * g for g in net.grads]             # a power of two: the same bits
    assert all(np.array_equal(a, b) for a, b in zip(clipped, sum(net.run(zero=False), [])))
    assert all(np.array_equal(a, b) for a, b in zip(p + m, net.params + net.momentum))


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1000, 4100), (4100, 1001)])
def test_nothing_is_written_past_a_tensor_or_its_workspace_in_tiles_of_128(shape):
    net = Muon([(shape, False)], seed=39)
    n = net.params[0].size
    flat = [torch.full((n + 64,), 3.0, device="cuda") for _ in range(3)]
    for t, src in zip(flat, (net.params[0], net.grads[0], net.momentum[0])):
        t[:n] = torch.from_numpy(src.copy()).reshape(-1).cuda()
    tensors = B.make_muon_tensors(*[[t[:n].view(shape)] for t in flat])
    need = B.fno_muon_workspace_bytes(tensors)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    B.fno_muon_step(tensors, 0.1, MU, ws[:need])
    torch.cuda.synchronize()
    assert all(torch.all(t[n:] == 3.0) for t in flat) and torch.all(ws[need:] == 77)
    assert torch.equal(flat[1][:n].cpu(), torch.from_numpy(net.grads[0].copy()).reshape(-1))


# ------------------------------------------------------------------------------------------ what the limit sees, without a device

@pytest.mark.parametrize("shape", IN_64 + [(1000, 1536)], ids=lambda s: f"{s[0]}x{s[1]}")
def test_a_lost_part_is_far_beyond_the_limit(shape):
    net = Muon([(shape, False)], seed=31 + shape[0])
    fine, u = what_is_orthogonalised(net.grads[0], net.momentum[0])
    ref = O.newton_schulz(fine)
    limit = 4 * off(same_roundings(u), ref)
    for lost in ("second parts", "left cross term", "right cross term"):
        for where in ((0, 1, 2), (0,), (1,), (2,)) if max(shape) <= 600 else ((0, 1, 2),):
            assert off(same_roundings(u, lost=lost, where=where), ref) >= 30 * limit, (lost, where)
