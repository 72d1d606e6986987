"""Training of a network whose blocks are normalised, nu_{k+1} = gelu(groupnorm(W nu_k + b + K(phi) nu_k)): group norm, the
norm of all gradients and AdamW beside the library's other calls, as a program runs them.

The gradients pass through two blocks, two norms and three pointwise stages in float32: 5e-5 of their norm, as for the plain
network; the loss and the output 1e-5."""
import numpy as np
import pytest
import torch

from oracle import fno_oracle as O
from paper_2204_01205_amd import binding as B
from paper_2204_01205_amd import synth

TOL, EPS = 1e-5, 1e-5


def rel(a, b):
    a, b = a.detach().cpu().numpy() if isinstance(a, torch.Tensor) else np.asarray(a), np.asarray(b)
    return float(np.linalg.norm((a - b).ravel()) / max(np.linalg.norm(b.ravel()), 1e-300))


class Network:
    grid, modes, batch, c_in, width, hidden, nblocks, groups = (8, 10, 6, 8), (2, 3, 2, 3), 2, 3, 8, 16, 2, 2

    def __init__(self):
        self.spec = O.LayerSpec(self.grid, self.modes, 0)
        self.counts = tuple(len(k) for k in O.mode_lists(self.spec))
        self.npts = int(np.prod(self.grid))
        w, rng = self.width, np.random.default_rng(5)
        self.a = synth.normal_field(0, synth.T_X, self.batch, self.c_in, self.grid)
        self.y = synth.normal_field(1, synth.T_TARGET, self.batch, 1, self.grid)
        # lift W, b; projection W1, b1, W2, b2; then R, W, b, gamma, beta of every block
        self.params = [synth.linear_weights(0, w, self.c_in, synth.T_LIFT), synth.bias(0, w, synth.T_LIFT),
                       synth.linear_weights(1, self.hidden, w, synth.T_PROJ), synth.bias(1, self.hidden, synth.T_PROJ),
                       synth.linear_weights(2, 1, self.hidden, synth.T_PROJ), synth.bias(2, 1, synth.T_PROJ)]
        for k in range(self.nblocks):
            self.params += [synth.spectral_weights(k, w, w, self.counts), synth.linear_weights(10 + k, w, w), synth.bias(10 + k, w),
                            (1 + 0.2 * rng.standard_normal(w)).astype(np.float32), (0.2 * rng.standard_normal(w)).astype(np.float32)]

    def blocks(self, flat):
        return [tuple(flat[6 + 5 * k: 11 + 5 * k]) for k in range(self.nblocks)]

    def oracle(self):
        """Output and gradients of every parameter, in float64."""
        lw, lb, w1, b1, w2, b2 = self.params[:6]
        vs, saved = [O.pointwise_linear(self.a, lw, lb)], []
        for R, W, b, ga, be in self.blocks(self.params):
            z = O.block_fwd(vs[-1], R, W, b, self.spec, "identity")[0]
            v, mean, rstd = O.group_norm_fwd(z, ga, be, self.groups, EPS, "gelu")
            saved.append((z, mean, rstd))
            vs.append(v)
        u = O.pointwise_mlp2(vs[-1], w1, b1, w2, b2)
        gp = O.pointwise_mlp2_bwd(vs[-1], w1, b1, w2, O.rel_l2_grad(u, self.y))
        grads, gv = [None] * len(self.params), gp["gx"]
        grads[2:6] = gp["gW1"], gp["gb1"], gp["gW2"], gp["gb2"]
        for k in reversed(range(self.nblocks)):
            R, W, b, ga, be = self.blocks(self.params)[k]
            z, mean, rstd = saved[k]
            gn = O.group_norm_bwd(z, ga, be, mean, rstd, self.groups, gv, "gelu")
            g = O.block_bwd(vs[k], R, W, b, gn["gx"], self.spec, "identity")
            grads[6 + 5 * k: 11 + 5 * k] = g["gR"], g["gW"], g["gb"], gn["ggamma"], gn["gbeta"]
            gv = g["gx"]
        lift = O.pointwise_linear_bwd(self.a, lw, gv)
        grads[0:2] = lift["gW"], lift["gb"]
        return u, grads

    def device(self, bits):
        """Everything that a program keeps on the GPU."""
        self.dp = [torch.from_numpy(p.copy()).cuda() for p in self.params]
        self.dg = [torch.empty_like(p) for p in self.dp]
        kind = torch.float32 if bits == 32 else torch.uint8
        sizes = [p.numel() * (2 if p.is_complex() else 1) for p in self.dp]
        self.m, self.v = ([torch.zeros(n, dtype=kind, device="cuda") for n in sizes] for _ in range(2))
        exps = None if bits == 32 else [torch.zeros(B.adamw_exps_shape(n), dtype=torch.uint8, device="cuda") for n in sizes]
        self.decay = [0.01 if p.ndim > 1 else 0.0 for p in self.params]
        self.list = B.make_adamw_tensors(self.dp, self.dg, self.m, self.v, exps, self.decay)
        w, field = self.width, (self.batch, self.width) + self.grid
        self.desc = B.make_desc(self.batch, w, w, self.grid, self.modes, 0, B.FNO_ACT_IDENTITY)
        self.norm = B.make_norm_desc(self.batch, w, self.groups, self.npts, activation=B.FNO_ACT_GELU, eps=EPS)
        self.ws, self.nws = B.alloc_workspace(self.desc, B.FNO_OP_BLOCK_BWD), B.alloc_norm_workspace(self.norm)
        self.da, self.dy = torch.from_numpy(self.a).cuda(), torch.from_numpy(self.y).cuda()
        self.vs = [torch.empty(field, device="cuda") for _ in range(self.nblocks + 1)]
        self.zs = [torch.empty(field, device="cuda") for _ in range(self.nblocks)]
        self.xh = [torch.empty((self.batch, w) + self.counts, dtype=torch.complex64, device="cuda") for _ in range(self.nblocks)]
        self.stats = [[torch.empty(self.batch, self.groups, device="cuda") for _ in range(2)] for _ in range(self.nblocks)]
        self.gv = [torch.empty(field, device="cuda") for _ in range(2)]
        self.u, self.loss, self.gnorm = torch.empty_like(self.dy), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
        self.gu = torch.empty_like(self.u)
        self.lws = torch.empty(B.fno_rel_l2_workspace_bytes() // 4, device="cuda")
        self.pws = torch.empty(max(B.fno_pointwise_bwd_workspace_bytes(w, self.hidden, 1),
                                   B.fno_pointwise_bwd_workspace_bytes(self.c_in, 0, w)) // 4 + 2, device="cuda")
        self.gws = B.alloc_grad_norm_workspace(self.list)

    def step(self, number, lr, max_norm):
        n, w, p, g = self.npts, self.width, self.dp, self.dg
        B.fno_pointwise_linear(self.batch, self.c_in, w, n, self.da, p[0], p[1], self.vs[0])
        for k, (R, W, b, ga, be) in enumerate(self.blocks(p)):
            B.fno_block_fwd(self.desc, self.vs[k], R, W, b, self.zs[k], None, self.xh[k], self.ws)
            B.fno_group_norm_fwd(self.norm, self.zs[k], ga, be, self.vs[k + 1], *self.stats[k], self.nws)
        B.fno_pointwise_mlp2(self.batch, w, self.hidden, 1, n, self.vs[-1], *p[2:6], self.u)
        B.fno_rel_l2_loss(self.u.numel(), self.u, self.dy, self.loss, self.gu, self.lws)
        gin, gout = self.gv
        B.fno_pointwise_mlp2_bwd(self.batch, w, self.hidden, 1, n, self.vs[-1], p[2], p[3], p[4], self.gu, gin, *g[2:6], self.pws)
        for k in reversed(range(self.nblocks)):
            (R, W, b, ga, be), (gR, gW, gb, gga, gbe) = self.blocks(p)[k], self.blocks(g)[k]
            B.fno_group_norm_bwd(self.norm, self.zs[k], ga, be, *self.stats[k], gin, gin, gga, gbe, self.nws)
            B.fno_block_bwd(self.desc, self.vs[k], R, W, self.zs[k], self.xh[k], gin, gout, gR, gW, gb, self.ws)
            gin, gout = gout, gin
        B.fno_pointwise_linear_bwd(self.batch, self.c_in, w, n, self.da, p[0], gin, None, g[0], g[1], self.pws)
        B.fno_grad_norm(self.list, self.gnorm, self.gws)
        B.fno_adamw_step(self.list, lr, 0.9, 0.999, 1e-8, number, grad_norm=self.gnorm, max_norm=max_norm, seed=7)


@pytest.mark.gpu
def test_training_step_of_a_normalised_network_matches_the_oracle():
    net = Network()
    net.device(32)
    net.step(1, 1e-3, 0.1)
    torch.cuda.synchronize()
    u, grads = net.oracle()
    assert rel(net.u, u) <= TOL
    assert abs(float(net.loss) - O.rel_l2_loss(u, net.y)) <= TOL * O.rel_l2_loss(u, net.y)
    for k, (g, ref) in enumerate(zip(net.dg, grads)):
        assert rel(g, ref) <= 5 * TOL, k
    norm = np.sqrt(sum((np.abs(g) ** 2).sum() for g in grads))
    assert abs(float(net.gnorm) - norm) <= TOL * norm and norm > 0.1
    for k, (p, start, g) in enumerate(zip(net.dp, net.params, grads)):
        as_real = lambda t: np.ascontiguousarray(t, np.complex128).view(np.float64) if np.iscomplexobj(t) else np.asarray(t, np.float64)
        ref, _, _ = O.adamw_step(as_real(start), as_real(g), 0.0, 0.0, 1, weight_decay=net.decay[k], scale=0.1 / norm)
        got = torch.view_as_real(p).reshape(-1) if p.is_complex() else p
        # the first step is lr g / (|g| + eps): a gradient off by 5e-5 of its tensor's norm moves few entries, by 2 lr at most
        got, ref = got.cpu().numpy().ravel(), ref.ravel()
        assert np.linalg.norm(got - ref) <= 1e-3 * 2 * 0.05 * np.sqrt(ref.size), k
        assert np.all(np.abs(got - as_real(start).ravel()) <= 1e-3 * 1.001 + 1e-5 * np.abs(as_real(start).ravel()) + 1e-7)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_normalised_network_learns(bits):
    """60 steps on one batch: the loss falls to a tenth less than it started from, the same way with 8-bit moments."""
    net = Network()
    net.device(bits)
    losses = []
    for number in range(1, 61):
        net.step(number, 3e-3, 1.0)
        losses.append(float(net.loss))
    assert np.isfinite(losses).all() and losses[-1] < 0.9 * losses[0], losses[::10]
    assert all(torch.isfinite(p.abs()).all() for p in net.dp)


def test_the_oracle_network_differentiates_its_own_forward():
    net = Network()
    u, grads = net.oracle()
    rng = np.random.default_rng(2)
    for k in (0, 2, 7, 8, 9, 10, 14):
        p = net.params[k].astype(np.float64)
        step = rng.standard_normal(p.shape)
        values = []
        for sign in (1, -1):
            keep = net.params[k]
            net.params[k] = p + sign * 1e-5 * step
            values.append(O.rel_l2_loss(net.oracle()[0], net.y))
            net.params[k] = keep
        diff, want = (values[0] - values[1]) / 2e-5, float((grads[k] * step).sum())
        assert abs(diff - want) <= 1e-6 * max(1.0, abs(want)) + 1e-5 * abs(want), (k, diff, want)
