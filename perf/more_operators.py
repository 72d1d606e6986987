"""Layer norm and the Muon step, as measurable cases.

A case is one pass through one of them: layer norm with an activation over fields [B][C][P] or [B][P][C], whose statistics are
those of each point over its channels (forward, or backward with the gradients of gamma and beta), or one Muon step over all
matrices of a network: the momentum of every matrix, made orthogonal by a fixed number of Newton-Schulz products, moves the
weights.  The spectral weights of a block are one complex matrix for each kept mode.  `listed()` names the cases that stand for
the uses, `draw()` gives more of the same ranges, `prepare()` makes what a program holds before the call, `run()` is the pass, in
plain torch operations or through the library where `own` is set, `exact()` the definition in 64 bits and `work()` the bytes
and operations that a pass cannot do without.
"""
import math

import torch

own = False

ACTS = ("identity", "gelu", "silu")
EPS_NORM = 1e-5
LR, MOMENTUM, EPS, DECAY, MAX_NORM, ITERATIONS = 0.02, 0.95, 1e-7, 0.01, 1.0, 5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _norm(name, op, layout, dtype, act, batch, channels, points):
    """op ln_fwd or ln_bwd; layout "first" ([B][C][P]) or "last" ([B][P][C]); dtype of the fields "f32" or "bf16"."""
    case = dict(op=op, layout=layout, dtype=dtype, act=act, batch=batch, channels=channels, points=points)
    return case if name is None else dict(name=name, **case)


def _network(name, clip, c_in, width, hidden, blocks, counts):
    """The matrices of a network: lift c_in -> width, `blocks` blocks of width channels with counts[0..3] kept modes on
    x, y, z, t, projection width -> hidden -> 1.  clip: the gradients are scaled by their norm, which is part of the pass."""
    case = dict(op="muon", clip=clip, c_in=c_in, width=width, hidden=hidden, blocks=blocks, kx=counts[0], ky=counts[1],
                kz=counts[2], kt=counts[3])
    return case if name is None else dict(name=name, **case)


def _dense(name, clip, shapes):
    """Real matrices: "4*1024x1024,1000x1536" is a stack of four and one more."""
    case = dict(op="dense", clip=clip, shapes=shapes)
    return case if name is None else dict(name=name, **case)


def listed():
    return [
        # a small surrogate served with normalised points: bound by latency
        _norm("ln_16", "ln_fwd", "first", "f32", "gelu", 1, 8, 16 * 16 * 16 * 8),
        # a batch of features of the user's own model, channels last in 16 bits, an odd number of channels
        _norm("ln_last_odd", "ln_fwd", "last", "bf16", "silu", 4, 27, 28 * 24 * 20),
        # training on an odd grid, channels first
        _norm("ln_train_odd", "ln_bwd", "first", "f32", "gelu", 2, 12, 30 * 27 * 21 * 14 + 3),
        # training of wide rows in 16 bits, as a token mixer or a wide channel map has them
        _norm("ln_train_rows", "ln_bwd", "last", "bf16", "identity", 8, 1024, 4096),
        # one block's field at the paper's training samples, behind the spectral convolution
        _norm("ln_60", "ln_fwd", "first", "f32", "gelu", 1, 20, 60 * 60 * 64 * 30),
        # training at the grid of the benchmark network: the largest
        _norm("ln_train_128", "ln_bwd", "first", "f32", "gelu", 1, 20, 128 * 128 * 64 * 32),
        # the step of the smallest network: small matrices and 6144 modes of 8 x 8, clipping
        _network("muon_small", True, 5, 8, 32, 4, (8, 8, 8, 3)),
        # odd widths and kept modes of the symmetric rule, clipping
        _network("muon_odd", True, 3, 13, 37, 3, (13, 11, 9, 5)),
        # the network of the paper's training samples
        _network("muon_60", False, 2, 20, 128, 4, (24, 24, 24, 8)),
        # the benchmark network: the largest
        _network("muon_128", False, 5, 20, 128, 4, (32, 32, 24, 9)),
        # narrow dense layers of a user's own model, odd ones among them
        _dense("muon_dense_256", False, "6*256x256,2*1024x256,200x333,37x512"),
        # wide dense layers
        _dense("muon_dense_1024", False, "4*1024x1024,1024x4096,4096x1024,1000x1536"),
    ]


def draw(rng):
    """One more case of the same ranges: fields from one point to those of the benchmark network, networks from a few
    thousand parameters to those of the paper's samples, dense matrices from single rows to 4096 on a side."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.random()
        if kind < 0.5:
            op, layout, dtype = rng.choice(("ln_fwd", "ln_bwd")), rng.choice(("first", "last")), rng.choice(("f32", "bf16"))
            channels = rng.choice((rng.randint(4, 32), rng.choice((8, 16, 20, 32)), spread(32, 400 if layout == "first" else 8192)))
            batch, points = spread(1, 16), spread(1, 3.4e7)
            if batch * channels * points > 6.5e8:
                continue
            return _norm(None, op, layout, dtype, rng.choice(("gelu", "silu", "identity")), batch, channels, points)
        if kind < 0.8:
            width, hidden = rng.choice((8, 16, 20, 24, 32, rng.randint(4, 32))), rng.choice((32, 64, 128, rng.randint(8, 200)))
            counts = [rng.randint(4, 28) for _ in range(3)] + [rng.randint(2, 9)]
            case = _network(None, rng.random() < 0.5, rng.randint(1, 6), width, hidden, rng.choice((1, 2, 3, 4)), counts)
            if sum(math.prod(shape) for shape, _ in _shapes(case)) <= 4e8:
                return case
            continue
        shapes = []
        for _ in range(rng.randint(1, 5)):
            rows, cols = spread(1, 4096), spread(16, 4096)
            shapes.append(rng.choice((f"{rows}x{cols}", f"{rows}x{cols}", f"{rng.randint(2, 6)}*{rows}x{cols}")))
        case = _dense(None, rng.random() < 0.5, ",".join(shapes))
        if work(case)["flops"] <= work(listed()[-1])["flops"]:
            return case


def _shapes(case):
    """Shapes of a case's tensors, with the two parts of complex ones last, and whether they are complex.  Real: [rows][cols]
    or a stack of them; complex: [rows][cols] and the kept modes."""
    if case["op"] == "dense":
        out = []
        for text in case["shapes"].split(","):
            count, _, size = text.rpartition("*")
            rows, cols = (int(v) for v in size.split("x"))
            out.append(((rows, cols) if count == "" else (int(count), rows, cols), False))
        return out
    ci, w, h = case["c_in"], case["width"], case["hidden"]
    out = [((w, ci), False), ((h, w), False), ((1, h), False)]
    for _ in range(case["blocks"]):
        out += [((w, w, case["kx"], case["ky"], case["kz"], case["kt"], 2), True), ((w, w), False)]
    return out


def _matrices(shape, is_complex):
    """(count, rows, cols) of a tensor's matrices."""
    if is_complex:
        return math.prod(shape[2:-1]), shape[0], shape[1]
    return math.prod(shape[:-2]), shape[-2], shape[-1]


def _step_scale(rows, cols):
    """What a matrix's step is multiplied by, so that tall ones move as far as square ones."""
    return math.sqrt(max(1.0, rows / cols))


def _field_shape(case):
    b, c, p = case["batch"], case["channels"], case["points"]
    return (b, c, p) if case["layout"] == "first" else (b, p, c)


# ------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    return (_prepare_norm if case["op"].startswith("ln") else _prepare_muon)(case, normal)


def _prepare_norm(case, normal):
    c, shape = case["channels"], _field_shape(case)
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    # every channel has a mean and a scale of its own, as what comes out of a channel map has
    mean, scale = 0.5 + normal(c).abs_(), 0.5 + 0.5 * normal(c).abs_()
    if case["layout"] == "first":
        mean, scale = mean[:, None], scale[:, None]
    x = normal(*shape).mul_(scale).add_(mean).to(dtype)
    s = dict(case=case, x=x, gamma=1 + 0.2 * normal(c), beta=0.3 * normal(c))
    if case["op"] == "ln_fwd":
        s["y"] = torch.empty_like(x)
    else:
        s.update(gy=normal(*shape).to(dtype), gx=torch.empty_like(x), ggamma=torch.empty(c, device="cuda"),
                 gbeta=torch.empty(c, device="cuda"))
    if own:                      # the descriptor and the workspace that a program keeps
        from paper_2204_01205_amd import binding as B
        s["desc"] = B.make_layer_norm_desc(case["batch"], c, case["points"],
                                           layout=B.FNO_LAYOUT_CHANNELS_FIRST if case["layout"] == "first" else B.FNO_LAYOUT_CHANNELS_LAST,
                                           dtype=B.FNO_DTYPE_F32 if case["dtype"] == "f32" else B.FNO_DTYPE_BF16,
                                           activation=ACTS.index(case["act"]), eps=EPS_NORM)
        if case["op"] == "ln_bwd":
            s["ws"] = B.alloc_layer_norm_workspace(s["desc"])
    return s


def _prepare_muon(case, normal):
    shapes = _shapes(case)
    s = dict(case=case, params=[], grads=[], momentum=[], norm=torch.empty(1, device="cuda"),
             scale=[_step_scale(*_matrices(*sh)[1:]) for sh in shapes])
    for shape, is_complex in shapes:
        _, rows, cols = _matrices(shape, is_complex)
        # gradients that fall with the frequency along the modes of t, and momenta in the middle of a training run
        falloff = torch.logspace(0, -3, case["kt"], device="cuda")[:, None] if is_complex else 1.0
        tensors = (normal(*shape).mul_(0.5 / math.sqrt(cols)), normal(*shape).mul_(3e-3 * falloff),
                   normal(*shape).mul_(9e-3 * falloff))
        for name, t in zip(("params", "grads", "momentum"), tensors):
            s[name].append(torch.view_as_complex(t) if is_complex else t)
    if own:                      # the lists of tensors that a program keeps, and the scratch
        from paper_2204_01205_amd import binding as B
        s["list"] = B.make_muon_tensors(s["params"], s["grads"], s["momentum"], scale=s["scale"], weight_decay=DECAY)
        s["ws"] = B.alloc_muon_workspace(s["list"])
        if case["clip"]:
            s["norm_list"] = B.make_grad_tensors(s["grads"])
            s["norm_ws"] = B.alloc_grad_norm_workspace(s["norm_list"])
    return s


# ------------------------------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _own(s)
    return {"ln_fwd": _plain_norm_fwd, "ln_bwd": _plain_norm_bwd}.get(s["case"]["op"], _plain_muon)(s, s["case"])


def _own(s):
    from paper_2204_01205_amd import binding as B
    case = s["case"]
    if case["op"] == "ln_fwd":
        B.fno_layer_norm_fwd(s["desc"], s["x"], s["gamma"], s["beta"], s["y"])
        return s["y"]
    if case["op"] == "ln_bwd":
        B.fno_layer_norm_bwd(s["desc"], s["x"], s["gamma"], s["beta"], s["gy"], s["gx"], s["ggamma"], s["gbeta"], s["ws"])
        return s["gx"], s["ggamma"], s["gbeta"]
    norm = s["norm"] if case["clip"] else None
    if case["clip"]:
        B.fno_grad_norm(s["norm_list"], norm, s["norm_ws"])
    B.fno_muon_step(s["list"], LR, MOMENTUM, s["ws"], iterations=ITERATIONS, coefficients=COEFFICIENTS, eps=EPS, nesterov=True,
                    grad_norm=norm, max_norm=MAX_NORM)
    return _muon_outputs(s, case)


def _muon_outputs(s, case):
    """Parameters and momenta, complex ones as pairs of floats, and the norm where it is part of the pass."""
    out = {k: [torch.view_as_real(t) if t.is_complex() else t for t in s[k]] for k in ("params", "momentum")}
    if case["clip"]:
        out["norm"] = s["norm"]
    return out


# ------------------------------------------------------------------------------------------ plain forms

def _activation(act, z):
    if act == "identity":
        return z
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z / (1.0 + torch.exp(-z))


def _slope(act, z):
    if act == "identity":
        return torch.ones_like(z)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig))


def _standard(case, x):
    """xh and rstd of every point, and the axis of the channels."""
    axis = 1 if case["layout"] == "first" else 2
    d = x - x.mean(axis, keepdim=True)
    rstd = 1.0 / torch.sqrt(d.square().mean(axis, keepdim=True) + EPS_NORM)
    return d * rstd, rstd, axis


def _channelwise(case, v):
    return v[:, None] if case["layout"] == "first" else v


def _plain_norm_fwd(s, case):
    xh, _, _ = _standard(case, s["x"].float())
    return _activation(case["act"], xh * _channelwise(case, s["gamma"]) + _channelwise(case, s["beta"])).to(s["x"].dtype)


def _plain_norm_bwd(s, case):
    xh, rstd, axis = _standard(case, s["x"].float())
    gamma, beta = _channelwise(case, s["gamma"]), _channelwise(case, s["beta"])
    gz = s["gy"].float() * _slope(case["act"], xh * gamma + beta)
    points = 2 if axis == 1 else 1
    ggamma, gbeta = (gz * xh).sum(points).sum(0), gz.sum(points).sum(0)
    h = gz * gamma
    gx = rstd * (h - h.mean(axis, keepdim=True) - xh * (h * xh).mean(axis, keepdim=True))
    return gx.to(s["x"].dtype), ggamma, gbeta


def _stacked(t):
    """The matrices of a tensor as [count][rows][cols], and the way back."""
    if t.is_complex():
        rows, cols = t.shape[:2]
        return t.reshape(rows, cols, -1).permute(2, 0, 1), lambda x: x.permute(1, 2, 0).reshape(t.shape)
    return t.reshape(-1, *t.shape[-2:]), lambda x: x.reshape(t.shape)


def _adjoint(x):
    return (x.conj() if x.is_complex() else x).transpose(1, 2).contiguous().resolve_conj()


def _plain_muon(s, case):
    scale, fine = 1.0, None
    if case["clip"]:
        flat = [torch.view_as_real(g) if g.is_complex() else g for g in s["grads"]]
        norm = torch.stack([g.square().sum() for g in flat]).sum().sqrt()
        s["norm"].copy_(norm.reshape(1))
        scale = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))
        fine = torch.isfinite(norm)
    a, b, c = COEFFICIENTS
    for p, g, m, step in zip(s["params"], s["grads"], s["momentum"], s["scale"]):
        g = g * scale
        new = MOMENTUM * m + g
        u, back = _stacked(g + MOMENTUM * new)
        tall = u.shape[1] > u.shape[2]
        x = u.transpose(1, 2).contiguous() if tall else u.contiguous()
        size = (torch.view_as_real(x) if x.is_complex() else x).square().flatten(1).sum(1).sqrt()
        x = x / (size + EPS)[:, None, None]
        for _ in range(ITERATIONS):
            gram = torch.matmul(x, _adjoint(x))
            x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
        x = back(x.transpose(1, 2) if tall else x)
        moved = p * (1.0 - LR * DECAY) - LR * step * x
        for to, value in ((m, new), (p, moved)):       # a step whose norm is not finite changes nothing
            to.copy_(value if fine is None else torch.where(fine, value, to))
    return _muon_outputs(s, case)


# ------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    return {"ln_fwd": _exact_norm_fwd, "ln_bwd": _exact_norm_bwd}.get(case["op"], _exact_muon)(case, prepare(case, seed))


def _rows(case, t):
    """[B, C, P] of a field, in 64 bits."""
    t = t.double()
    return t if case["layout"] == "first" else t.transpose(1, 2)


def _back(case, t):
    return t if case["layout"] == "first" else t.transpose(1, 2)


def _phi(z):
    """Distribution function and density of the normal distribution."""
    return 0.5 * torch.erfc(-z / math.sqrt(2.0)), torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)


def _exact_hat(case, s):
    x = _rows(case, s["x"])
    x = x - x.sum(1, keepdim=True) / case["channels"]
    rstd = (x.square().sum(1, keepdim=True) / case["channels"] + EPS_NORM).rsqrt()
    return x.mul_(rstd), rstd


def _exact_norm_fwd(case, s):
    xh, _ = _exact_hat(case, s)
    z = xh.mul_(s["gamma"].double()[:, None]).add_(s["beta"].double()[:, None])
    if case["act"] == "gelu":
        z = z * _phi(z)[0]
    elif case["act"] == "silu":
        z = z * torch.sigmoid(z)
    return _back(case, z)


def _exact_norm_bwd(case, s):
    xh, rstd = _exact_hat(case, s)
    gamma = s["gamma"].double()[:, None]
    z = (xh * gamma).add_(s["beta"].double()[:, None])
    d = _rows(case, s["gy"])
    if case["act"] == "gelu":
        cdf, pdf = _phi(z)
        d = d * pdf.mul_(z).add_(cdf)
        del cdf, pdf
    elif case["act"] == "silu":
        sig = torch.sigmoid(z)
        d = d * (sig + z * sig * torch.sigmoid(-z))
        del sig
    del z
    ggamma, gbeta = (d * xh).sum(2).sum(0), d.sum(2).sum(0)
    h = d * gamma
    del d
    c = case["channels"]
    gx = h - h.sum(1, keepdim=True) / c - xh * ((h * xh).sum(1, keepdim=True) / c)
    return _back(case, gx.mul_(rstd)), ggamma, gbeta


def _exact_muon(case, s):
    out, scale = dict(params=[], momentum=[]), 1.0
    if case["clip"]:
        norm = math.sqrt(sum(float((torch.view_as_real(g) if g.is_complex() else g).double().square().sum()) for g in s["grads"]))
        out["norm"] = torch.tensor([norm], dtype=torch.float64)
        scale = min(1.0, MAX_NORM / norm)
    for p, g, m, step in zip(s["params"], s["grads"], s["momentum"], s["scale"]):
        wide = torch.complex128 if p.is_complex() else torch.float64
        m = m.to(wide) * MOMENTUM + g.to(wide) * scale
        u = m * MOMENTUM + g.to(wide) * scale
        o = _polynomial(u.reshape(*u.shape[:2], -1).permute(2, 0, 1) if p.is_complex() else u.reshape(-1, *u.shape[-2:]))
        o = o.permute(1, 2, 0).reshape(p.shape) if p.is_complex() else o.reshape(p.shape)
        p = p.to(wide) - (p.to(wide) * DECAY + o * step) * LR
        out["params"].append(torch.view_as_real(p) if p.is_complex() else p)
        out["momentum"].append(torch.view_as_real(m.contiguous()) if m.is_complex() else m)
        del u, o
    return out


def _polynomial(u):
    """The iteration with the Gram matrix of the columns (of the rows' transpose where they are fewer), matrices 32768 at a time."""
    if u.shape[1] < u.shape[2]:
        return _polynomial(u.transpose(1, 2)).transpose(1, 2)
    a, b, c = COEFFICIENTS
    out = torch.empty(u.shape, dtype=u.dtype, device=u.device)
    for lo in range(0, u.shape[0], 32768):
        x = u[lo: lo + 32768].contiguous()
        x = x / (x.abs().square().sum((1, 2), keepdim=True).sqrt() + EPS)
        one = torch.eye(x.shape[2], dtype=x.dtype, device=x.device)
        for _ in range(ITERATIONS):
            gram = torch.matmul(_adjoint(x), x)
            x = torch.matmul(x, a * one + torch.matmul(gram, b * one + c * gram))
        out[lo: lo + 32768] = x
    return out


# ------------------------------------------------------------------------------------------ work

def work(case):
    """Bytes: every input read once, every output written once.  Operations: norms about what the formulas have a value; a
    Newton-Schulz step on m x n, m <= n, the halves of two symmetric products (m x n by n x m, m x m by m x m) and a whole one
    (m x m by m x n), of 2 operations a term, complex ones of 8."""
    if case["op"].startswith("ln"):
        n, size = float(case["batch"] * case["channels"] * case["points"]), 4 if case["dtype"] == "f32" else 2
        forward = case["op"] == "ln_fwd"
        return {"bytes": n * size * (2 if forward else 3) + 4.0 * case["channels"] * (2 if forward else 4),
                "flops": n * (20.0 if forward else 40.0)}
    values, flops = 0.0, 0.0
    for shape, is_complex in _shapes(case):
        count, rows, cols = _matrices(shape, is_complex)
        m, n = float(min(rows, cols)), float(max(rows, cols))
        values += math.prod(shape)
        flops += ITERATIONS * count * (8.0 if is_complex else 2.0) * (0.5 * m * (m + 1.0) * (n + m) + m * m * n)
    return {"bytes": 20.0 * values, "flops": flops + 10.0 * values + (2.0 * values if case["clip"] else 0.0)}
