"""The operators that a training step of a normalised network uses beside its blocks, as measurable cases.

A case is one pass through one of them: group norm with an activation over fields [B][C][P] or [B][P][C]
(forward, or backward from the saved statistics), or one AdamW step over all parameters of a network, with
moments in 32 or 8 bits, with or without clipping by the norm of all gradients.  `listed()` names the cases
that stand for the uses, `draw()` gives more of the same ranges, `prepare()` makes what a program holds before
the call, `run()` is the pass, in plain torch operations or through the library where `own` is set, `exact()` the
definition in 64 bits and `work()` the bytes and operations that a pass cannot do without.
"""
import math

import torch

own = False

ACTS = ("identity", "gelu", "silu")
EPS_NORM = 1e-5
LR, BETA1, BETA2, EPS, DECAY, MAX_NORM = 1e-4, 0.9, 0.999, 1e-8, 0.01, 1.0
SEED, FIRST_STEP = 20220401, 1000
GROUP = 256                      # values that share an exponent in an 8-bit moment


def _norm(name, op, layout, dtype, act, batch, channels, groups, points):
    """op norm_fwd or norm_bwd; layout "first" ([B][C][P]) or "last" ([B][P][C]); dtype of the fields "f32" or "bf16"."""
    case = dict(op=op, layout=layout, dtype=dtype, act=act, batch=batch, channels=channels, groups=groups, points=points)
    return case if name is None else dict(name=name, **case)


def _adamw(name, bits, clip, c_in, width, hidden, blocks, counts):
    """The parameters of a network: lift c_in -> width, `blocks` blocks of width channels with counts[0..3] kept modes
    on x, y, z, t and a group norm each, projection width -> hidden -> 1."""
    case = dict(op="adamw", bits=bits, clip=clip, c_in=c_in, width=width, hidden=hidden, blocks=blocks, kx=counts[0],
                ky=counts[1], kz=counts[2], kt=counts[3])
    return case if name is None else dict(name=name, **case)


def listed():
    return [
        # a small surrogate served with normalised blocks: bound by latency
        _norm("norm_16", "norm_fwd", "first", "f32", "gelu", 1, 8, 2, 16 * 16 * 16 * 8),
        # a batch of features of the user's own model, channels last in 16 bits, an odd number of channels
        _norm("norm_last_odd", "norm_fwd", "last", "bf16", "silu", 4, 27, 9, 28 * 24 * 20),
        # training on an odd grid, channels first
        _norm("norm_train_odd", "norm_bwd", "first", "f32", "gelu", 2, 12, 3, 30 * 27 * 21 * 14),
        # one block's field at the paper's training samples, behind the spectral convolution
        _norm("norm_60", "norm_fwd", "first", "f32", "gelu", 1, 20, 4, 60 * 60 * 64 * 30),
        # training with fields kept channels last in 16 bits
        _norm("norm_train_last_64", "norm_bwd", "last", "bf16", "gelu", 2, 20, 5, 64 * 64 * 64 * 16),
        # a wide field, channels last, in 32 bits
        _norm("norm_last_wide", "norm_fwd", "last", "f32", "silu", 1, 32, 8, 64 * 64 * 64 * 20),
        # training at the grid of the benchmark network
        _norm("norm_train_128", "norm_bwd", "first", "f32", "gelu", 1, 20, 4, 128 * 128 * 64 * 32),
        # the step of the smallest network: 21 tensors, most of them a few values, bound by launches
        _adamw("adamw_small", 32, True, 5, 8, 32, 4, (8, 8, 8, 3)),
        # odd widths and kept modes of the symmetric rule, moments in 8 bits
        _adamw("adamw8_odd", 8, True, 3, 13, 37, 3, (13, 11, 9, 5)),
        # the network of the paper's training samples, moments in 32 bits
        _adamw("adamw_60", 32, False, 2, 20, 128, 4, (24, 24, 24, 8)),
        # the same with moments in 8 bits and clipping
        _adamw("adamw8_60", 8, True, 2, 20, 128, 4, (24, 24, 24, 8)),
        # the benchmark network, clipping: the largest
        _adamw("adamw_128", 32, True, 5, 20, 128, 4, (32, 32, 24, 9)),
    ]


def draw(rng):
    """One more case of the same ranges: fields from one point to those of the benchmark network, networks from a few
    thousand parameters to those of the paper's samples."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        if rng.random() < 0.6:
            op, layout, dtype = rng.choice(("norm_fwd", "norm_bwd")), rng.choice(("first", "last")), rng.choice(("f32", "bf16"))
            groups = rng.choice((1, 2, 3, 4, 5, 8, 16))
            channels = groups * spread(1, 40)
            batch, points = spread(1, 16), spread(1, 3.4e7)
            if channels > 320 or batch * channels * points > 6.5e8 or channels // groups * points < 16:
                continue
            return _norm(None, op, layout, dtype, rng.choice(("gelu", "gelu", "silu", "identity")), batch, channels, groups,
                         points)
        width, hidden = rng.choice((8, 16, 20, 24, 32, rng.randint(4, 32))), rng.choice((32, 64, 128, rng.randint(8, 200)))
        counts = [rng.randint(4, 28) for _ in range(3)] + [rng.randint(2, 9)]
        case = _adamw(None, rng.choice((8, 32)), rng.random() < 0.6, rng.randint(1, 6), width, hidden, rng.choice((1, 2, 3, 4)),
                      counts)
        if _parameters(case) <= 4e8:
            return case


def _shapes(case):
    """Shapes of a network's parameters as reals, and whether they decay: matrices do, biases and norms do not."""
    ci, w, h = case["c_in"], case["width"], case["hidden"]
    out = [((w, ci), True), ((h, w), True), ((h,), False), ((1, h), True), ((1,), False)]
    for _ in range(case["blocks"]):
        out += [((w, w, case["kx"], case["ky"], case["kz"], case["kt"], 2), True), ((w, w), True), ((w,), False),
                ((2, w), False)]
    return out


def _parameters(case):
    return sum(math.prod(shape) for shape, _ in _shapes(case))


def _field_shape(case):
    b, c, p = case["batch"], case["channels"], case["points"]
    return (b, c, p) if case["layout"] == "first" else (b, p, c)


# ------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    return (_prepare_adamw if case["op"] == "adamw" else _prepare_norm)(case, normal)


def _prepare_norm(case, normal):
    c, shape = case["channels"], _field_shape(case)
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    # every channel has a mean and a scale of its own, as what comes out of a channel map has
    mean, scale = 0.5 + normal(c).abs_(), 0.5 + 0.5 * normal(c).abs_()
    if case["layout"] == "first":
        mean, scale = mean[:, None], scale[:, None]
    x = normal(*shape).mul_(scale).add_(mean).to(dtype)
    s = dict(case=case, x=x, gamma=1 + 0.2 * normal(c), beta=0.3 * normal(c))
    if case["op"] == "norm_fwd":
        s.update(y=torch.empty_like(x), mean=torch.empty(case["batch"], case["groups"], device="cuda"),
                 rstd=torch.empty(case["batch"], case["groups"], device="cuda"))
    else:                        # the statistics that the forward pass saved, and the cotangent
        mu, rstd = _statistics(case, x.float())
        s.update(mean=mu.reshape(case["batch"], -1).contiguous(), rstd=rstd.reshape(case["batch"], -1).contiguous(),
                 gy=normal(*shape).to(dtype), gx=torch.empty_like(x), ggamma=torch.empty(c, device="cuda"),
                 gbeta=torch.empty(c, device="cuda"))
    if own:                      # the descriptor and the workspace that a program keeps
        from paper_2204_01205_amd import binding as B
        s["desc"] = B.make_norm_desc(case["batch"], c, case["groups"], case["points"],
                                     layout=B.FNO_LAYOUT_CHANNELS_FIRST if case["layout"] == "first" else B.FNO_LAYOUT_CHANNELS_LAST,
                                     dtype=B.FNO_DTYPE_F32 if case["dtype"] == "f32" else B.FNO_DTYPE_BF16,
                                     activation=ACTS.index(case["act"]), eps=EPS_NORM)
        s["ws"] = B.alloc_norm_workspace(s["desc"])
    return s


def _prepare_adamw(case, normal):
    s = dict(case=case, step=FIRST_STEP, params=[], grads=[], m=[], v=[], exps=[], m_out=[], v_out=[],
             norm=torch.empty(1, device="cuda"), decay=[DECAY if d else 0.0 for _, d in _shapes(case)])
    for k, (shape, _) in enumerate(_shapes(case)):
        n = math.prod(shape)
        # weights of the size that their fan-in gives, gradients that fall with the frequency along the modes of t
        s["params"].append(normal(*shape).mul_(0.5 / math.sqrt(shape[-1] if len(shape) < 7 else case["width"])))
        falloff = torch.logspace(0, -3, case["kt"], device="cuda")[:, None] if len(shape) == 7 else 1.0
        size = 3e-3 * falloff
        s["grads"].append(normal(*shape).mul_(size))
        # moments in the middle of a training run
        m = normal(*shape).mul_(0.3 * size).reshape(-1)
        v = normal(*shape).mul_(size).square_().add_(0.1 * size * size).reshape(-1)
        if case["bits"] == 32:
            s["m"].append(m)
            s["v"].append(v)
        else:
            codes, em = _encode_m(m, _random_bits(n, SEED, 0, k))
            s["m"].append(codes)
            codes, ev = _encode_v(v, _random_bits(n, SEED, 0, k))
            s["v"].append(codes)
            s["exps"].append(torch.stack((em, ev), 1).contiguous())
            s["m_out"].append(torch.empty(n, dtype=torch.bfloat16, device="cuda"))
            s["v_out"].append(torch.empty(n, dtype=torch.bfloat16, device="cuda"))
    if own:                      # the list of tensors that a program keeps, and the scratch of the gradients' norm
        from paper_2204_01205_amd import binding as B
        s["list"] = B.make_adamw_tensors(s["params"], s["grads"], s["m"], s["v"], s["exps"] or None, s["decay"])
        s["ws"] = B.alloc_grad_norm_workspace(s["list"])
    return s


# ------------------------------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _own(s)
    return {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "adamw": _plain_adamw}[s["case"]["op"]](s, s["case"])


def _own(s):
    from paper_2204_01205_amd import binding as B
    case = s["case"]
    if case["op"] == "norm_fwd":
        B.fno_group_norm_fwd(s["desc"], s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], s["ws"])
        return s["y"], s["mean"], s["rstd"]
    if case["op"] == "norm_bwd":
        B.fno_group_norm_bwd(s["desc"], s["x"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["gy"], s["gx"], s["ggamma"],
                             s["gbeta"], s["ws"])
        return s["gx"], s["ggamma"], s["gbeta"]
    s["step"] += 1
    norm = s["norm"] if case["clip"] else None
    if case["clip"]:
        B.fno_grad_norm(s["list"], norm, s["ws"])
    B.fno_adamw_step(s["list"], LR, BETA1, BETA2, EPS, s["step"], grad_norm=norm, max_norm=MAX_NORM, seed=SEED)
    if case["bits"] == 8:
        B.fno_adamw_state_read(s["list"], s["m_out"], s["v_out"])
    return _adamw_outputs(s, case)


def _adamw_outputs(s, case):
    """Parameters and moments; those in 8 bits as the values they stand for, each of which is a bf16 value."""
    out = dict(params=s["params"], m=s["m"] if case["bits"] == 32 else s["m_out"], v=s["v"] if case["bits"] == 32 else s["v_out"])
    if case["clip"]:
        out["norm"] = s["norm"]
    return out


# ------------------------------------------------------------------------------------------ plain forms

def _grouped(case, t):
    """A field or a vector of channels as [B, G, D, P] or [B, P, G, D]."""
    g, d = case["groups"], case["channels"] // case["groups"]
    if case["layout"] == "first":
        return t.reshape(1, g, d, 1) if t.dim() == 1 else t.reshape(case["batch"], g, d, case["points"])
    return t.reshape(1, 1, g, d) if t.dim() == 1 else t.reshape(case["batch"], case["points"], g, d)


def _points_mean(case, t):
    """Mean over the points of every channel of a grouped field (over all axes of a group at once the same sums take
    up to ten times as long)."""
    return t.mean(3 if case["layout"] == "first" else 1, keepdim=True)


def _group_mean(case, t):
    return t.mean(2 if case["layout"] == "first" else 3, keepdim=True)


def _statistics(case, x):
    x = _grouped(case, x)
    mean = _group_mean(case, _points_mean(case, x))
    var = _group_mean(case, _points_mean(case, (x - mean).square()))
    return mean, 1.0 / torch.sqrt(var + EPS_NORM)


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


def _plain_norm_fwd(s, case):
    x = s["x"].float()
    mean, rstd = _statistics(case, x)
    z = (_grouped(case, x) - mean) * rstd * _grouped(case, s["gamma"]) + _grouped(case, s["beta"])
    y = _activation(case["act"], z).reshape(_field_shape(case)).to(s["x"].dtype)
    return y, mean.reshape(case["batch"], -1), rstd.reshape(case["batch"], -1)


def _plain_norm_bwd(s, case):
    x, gy = _grouped(case, s["x"].float()), _grouped(case, s["gy"].float())
    gamma, beta = _grouped(case, s["gamma"]), _grouped(case, s["beta"])
    shape = [1] * 4
    shape[0], shape[1 if case["layout"] == "first" else 2] = case["batch"], case["groups"]
    rstd = s["rstd"].reshape(shape)
    xh = (x - s["mean"].reshape(shape)) * rstd
    gz = gy * _slope(case["act"], xh * gamma + beta)
    a, b = _points_mean(case, gz), _points_mean(case, gz * xh)
    ggamma, gbeta = b.sum(0).reshape(-1) * case["points"], a.sum(0).reshape(-1) * case["points"]
    gx = rstd * (gz * gamma - _group_mean(case, a * gamma) - xh * _group_mean(case, b * gamma))
    return gx.reshape(_field_shape(case)).to(s["x"].dtype), ggamma, gbeta


MASK = 0xFFFFFFFF


def _mix(x):
    """A mix of 32 bits, on whole numbers or on int64 tensors that hold them."""
    x = x ^ (x >> 16)
    x = (x * 0xCB4F2D3B) & MASK
    x = x ^ (x >> 13)
    x = (x * 0xFDB6A5C3) & MASK
    return x ^ (x >> 16)


def _random_bits(n, seed, step, tensor):
    """32 bits for each value of a tensor in one step: 16 for each moment's rounding."""
    key = _mix(_mix(_mix(seed & MASK) ^ (step & MASK)) ^ tensor)
    at = torch.arange(-(-n // GROUP), device="cuda")
    block = _mix((_mix((at + key) & MASK) + (at >> 32)) & MASK)
    inner = torch.arange(GROUP, device="cuda") * 0x9E3779B1
    return _mix((block[:, None] + inner) & MASK)


def _blocks(t):
    """A flat float tensor as rows of 256, zeros behind the last value."""
    return torch.nn.functional.pad(t, (0, -t.numel() % GROUP)).reshape(-1, GROUP)


def _exponent(bits, least):
    """Shared exponents of rows whose values have these bits: that of the largest, rounded up to four bits; 255 where a
    value is not finite."""
    top = bits.amax(1)
    e = ((top + 0xFFFFF) >> 23).clamp(least, 254)
    return torch.where(top >= 0x7F800000, torch.full_like(e, 255), e)


def _encode_m(t, random):
    """Codes (sign, 4 exponent bits, 3 bits; zero is 0) and shared exponents of a flat tensor, rounded up with the
    probability of the part that is cut, below the smallest code too."""
    x = _blocks(t)
    bits = x.abs().view(torch.int32).to(torch.int64)
    e = _exponent(bits, 16)
    r = random & 0xFFFF
    first = ((e - 15) << 23) + (1 << 20)
    code = (((bits + (r << 4)) >> 20) - ((e - 15) << 3)[:, None]).clamp(0, 127)
    small = first.to(torch.int32).view(torch.float32)[:, None] * (r.float() * (1.0 / 65536.0)) < x.abs()
    code = torch.where(bits < first[:, None], small.to(torch.int64), code)
    code = torch.where(x < 0, code + 128, code)
    return code.to(torch.uint8).reshape(-1)[: t.numel()].contiguous(), e.to(torch.uint8)


def _encode_v(t, random):
    """The same for values that are never negative: 5 exponent bits and 3, and what is not zero never becomes zero."""
    x = _blocks(t)
    bits = x.view(torch.int32).to(torch.int64)
    e = _exponent(bits, 32)
    code = (((bits + ((random >> 16) << 4)) >> 20) - ((e - 31) << 3)[:, None]).clamp(1, 255)
    code = torch.where(bits == 0, torch.zeros_like(code), code)
    return code.to(torch.uint8).reshape(-1)[: t.numel()].contiguous(), e.to(torch.uint8)


def _decode(codes, exps, signed):
    c = torch.nn.functional.pad(codes, (0, -codes.numel() % GROUP)).reshape(-1, GROUP).to(torch.int32)
    e = exps.to(torch.int32)[:, None]
    mag = c & (127 if signed else 255)
    x = ((mag << 20) + ((e - (15 if signed else 31)) << 23)).view(torch.float32)
    x = torch.where(mag == 0, torch.zeros_like(x), x)
    if signed:
        x = torch.where(c >= 128, -x, x)
    x = torch.where(e == 255, torch.full_like(x, math.nan), x)
    return x.reshape(-1)[: codes.numel()]


def _plain_adamw(s, case):
    s["step"] += 1
    scale, fine = 1.0, None
    if case["clip"]:
        norm = torch.stack([g.square().sum() for g in s["grads"]]).sum().sqrt()
        s["norm"].copy_(norm.reshape(1))
        scale = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))
        fine = torch.isfinite(norm)
    for k in range(len(s["params"])):
        _plain_adamw_tensor(s, case, k, scale, fine)
    return _adamw_outputs(s, case)


def _plain_adamw_tensor(s, case, k, scale, fine):
    step, p, g = s["step"], s["params"][k].reshape(-1), s["grads"][k].reshape(-1) * scale
    m, v = s["m"][k], s["v"][k]
    if case["bits"] == 8:
        m, v = _decode(m, s["exps"][k][:, 0], True), _decode(v, s["exps"][k][:, 1], False)
    m, v = BETA1 * m + (1.0 - BETA1) * g, BETA2 * v + (1.0 - BETA2) * (g * g)
    q = p * (1.0 - LR * s["decay"][k])
    q = q - LR * (m / (1.0 - BETA1 ** step)) / (torch.sqrt(v / (1.0 - BETA2 ** step)) + EPS)

    def put(to, new):            # a step whose norm is not finite changes nothing
        to.copy_(new if fine is None else torch.where(fine, new, to))

    put(p, q)
    if case["bits"] == 32:
        put(s["m"][k], m)
        put(s["v"][k], v)
        return
    random = _random_bits(p.numel(), SEED, step, k)
    for j, (to, new, encode) in enumerate(((s["m"][k], m, _encode_m), (s["v"][k], v, _encode_v))):
        codes, e = encode(new, random)
        put(to, codes)
        put(s["exps"][k][:, j], e)
    s["m_out"][k].copy_(_decode(s["m"][k], s["exps"][k][:, 0], True))
    s["v_out"][k].copy_(_decode(s["v"][k], s["exps"][k][:, 1], False))


# ------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    return {"norm_fwd": _exact_norm_fwd, "norm_bwd": _exact_norm_bwd, "adamw": _exact_adamw}[case["op"]](case, prepare(case, seed))


def _rows(case, t):
    """[B, G, D, P] of a field, in 64 bits."""
    t = t.double()
    if case["layout"] == "last":
        t = t.transpose(1, 2)
    return t.reshape(case["batch"], case["groups"], -1, case["points"])


def _back(case, t):
    t = t.reshape(case["batch"], case["channels"], case["points"])
    return t if case["layout"] == "first" else t.transpose(1, 2)


def _phi(z):
    """Distribution function and density of the normal distribution."""
    return 0.5 * torch.erfc(-z / math.sqrt(2.0)), torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)


def _exact_norm_fwd(case, s):
    x, side = _rows(case, s["x"]), (1, case["groups"], -1, 1)
    n = x.shape[2] * x.shape[3]
    mean = x.sum((2, 3), keepdim=True) / n
    x -= mean
    rstd = (x.square().sum((2, 3), keepdim=True) / n + EPS_NORM).rsqrt()
    z = x.mul_(rstd).mul_(s["gamma"].double().view(side)).add_(s["beta"].double().view(side))
    if case["act"] == "gelu":
        z = z * _phi(z)[0]
    elif case["act"] == "silu":
        z = z * torch.sigmoid(z)
    return _back(case, z), mean.view(case["batch"], -1), rstd.view(case["batch"], -1)


def _exact_norm_bwd(case, s):
    side, stat = (1, case["groups"], -1, 1), (case["batch"], case["groups"], 1, 1)
    rstd, gamma = s["rstd"].double().view(stat), s["gamma"].double().view(side)
    xh = _rows(case, s["x"]).sub(s["mean"].double().view(stat)).mul_(rstd)
    z = (xh * gamma).add_(s["beta"].double().view(side))
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
    s1, s2 = d.sum(3), (d * xh).sum(3)                       # [B, G, D]
    n = xh.shape[2] * xh.shape[3]
    a = (s1 * gamma[..., 0]).sum(2)[..., None, None] / n
    b = (s2 * gamma[..., 0]).sum(2)[..., None, None] / n
    gx = d.mul_(gamma).sub_(a).sub_(xh.mul_(b)).mul_(rstd)
    return _back(case, gx), s2.sum(0).reshape(-1), s1.sum(0).reshape(-1)


def _code_values(x, random, low, keep):
    """What 8-bit codes of x >= 0 stand for: steps of an eighth of a power of two from the shared exponent of 256 values
    down `low` powers, rounded by `random` / 65536; `keep`: what is not zero stays at least the smallest code."""
    n = x.numel()
    x = torch.nn.functional.pad(x, (0, -n % GROUP)).reshape(-1, GROUP)
    top = x.amax(1, keepdim=True)
    power = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top))))
    power = power + (top > 1.875 * torch.exp2(power))
    power = torch.where(top > 0, power, torch.full_like(power, -200.0)).clamp(min=low + 1 - 127)
    least = 1.125 * torch.exp2(power - low)
    own_power = torch.floor(torch.log2(torch.where(x > 0, x, torch.ones_like(x))))
    ulp = torch.exp2(own_power - 3)
    y = torch.floor(x / ulp + random / 65536.0) * ulp
    small = x < least
    y = torch.where(small, torch.where(x > least * random / 65536.0, least, torch.zeros_like(x)), y)
    if keep:
        y = torch.where(x > 0, torch.maximum(y, least), y)
    return y.reshape(-1)[:n]


def _exact_adamw(case, s):
    step = s["step"] + 1
    out, scale = dict(params=[], m=[], v=[]), 1.0
    if case["clip"]:
        norm = math.sqrt(sum(float(g.double().square().sum()) for g in s["grads"]))
        out["norm"] = torch.tensor([norm], dtype=torch.float64)
        scale = min(1.0, MAX_NORM / norm)
    for k, (p, g) in enumerate(zip(s["params"], s["grads"])):
        m, v = s["m"][k], s["v"][k]
        if case["bits"] == 8:
            m, v = _decode(m, s["exps"][k][:, 0], True), _decode(v, s["exps"][k][:, 1], False)
        g = g.double().reshape(-1) * scale
        m, v = m.double() * BETA1 + g * (1.0 - BETA1), v.double() * BETA2 + g.square() * (1.0 - BETA2)
        move = (m / (1.0 - BETA1 ** step)) / ((v / (1.0 - BETA2 ** step)).sqrt() + EPS) + s["decay"][k] * p.double().reshape(-1)
        out["params"].append((p.double().reshape(-1) - LR * move).reshape(p.shape))
        del move
        if case["bits"] == 8:
            r = _random_bits(m.numel(), SEED, step, k)
            m = torch.copysign(_code_values(m.abs(), (r & 0xFFFF).double(), 15, False), m)
            v = _code_values(v, (r >> 16).double(), 31, True)
        out["m"].append(m)
        out["v"].append(v)
    return out


# ------------------------------------------------------------------------------------------ work

def work(case):
    """Bytes: every input read once, every output written once.  Operations: about what the formulas have a value."""
    if case["op"] == "adamw":
        n = _parameters(case)
        # p, g, m, v in and p, m, v out; in 8 bits m and v a byte each way, two exponents a block of 256, and the values
        # they stand for in 16 bits
        return {"bytes": n * (28.0 if case["bits"] == 32 else 12.0 + 4.0 + 4.0 / GROUP + 4.0),
                "flops": n * (16.0 if case["bits"] == 32 else 40.0) + (2.0 * n if case["clip"] else 0.0)}
    n, size = float(case["batch"] * case["channels"] * case["points"]), 4 if case["dtype"] == "f32" else 2
    return {"bytes": n * size * (2 if case["op"] == "norm_fwd" else 3) + 8.0 * (case["batch"] * case["groups"] + 2 * case["channels"]),
            "flops": n * (20.0 if case["op"] == "norm_fwd" else 40.0)}
