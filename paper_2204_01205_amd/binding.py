"""Thin ctypes binding of libfno.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/fno.h) and hands it the
device pointers of torch tensors; all arithmetic happens in the HIP kernels.  torch is used
for device memory and the current stream, nothing else.  If libfno.so is missing the first
call raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfno.so")

FNO_OK, FNO_EINVAL, FNO_EUNSUPPORTED, FNO_ENOSPC, FNO_EHIP = 0, -1, -2, -3, -4
FNO_ACT_IDENTITY, FNO_ACT_GELU = 0, 1
FNO_ACT_SILU = 2                 # group norm only
FNO_LAYOUT_CHANNELS_FIRST, FNO_LAYOUT_CHANNELS_LAST = 0, 1
FNO_DTYPE_F32, FNO_DTYPE_BF16 = 0, 1
FNO_OP_SPECTRAL_CONV_FWD, FNO_OP_SPECTRAL_CONV_BWD, FNO_OP_BLOCK_FWD, FNO_OP_BLOCK_BWD = 0, 1, 2, 3
FNO_FLAG_MSE_TARGET = 1
FNO_FLAG_ACCUMULATE_GRADS = 2
FNO_FLAG_TABLES_READY = 4
FNO_STATIC_SCRATCH_BYTES = 64 << 20

EXPORTS = [
    "fno_workspace_bytes", "fno_plan_tables", "fno_mode_indices", "fno_spectral_conv_fwd", "fno_spectral_conv_bwd",
    "fno_block_fwd", "fno_block_bwd", "fno_pointwise_linear", "fno_pointwise_mlp2", "fno_time_lift",
    "fno_rel_l2_workspace_bytes", "fno_rel_l2_loss", "fno_adam_step",
    "fno_pointwise_bwd_workspace_bytes", "fno_pointwise_linear_bwd", "fno_pointwise_mlp2_bwd",
    "fno_time_lift_bwd_workspace_bytes", "fno_time_lift_bwd",
    "fno_spectral_conv_fwd_static",
    "fno_group_norm_workspace_bytes", "fno_group_norm_fwd", "fno_group_norm_bwd",
    "fno_adamw_step", "fno_grad_norm_workspace_bytes", "fno_grad_norm", "fno_adamw_state_read",
    "fno_status_string", "fno_timing_enable", "fno_timing_read",
]

STAGE_NAMES = ["tz_fwd", "y_fwd", "x_fwd", "mix", "x_inv", "y_inv", "zt_inv", "mix_bwd", "bwd_pointwise"]


class FnoDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("c_in", ctypes.c_int32), ("c_out", ctypes.c_int32),
                ("grid", ctypes.c_int32 * 4), ("modes", ctypes.c_int32 * 4),
                ("mode_rule", ctypes.c_int32), ("activation", ctypes.c_int32),
                ("flags", ctypes.c_int32)]


class FnoNormDesc(ctypes.Structure):
    _fields_ = [("npoints", ctypes.c_int64), ("eps", ctypes.c_double), ("batch", ctypes.c_int32),
                ("channels", ctypes.c_int32), ("groups", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("activation", ctypes.c_int32), ("flags", ctypes.c_int32)]


class FnoAdamwTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("exps", ctypes.c_void_p), ("n", ctypes.c_int64), ("weight_decay", ctypes.c_double)]


class FnoError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"libfno status {status}: {text}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
        l = ctypes.CDLL(LIB_PATH)
        l.fno_status_string.restype = ctypes.c_char_p
        l.fno_status_string.argtypes = [ctypes.c_int]
        for name in EXPORTS:
            if name != "fno_status_string":
                getattr(l, name).restype = ctypes.c_int
        # calls that small workloads make often take plain numbers and addresses
        p, i32, f64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_double, ctypes.c_size_t
        l.fno_group_norm_fwd.argtypes = [p] * 8 + [size, p]
        l.fno_group_norm_bwd.argtypes = [p] * 11 + [size, p]
        l.fno_adamw_step.argtypes = [i32, p, i32, f64, f64, f64, f64, i32, p, f64, ctypes.c_uint32, p]
        l.fno_grad_norm.argtypes = [i32, p, p, p, size, p]
        l.fno_adamw_state_read.argtypes = [i32, p, p, p, p]
        _lib = l
    return _lib


def make_desc(batch: int, c_in: int, c_out: int, grid: Sequence[int], modes: Sequence[int],
              mode_rule: int = 0, activation: int = FNO_ACT_GELU, flags: int = 0) -> FnoDesc:
    return FnoDesc(batch, c_in, c_out, (ctypes.c_int32 * 4)(*grid), (ctypes.c_int32 * 4)(*modes),
                   mode_rule, activation, flags)


def _check(status: int) -> None:
    if status != FNO_OK:
        raise FnoError(status, lib().fno_status_string(status).decode())


def _ptr(t: Optional[torch.Tensor], dtype=torch.float32, name: str = "tensor"):
    if t is None:
        return ctypes.c_void_p(0)
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    want = (dtype, torch.complex64) if dtype == torch.float32 else (dtype,)
    if t.dtype not in want:
        raise ValueError(f"{name} has dtype {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


def _sizes(desc: FnoDesc):
    """(grid points, kept modes) per (batch, channel) slab, from the library's own mode lists."""
    npts = 1
    for n in desc.grid:
        npts *= int(n)
    kept = 1
    for axis in range(4):
        n = ctypes.c_int32(0)
        _check(lib().fno_mode_indices(ctypes.byref(desc), ctypes.c_int(axis), None, ctypes.byref(n)))
        kept *= int(n.value)
    return npts, kept


def _expect(t: Optional[torch.Tensor], name: str, numel: int) -> None:
    """A tensor handed to the kernels must hold exactly the elements the descriptor implies: the
    kernels index by the descriptor alone, and a short buffer would be read or written out of bounds."""
    if t is None:
        return
    have = t.numel() * (2 if t.dtype == torch.complex64 else 1)
    if have != numel:
        raise ValueError(f"{name} holds {have} floats, the descriptor implies {numel}")


def _check_layer_tensors(desc, *, x=None, y=None, R=None, xhat=None, W=None, b=None, extra_in=(), extra_out=()):
    npts, kept = _sizes(desc)
    B_, ci, co = int(desc.batch), int(desc.c_in), int(desc.c_out)
    _expect(x, "x", B_ * ci * npts)
    _expect(y, "output", B_ * co * npts)
    _expect(R, "R", 2 * ci * co * kept)
    _expect(xhat, "xhat", 2 * B_ * ci * kept)
    _expect(W, "W", co * ci)
    _expect(b, "b", co)
    for name, t in extra_in:
        _expect(t, name, B_ * ci * npts)
    for name, t in extra_out:
        _expect(t, name, B_ * co * npts)


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _raw_stream(device: Optional[int] = None) -> int:
    """The current stream's handle, without the stream object that _stream() makes (0.3 us instead of 3), where torch has the
    call that its own generated code uses for that; it is not among the documented ones."""
    device = torch.cuda.current_device() if device is None else device
    handle = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return handle(device) if handle is not None else torch.cuda.current_stream(device).cuda_stream


def _address(t: Optional[torch.Tensor], dtype, numel: int, name: str):
    """A tensor's address for a call with argtypes, after the checks of _ptr() and _expect() in the order of their cost:
    small calls are bound by the host."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != numel or not t.is_cuda or not t.is_contiguous():
        if t.dtype is not dtype:
            raise ValueError(f"{name} has dtype {t.dtype}")
        _expect(t, name, numel)
        _ptr(t, dtype, name)
    return t.data_ptr()


def fno_status_string(status: int) -> str:
    return lib().fno_status_string(status).decode()


def fno_workspace_bytes(desc: FnoDesc, op: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fno_workspace_bytes(ctypes.byref(desc), ctypes.c_int(op), ctypes.byref(n)))
    return int(n.value)


def fno_plan_tables(desc: FnoDesc, op: int, ws) -> None:
    p, n = _ws(ws)
    _check(lib().fno_plan_tables(ctypes.byref(desc), ctypes.c_int(op), p, n, _stream()))


def fno_mode_indices(desc: FnoDesc, axis: int) -> list[int]:
    n = ctypes.c_int32(0)
    _check(lib().fno_mode_indices(ctypes.byref(desc), ctypes.c_int(axis), None, ctypes.byref(n)))
    buf = (ctypes.c_int32 * max(n.value, 1))()
    _check(lib().fno_mode_indices(ctypes.byref(desc), ctypes.c_int(axis), buf, ctypes.byref(n)))
    return [int(buf[i]) for i in range(n.value)]


def kept_counts(desc: FnoDesc) -> tuple:
    """Number of kept modes per axis (x, y, z, t): the lengths of the library's mode lists."""
    return tuple(len(fno_mode_indices(desc, axis)) for axis in range(4))


def alloc_workspace(desc: FnoDesc, op: int, device="cuda") -> torch.Tensor:
    """A byte tensor of the size the op asks for (torch allocations are 256-byte aligned)."""
    return torch.empty(max(fno_workspace_bytes(desc, op), 256), dtype=torch.uint8, device=device)


def _ws(ws: torch.Tensor):
    if not ws.is_cuda or ws.dtype != torch.uint8:
        raise ValueError("workspace must be a uint8 GPU tensor")
    return ctypes.c_void_p(ws.data_ptr()), ctypes.c_size_t(ws.numel())


def fno_spectral_conv_fwd(desc, x, R, y, xhat_save, ws) -> None:
    _check_layer_tensors(desc, x=x, y=y, R=R, xhat=xhat_save)
    p, n = _ws(ws)
    _check(lib().fno_spectral_conv_fwd(ctypes.byref(desc), _ptr(x, name="x"), _ptr(R, name="R"),
                                       _ptr(y, name="y"), _ptr(xhat_save, name="xhat_save"),
                                       p, n, _stream()))


def fno_spectral_conv_fwd_static(desc, x, R, y, xhat_save) -> None:
    _check_layer_tensors(desc, x=x, y=y, R=R, xhat=xhat_save)
    _check(lib().fno_spectral_conv_fwd_static(ctypes.byref(desc), _ptr(x, name="x"), _ptr(R, name="R"),
                                              _ptr(y, name="y"), _ptr(xhat_save, name="xhat_save"),
                                              _stream()))


def fno_spectral_conv_bwd(desc, x, xhat_saved, R, gy, gx, gR, ws) -> None:
    _check_layer_tensors(desc, x=x, y=gy, R=R, xhat=xhat_saved, extra_in=(("gx", gx),))
    _expect(gR, "gR", R.numel() * 2 if R is not None else 0)
    p, n = _ws(ws)
    _check(lib().fno_spectral_conv_bwd(ctypes.byref(desc), _ptr(x, name="x"),
                                       _ptr(xhat_saved, name="xhat_saved"), _ptr(R, name="R"),
                                       _ptr(gy, name="gy"), _ptr(gx, name="gx"), _ptr(gR, name="gR"),
                                       p, n, _stream()))


def fno_block_fwd(desc, x, R, W, b, out, z_save, xhat_save, ws) -> None:
    _check_layer_tensors(desc, x=x, y=out, R=R, xhat=xhat_save, W=W, b=b, extra_out=(("z_save", z_save),))
    p, n = _ws(ws)
    _check(lib().fno_block_fwd(ctypes.byref(desc), _ptr(x, name="x"), _ptr(R, name="R"),
                               _ptr(W, name="W"), _ptr(b, name="b"), _ptr(out, name="out"),
                               _ptr(z_save, name="z_save"), _ptr(xhat_save, name="xhat_save"),
                               p, n, _stream()))


def fno_block_bwd(desc, x, R, W, z_saved, xhat_saved, gout, gx, gR, gW, gb, ws) -> None:
    _check_layer_tensors(desc, x=x, y=gout, R=R, xhat=xhat_saved, W=W, b=gb,
                         extra_in=(("gx", gx),), extra_out=(("z_saved", z_saved),))
    _expect(gR, "gR", R.numel() * 2 if R is not None else 0)
    _expect(gW, "gW", W.numel() if W is not None else 0)
    p, n = _ws(ws)
    _check(lib().fno_block_bwd(ctypes.byref(desc), _ptr(x, name="x"), _ptr(R, name="R"),
                               _ptr(W, name="W"), _ptr(z_saved, name="z_saved"),
                               _ptr(xhat_saved, name="xhat_saved"), _ptr(gout, name="gout"),
                               _ptr(gx, name="gx"), _ptr(gR, name="gR"), _ptr(gW, name="gW"),
                               _ptr(gb, name="gb"), p, n, _stream()))


def fno_pointwise_linear(batch, c_in, c_out, npoints, x, W, bias, y) -> None:
    _check(lib().fno_pointwise_linear(ctypes.c_int32(batch), ctypes.c_int32(c_in), ctypes.c_int32(c_out),
                                      ctypes.c_int64(npoints), _ptr(x, name="x"), _ptr(W, name="W"),
                                      _ptr(bias, name="bias"), _ptr(y, name="y"), _stream()))


def fno_time_lift(batch, c_in, c_out, nspace, nt, a, Wt, bt, Wc, bc, out) -> None:
    _check(lib().fno_time_lift(ctypes.c_int32(batch), ctypes.c_int32(c_in), ctypes.c_int32(c_out),
                               ctypes.c_int64(nspace), ctypes.c_int32(nt), _ptr(a, name="a"),
                               _ptr(Wt, name="Wt"), _ptr(bt, name="bt"), _ptr(Wc, name="Wc"),
                               _ptr(bc, name="bc"), _ptr(out, name="out"), _stream()))


def fno_time_lift_bwd_workspace_bytes(c_in, c_out, nt) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fno_time_lift_bwd_workspace_bytes(ctypes.c_int32(c_in), ctypes.c_int32(c_out), ctypes.c_int32(nt),
                                                   ctypes.byref(n)))
    return int(n.value)


def fno_time_lift_bwd(batch, c_in, c_out, nspace, nt, a, Wt, bt, Wc, g, gWt, gbt, gWc, gbc, ws) -> None:
    _check(lib().fno_time_lift_bwd(ctypes.c_int32(batch), ctypes.c_int32(c_in), ctypes.c_int32(c_out),
                                   ctypes.c_int64(nspace), ctypes.c_int32(nt), _ptr(a, name="a"),
                                   _ptr(Wt, name="Wt"), _ptr(bt, name="bt"), _ptr(Wc, name="Wc"),
                                   _ptr(g, name="g"), _ptr(gWt, name="gWt"), _ptr(gbt, name="gbt"),
                                   _ptr(gWc, name="gWc"), _ptr(gbc, name="gbc"), _ptr(ws, name="ws"),
                                   ctypes.c_size_t(ws.numel() * ws.element_size()), _stream()))


def fno_pointwise_bwd_workspace_bytes(c_in, hidden, c_out) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fno_pointwise_bwd_workspace_bytes(ctypes.c_int32(c_in), ctypes.c_int32(hidden),
                                                   ctypes.c_int32(c_out), ctypes.byref(n)))
    return int(n.value)


def fno_pointwise_linear_bwd(batch, c_in, c_out, npoints, x, W, g, gx, gW, gb, ws) -> None:
    _check(lib().fno_pointwise_linear_bwd(ctypes.c_int32(batch), ctypes.c_int32(c_in), ctypes.c_int32(c_out),
                                          ctypes.c_int64(npoints), _ptr(x, name="x"), _ptr(W, name="W"),
                                          _ptr(g, name="g"), _ptr(gx, name="gx"), _ptr(gW, name="gW"),
                                          _ptr(gb, name="gb"), _ptr(ws, name="ws"),
                                          ctypes.c_size_t(ws.numel() * ws.element_size()), _stream()))


def fno_pointwise_mlp2_bwd(batch, c_in, hidden, c_out, npoints, x, W1, b1, W2, g, gx, gW1, gb1, gW2, gb2, ws) -> None:
    _check(lib().fno_pointwise_mlp2_bwd(ctypes.c_int32(batch), ctypes.c_int32(c_in), ctypes.c_int32(hidden),
                                        ctypes.c_int32(c_out), ctypes.c_int64(npoints), _ptr(x, name="x"),
                                        _ptr(W1, name="W1"), _ptr(b1, name="b1"), _ptr(W2, name="W2"),
                                        _ptr(g, name="g"), _ptr(gx, name="gx"), _ptr(gW1, name="gW1"),
                                        _ptr(gb1, name="gb1"), _ptr(gW2, name="gW2"), _ptr(gb2, name="gb2"),
                                        _ptr(ws, name="ws"), ctypes.c_size_t(ws.numel() * ws.element_size()),
                                        _stream()))


def fno_rel_l2_workspace_bytes() -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fno_rel_l2_workspace_bytes(ctypes.byref(n)))
    return int(n.value)


def fno_rel_l2_loss(n, pred, target, loss, grad, ws) -> None:
    _check(lib().fno_rel_l2_loss(ctypes.c_int64(n), _ptr(pred, name="pred"), _ptr(target, name="target"),
                                 _ptr(loss, name="loss"), _ptr(grad, name="grad"), _ptr(ws, name="ws"),
                                 ctypes.c_size_t(ws.numel() * ws.element_size()), _stream()))


def fno_adam_step(n, param, grad, m, v, lr, beta1, beta2, eps, step) -> None:
    _check(lib().fno_adam_step(ctypes.c_int64(n), _ptr(param, name="param"), _ptr(grad, name="grad"),
                               _ptr(m, name="m"), _ptr(v, name="v"), ctypes.c_double(lr), ctypes.c_double(beta1),
                               ctypes.c_double(beta2), ctypes.c_double(eps), ctypes.c_int32(step), _stream()))


def make_norm_desc(batch: int, channels: int, groups: int, npoints: int, layout: int = FNO_LAYOUT_CHANNELS_FIRST,
                   dtype: int = FNO_DTYPE_F32, activation: int = FNO_ACT_GELU, eps: float = 1e-5,
                   flags: int = 0) -> FnoNormDesc:
    return FnoNormDesc(npoints, eps, batch, channels, groups, layout, dtype, activation, flags)


def fno_group_norm_workspace_bytes(desc: FnoNormDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fno_group_norm_workspace_bytes(ctypes.byref(desc), ctypes.byref(n)))
    return int(n.value)


def alloc_norm_workspace(desc: FnoNormDesc, device="cuda") -> torch.Tensor:
    return torch.empty(max(fno_group_norm_workspace_bytes(desc), 256), dtype=torch.uint8, device=device)


def _norm_sizes(desc):
    """Type and number of a field's values; number of channels and of groups."""
    dtype = torch.bfloat16 if desc.dtype == FNO_DTYPE_BF16 else torch.float32
    batch, channels = desc.batch, desc.channels
    return dtype, batch * channels * desc.npoints, channels, batch * desc.groups


def fno_group_norm_fwd(desc, x, gamma, beta, y, mean, rstd, ws) -> None:
    dtype, field, channels, groups = _norm_sizes(desc)
    f32 = torch.float32
    status = lib().fno_group_norm_fwd(
        ctypes.byref(desc), _address(x, dtype, field, "x"), _address(gamma, f32, channels, "gamma"),
        _address(beta, f32, channels, "beta"), _address(y, dtype, field, "y"), _address(mean, f32, groups, "mean"),
        _address(rstd, f32, groups, "rstd"), _address(ws, torch.uint8, ws.numel(), "ws"), ws.numel(), _raw_stream())
    if status:
        _check(status)


def fno_group_norm_bwd(desc, x, gamma, beta, mean, rstd, gy, gx, ggamma, gbeta, ws) -> None:
    dtype, field, channels, groups = _norm_sizes(desc)
    f32 = torch.float32
    status = lib().fno_group_norm_bwd(
        ctypes.byref(desc), _address(x, dtype, field, "x"), _address(gamma, f32, channels, "gamma"),
        _address(beta, f32, channels, "beta"), _address(mean, f32, groups, "mean"), _address(rstd, f32, groups, "rstd"),
        _address(gy, dtype, field, "gy"), _address(gx, dtype, field, "gx"), _address(ggamma, f32, channels, "ggamma"),
        _address(gbeta, f32, channels, "gbeta"), _address(ws, torch.uint8, ws.numel(), "ws"), ws.numel(), _raw_stream())
    if status:
        _check(status)


class AdamwTensors:
    """The host array of tensors that fno_adamw_step, fno_grad_norm and fno_adamw_state_read take, and the tensors
    themselves, which have to live as long as the array is used.  Built by make_adamw_tensors().  The array holds addresses: a
    program that puts another tensor in the place of one of these (a new gradient every step, as after grad = None) has to
    build the list again, or the calls go on with the old one."""

    def __init__(self, array, count, sizes, bits, device, keep):
        self.array, self.count, self.sizes, self.bits, self.device, self.keep = array, count, sizes, bits, device, keep


def adamw_exps_shape(n: int) -> tuple:
    """Shape of the uint8 tensor with the shared exponents of a tensor of n values (a complex one has 2 n)."""
    return (-(-n // 256), 2)


def make_adamw_tensors(params, grads, m, v, exps=None, weight_decay=0.0) -> AdamwTensors:
    """Lists of tensors on one GPU: parameters and gradients in float32 (or complex64, as pairs of floats), moments in
    float32, or in uint8 with exps (uint8, adamw_exps_shape()).  weight_decay: one number, or one a tensor."""
    count = len(params)
    decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * count
    if not (len(grads) == len(m) == len(v) == len(decay) == count) or (exps is not None and len(exps) != count):
        raise ValueError("params, grads, m, v, exps and weight_decay must have one entry a tensor")
    state = torch.float32 if exps is None else torch.uint8
    array, sizes = (FnoAdamwTensor * max(count, 1))(), []
    devices = set()
    for k in range(count):
        n = params[k].numel() * (2 if params[k].is_complex() else 1)
        _expect(grads[k], f"grads[{k}]", n)
        _expect(m[k], f"m[{k}]", n)
        _expect(v[k], f"v[{k}]", n)
        e = None if exps is None else exps[k]
        if e is not None and e.numel() != 2 * -(-n // 256):
            raise ValueError(f"exps[{k}] holds {e.numel()} bytes, its tensor implies {2 * -(-n // 256)}")
        array[k] = FnoAdamwTensor(_ptr(params[k], name=f"params[{k}]"), _ptr(grads[k], name=f"grads[{k}]"),
                                  _ptr(m[k], state, f"m[{k}]"), _ptr(v[k], state, f"v[{k}]"),
                                  _ptr(e, torch.uint8, f"exps[{k}]"), n, decay[k])
        sizes.append(n)
        devices |= {t.device for t in (params[k], grads[k], m[k], v[k]) + (() if e is None else (e,))}
    if len(devices) > 1:
        raise ValueError("all tensors of a list must live on one GPU")
    return AdamwTensors(array, count, sizes, 32 if exps is None else 8, devices.pop() if devices else None,
                        (list(params), list(grads), list(m), list(v), None if exps is None else list(exps)))


def _list_stream(tensors: AdamwTensors) -> int:
    """The current stream, for a list whose tensors live on the current GPU: the call goes to that stream alone."""
    current = torch.cuda.current_device()
    if tensors.device is not None and tensors.device.index != current:
        raise ValueError(f"the tensors of the list live on {tensors.device}, the current device is cuda:{current}")
    return _raw_stream(current)


def fno_adamw_step(tensors: AdamwTensors, lr, beta1, beta2, eps, step, grad_norm=None, max_norm=1.0, seed=0) -> None:
    status = lib().fno_adamw_step(tensors.count, tensors.array, tensors.bits, lr, beta1, beta2, eps, step,
                                  _address(grad_norm, torch.float32, 1, "grad_norm"), max_norm, seed, _list_stream(tensors))
    if status:
        _check(status)


def fno_grad_norm_workspace_bytes(tensors: AdamwTensors) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fno_grad_norm_workspace_bytes(ctypes.c_int32(tensors.count), tensors.array, ctypes.byref(n)))
    return int(n.value)


def alloc_grad_norm_workspace(tensors: AdamwTensors, device="cuda") -> torch.Tensor:
    return torch.empty(max(fno_grad_norm_workspace_bytes(tensors), 256), dtype=torch.uint8, device=device)


def fno_grad_norm(tensors: AdamwTensors, norm, ws) -> None:
    status = lib().fno_grad_norm(tensors.count, tensors.array, _address(norm, torch.float32, 1, "norm"),
                                 _address(ws, torch.uint8, ws.numel(), "ws"), ws.numel(), _list_stream(tensors))
    if status:
        _check(status)


def fno_adamw_state_read(tensors: AdamwTensors, m_out, v_out) -> None:
    """bf16 tensors m_out[k], v_out[k] receive what the 8-bit moments of tensor k stand for."""
    if tensors.bits != 8:
        raise ValueError("the moments of this list are in 32 bits")
    count, bf16 = tensors.count, torch.bfloat16
    if len(m_out) != count or len(v_out) != count:
        raise ValueError("m_out and v_out must have one entry a tensor")
    outs = [(ctypes.c_void_p * max(count, 1))(*[_address(t, bf16, n, name) for t, n in zip(out, tensors.sizes)])
            for name, out in (("m_out", m_out), ("v_out", v_out))]
    status = lib().fno_adamw_state_read(count, tensors.array, outs[0], outs[1], _list_stream(tensors))
    if status:
        _check(status)


def fno_pointwise_mlp2(batch, c_in, hidden, c_out, npoints, x, W1, b1, W2, b2, y) -> None:
    _check(lib().fno_pointwise_mlp2(ctypes.c_int32(batch), ctypes.c_int32(c_in), ctypes.c_int32(hidden),
                                    ctypes.c_int32(c_out), ctypes.c_int64(npoints), _ptr(x, name="x"),
                                    _ptr(W1, name="W1"), _ptr(b1, name="b1"), _ptr(W2, name="W2"),
                                    _ptr(b2, name="b2"), _ptr(y, name="y"), _stream()))


FNO_TIMING_ALL = -1


def fno_timing_enable(stages) -> None:
    """True: every stage; False: off; else stage names (as in STAGE_NAMES) to time alone."""
    if stages is True:
        mask = FNO_TIMING_ALL
    elif not stages:
        mask = 0
    else:
        mask = 0
        for name in stages:
            mask |= 1 << STAGE_NAMES.index(name)
    _check(lib().fno_timing_enable(ctypes.c_int(mask)))


def fno_timing_read(capacity: int = 8192):
    """List of (stage name, milliseconds) in launch order since the last read."""
    stages = (ctypes.c_int32 * capacity)()
    ms = (ctypes.c_float * capacity)()
    n = ctypes.c_int32(0)
    _check(lib().fno_timing_read(stages, ms, ctypes.c_int32(capacity), ctypes.byref(n)))
    return [(STAGE_NAMES[stages[i]], float(ms[i])) for i in range(n.value)]
