"""Binding of the operators around the GEMMs (second half of include/cleave.h).

Arguments are torch tensors on the GPU; outputs are written into tensors that the caller passes.  The binding
checks what the C library cannot see (types, shapes, strides, devices) and marshals (csrc/marshal.cpp; the optimizer's
handle by ctypes); the library checks the rest and computes.  `stream` is a torch stream, a raw cudaStream_t or None
for torch's current stream; tensors that were made on another stream are the caller's to order, as with any launch.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import _marshal
from .binding import _check, lib

_vp, _u32, _u64, _i, _f, _d = C.c_void_p, C.c_uint32, C.c_uint64, C.c_int, C.c_float, C.c_double

T_NONE, T_BF16, T_F32, T_E4M3 = 0, 1, 2, 3
_TYPE = {torch.bfloat16: T_BF16, torch.float32: T_F32, torch.float8_e4m3fn: T_E4M3}
ACT = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


class _AdamwTensor(C.Structure):
    _fields_ = [("numel", _u64), ("p", _vp), ("w", _vp), ("g", _vp), ("m", _vp), ("v", _vp), ("m_scale", _vp), ("v_scale", _vp),
                ("weight_decay", _d)]


class _AdamwStep(C.Structure):
    _fields_ = [("lr", _d), ("beta1", _d), ("beta2", _d), ("eps", _d), ("grad_scale", _d), ("step", _u64), ("seed", _u64)]


class _Rmsnorm(C.Structure):
    _fields_ = [("rows", _u64), ("cols", _u32), ("x_type", _u32), ("r_type", _u32), ("w_type", _u32), ("y_type", _u32), ("eps", _f),
                ("x", _vp), ("ldx", _u64), ("r", _vp), ("ldr", _u64), ("h", _vp), ("ldh", _u64), ("w", _vp), ("y", _vp), ("ldy", _u64),
                ("rstd", _vp), ("scale", _vp)]


class _RmsnormBackward(C.Structure):
    _fields_ = [("rows", _u64), ("cols", _u32), ("dy_type", _u32), ("h_type", _u32), ("w_type", _u32), ("pad_", _u32),
                ("dy", _vp), ("lddy", _u64), ("h", _vp), ("ldh", _u64), ("w", _vp), ("rstd", _vp), ("dres", _vp), ("lddres", _u64),
                ("dx", _vp), ("lddx", _u64), ("dw", _vp)]


class _Gemm(C.Structure):
    _fields_ = [("M", _u32), ("N", _u32), ("K", _u32), ("lda", _u32), ("ldb", _u32), ("transA", C.c_uint8), ("transB", C.c_uint8),
                ("level", C.c_uint16)]


class _Linear(C.Structure):
    _fields_ = [("g", _Gemm), ("in_type", _u32), ("c_type", _u32), ("bias_type", _u32), ("z_type", _u32), ("mul_type", _u32),
                ("res_type", _u32), ("act", _u32), ("pad_", _u32), ("A", _vp), ("B", _vp), ("scale_a", _vp), ("scale_b", _vp),
                ("bias", _vp), ("z", _vp), ("ldz", _u64), ("mul", _vp), ("ldmul", _u64), ("res", _vp), ("ldres", _u64), ("C", _vp),
                ("ldc", _u64)]


class _ActBackward(C.Structure):
    _fields_ = [("rows", _u64), ("cols", _u32), ("act", _u32), ("dy_type", _u32), ("z_type", _u32), ("mul_type", _u32),
                ("dz_type", _u32), ("dmul_type", _u32), ("pad_", _u32), ("dy", _vp), ("lddy", _u64), ("z", _vp), ("ldz", _u64),
                ("mul", _vp), ("ldmul", _u64), ("dz", _vp), ("lddz", _u64), ("dmul", _vp), ("lddmul", _u64), ("dbias", _vp)]


_sig = {
    "cleave_adamw_create": (_i, [C.POINTER(_AdamwTensor), _u32, _u32, _u32, C.POINTER(_vp)]),
    "cleave_adamw_set_grads": (_i, [_vp, _vp, _vp]),
    "cleave_adamw_step": (_i, [_vp, C.POINTER(_AdamwStep), _vp]),
    "cleave_adamw_destroy": (None, [_vp]),
    "cleave_rmsnorm": (_i, [C.POINTER(_Rmsnorm), _vp]),
    "cleave_rmsnorm_backward_workspace": (_u64, [_u64, _u32]),
    "cleave_rmsnorm_backward": (_i, [C.POINTER(_RmsnormBackward), _vp, _vp]),
    "cleave_quantize_rows": (_i, [_vp, _u32, _u64, _u32, _u64, _vp, _u64, _vp, _vp]),
    "cleave_linear": (_i, [C.POINTER(_Linear), _vp]),
    "cleave_linear_status": (_i, [_vp]),
    "cleave_linear_set_wait_limit_ns": (None, [_u64]),
    "cleave_act_backward_workspace": (_u64, [_u64, _u32]),
    "cleave_act_backward": (_i, [C.POINTER(_ActBackward), _vp, _vp]),
}
for _name, (_res, _args) in _sig.items():
    _fn = getattr(lib, _name)
    _fn.restype, _fn.argtypes = _res, _args


def _raw(stream):
    """What the marshalling takes: None for torch's current stream, else the raw stream."""
    return None if stream is None else (stream if isinstance(stream, int) else stream.cuda_stream)


def _raw_stream(stream, device=None) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if device is None else device)
    return _raw(stream)


def _bad(what: str):
    raise ValueError(what)


def _act_code(act: str) -> int:
    code = ACT.get(act)
    if code is None:
        _bad(f"act: one of {', '.join(ACT)} is wanted")
    return code


def _workspace(given, nbytes: int, like, stream):
    """For a launch on another stream than torch's current one: a workspace from that stream's own pool.  (A block of the
    current stream's pool may still be in use by work queued there, which the launch does not wait for.)"""
    if given is not None or stream is None:
        return given
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=like.device) if isinstance(stream, int) else stream):
        return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=like.device)


class AdamW:
    """AdamW over many tensors, one launch a step.  Owns a cleave_adamw_t; keeps the tensors it was given alive.

    params   fp32 tensors, updated in place
    grads    bf16 or fp32 tensors (one type), read at every step; set_grads gives others
    m, v     states, updated in place: fp32 tensors, or float8_e4m3fn codes with m_scales, v_scales (fp32, one per
             256 elements); all zero at the beginning
    copies   bf16 tensors that receive the rounded weights, or None (for all, or in a tensor's place)
    weight_decay   one number, or one per tensor
    Every tensor is contiguous."""

    def __init__(self, params, grads, m, v, *, copies=None, m_scales=None, v_scales=None, weight_decay=0.0):
        self._h = None
        n = len(params)
        if n == 0 or len(grads) != n or len(m) != n or len(v) != n:
            _bad("params, grads, m and v: one of each per tensor is wanted")
        for name, tensors in (("params", params), ("grads", grads), ("m", m), ("v", v), ("m_scales", m_scales or ()), ("v_scales", v_scales or ())):
            if any(t is None for t in tensors):
                _bad(f"{name}: a tensor in every place is wanted")
        state, grad = _TYPE.get(m[0].dtype, 0), _TYPE.get(grads[0].dtype, 0)
        if state not in (T_F32, T_E4M3) or grad not in (T_BF16, T_F32):
            _bad("states are float32 or float8_e4m3fn, gradients float32 or bfloat16")
        if (state == T_E4M3) != (m_scales is not None) or (state == T_E4M3) != (v_scales is not None):
            _bad("m_scales and v_scales go with 8-bit states")
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * n
        lists = [x for x in (copies, m_scales, v_scales) if x is not None]
        if len(decay) != n or any(len(x) != n for x in lists):
            _bad("copies, scales and weight_decay: one per tensor is wanted")
        device = params[0].device
        table = (_AdamwTensor * n)()
        for i in range(n):
            size = params[i].numel()
            blocks = -(-size // 256)
            for t, kind, count, name in ((params[i], T_F32, size, "params"), (grads[i], grad, size, "grads"), (m[i], state, size, "m"),
                                         (v[i], state, size, "v"), (copies and copies[i], T_BF16, size, "copies"),
                                         (m_scales and m_scales[i], T_F32, blocks, "m_scales"), (v_scales and v_scales[i], T_F32, blocks, "v_scales")):
                if t is None:
                    continue
                if not t.is_cuda or t.device != device or _TYPE.get(t.dtype, 0) != kind or t.numel() != count or not t.is_contiguous():
                    _bad(f"{name}[{i}]: a contiguous GPU tensor of {count} elements of the common type is wanted")
            r = table[i]
            r.numel, r.p, r.g, r.m, r.v = size, params[i].data_ptr(), grads[i].data_ptr(), m[i].data_ptr(), v[i].data_ptr()
            r.w = copies[i].data_ptr() if copies is not None and copies[i] is not None else None
            r.m_scale = m_scales[i].data_ptr() if m_scales is not None and size else None
            r.v_scale = v_scales[i].data_ptr() if v_scales is not None and size else None
            r.weight_decay = float(decay[i])
        self._keep = (list(params), list(grads), list(m), list(v), lists)
        self._n, self._grad = n, grad
        self._device = device.index
        h = _vp()
        with torch.cuda.device(device):
            _check(lib.cleave_adamw_create(table, n, state, grad, C.byref(h)), "cleave_adamw_create")
        self._h = h

    def _call(self, fn, arg, stream) -> int:
        """A library call with the handle's device current (its table lives there)."""
        if torch.cuda.current_device() == self._device:
            return fn(self._h, arg, _raw_stream(stream, self._device))
        with torch.cuda.device(self._device):
            return fn(self._h, arg, _raw_stream(stream, self._device))

    def set_grads(self, grads, stream=None) -> None:
        """Other gradient tensors (same type and sizes) from the next step on."""
        if len(grads) != self._n:
            _bad("grads: one per tensor is wanted")
        for i, (g, p) in enumerate(zip(grads, self._keep[0])):
            if not g.is_cuda or g.device != p.device or _TYPE.get(g.dtype, 0) != self._grad or g.numel() != p.numel() or not g.is_contiguous():
                _bad(f"grads[{i}]: a contiguous GPU tensor of the same type and size as before is wanted")
        ptrs = (_vp * self._n)(*[g.data_ptr() for g in grads])
        _check(self._call(lib.cleave_adamw_set_grads, ptrs, stream), "cleave_adamw_set_grads")
        self._keep = (self._keep[0], list(grads)) + self._keep[2:]

    def step(self, *, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, grad_scale: float = 1.0,
             seed: int = 0, stream=None) -> None:
        """One update; `step` counts from 1.  `seed` feeds the stochastic rounding of 8-bit states."""
        if step < 1:
            _bad("step counts from 1")
        s = _AdamwStep(lr, beta1, beta2, eps, grad_scale, step, seed & 0xFFFFFFFFFFFFFFFF)
        code = self._call(lib.cleave_adamw_step, C.byref(s), stream)
        if code:
            _check(code, "cleave_adamw_step")

    def close(self) -> None:
        if self._h:
            lib.cleave_adamw_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def rmsnorm(x, weight, y, *, residual=None, h=None, rstd=None, scale=None, eps: float = 1e-5, stream=None) -> None:
    """cleave_rmsnorm: h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight, row by row.

    x, residual (and h, of its type): bf16 or fp32 [rows, cols]; weight [cols] or None; y: bf16, fp32, or
    float8_e4m3fn with `scale` fp32 [rows]; rstd fp32 [rows] or None (what the backward pass needs)."""
    code = _marshal.rmsnorm(x, weight, y, residual, h, rstd, scale, eps, _raw(stream))
    if code:
        _check(code, "cleave_rmsnorm")


def rmsnorm_backward_workspace(rows: int, cols: int) -> int:
    return lib.cleave_rmsnorm_backward_workspace(rows, cols)


def rmsnorm_backward(dy, h, weight, rstd, dx, dweight=None, *, dres=None, workspace=None, stream=None) -> None:
    """cleave_rmsnorm_backward: dx (the gradient of x and of the residual alike) and dweight (fp32, or None) from the
    saved h and rstd; `dres`, of h's type, is the gradient that reaches h from the residual stream."""
    if dweight is not None and stream is not None:
        workspace = _workspace(workspace, rmsnorm_backward_workspace(*h.shape), h, stream)
    code = _marshal.rmsnorm_backward(dy, h, weight, rstd, dx, dweight, dres, workspace, _raw(stream))
    if code:
        _check(code, "cleave_rmsnorm_backward")


def quantize_rows(x, y, scale, *, stream=None) -> None:
    """cleave_quantize_rows: y (float8_e4m3fn) = x / scale, scale fp32 [rows] = largest magnitude of the row / 448."""
    code = _marshal.quantize_rows(x, y, scale, _raw(stream))
    if code:
        _check(code, "cleave_quantize_rows")


def linear(A, B, out, *, transA: bool = False, transB: bool = False, scale_a=None, scale_b=None, bias=None, act: str = "none", z=None,
           mul=None, residual=None, stream=None) -> None:
    """cleave_linear: out = act(scale_a scale_b op(A) op(B) + bias) * mul + residual, z = the activation's argument.

    A: [M, K] ([K, M] with transA), B: [K, N] ([N, K] with transB), both bf16, or both float8_e4m3fn with
    transB.  scale_a [M], scale_b [N] fp32.  bias [N], z, mul, residual [M, N], out [M, N]: bf16 or fp32.
    `residual` may be `out` itself (an accumulation)."""
    code = _marshal.linear(A, B, out, transA, transB, scale_a, scale_b, bias, _act_code(act), z, mul, residual, _raw(stream))
    if code:
        _check(code, "cleave_linear")


def linear_status(stream=None) -> int:
    """cleave_linear_status: 0, or E_TIMEOUT when a wait inside a product ran out; synchronises the stream."""
    return lib.cleave_linear_status(_raw_stream(stream))


def act_backward_workspace(rows: int, cols: int) -> int:
    return lib.cleave_act_backward_workspace(rows, cols)


def act_backward(dy, z, dz=None, *, act: str = "none", mul=None, dmul=None, dbias=None, workspace=None, stream=None) -> None:
    """cleave_act_backward: dz = dy mul act'(z), dmul = dy act(z), dbias (fp32) = column sums of dz before its rounding."""
    if dbias is not None and stream is not None:
        workspace = _workspace(workspace, act_backward_workspace(*dy.shape), dy, stream)
    code = _marshal.act_backward(dy, z, dz, _act_code(act), mul, dmul, dbias, workspace, _raw(stream))
    if code:
        _check(code, "cleave_act_backward")
