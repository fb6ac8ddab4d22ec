"""Forecasting operators: Python binding of ``include/themis_forecast.h``.

``ssm_scan`` / ``ssm_scan_backward`` / ``ssm_step`` (selective state space scan with its short
causal convolution and gate) and ``linear`` / ``linear_backward`` (matrix product with bias,
activation and residual) forward to the C entry points of ``libthemis.so`` on the current torch
CUDA stream: argument checks, allocation of what the caller does not give, and pointers.  Every
step runs in the library's CUDA kernels; there is no CPU fallback.  ``SsmScan`` and ``Linear`` are
the same operators as ``torch.autograd`` functions.

Sequence tensors may be strided views (slices of one projection, say) as long as their last axis
is contiguous.  Parameters (``A``, ``conv_weight``, biases, ``skip``) are contiguous float32.
"""
from __future__ import annotations

import ctypes
import struct
from typing import NamedTuple, Optional

import torch

from . import solver
from .solver import E_INVALID_ARG, E_UNSUPPORTED_SIZE, E_WORKSPACE_TOO_SMALL, OK, STATUS_TIMEOUT, ThemisError  # noqa: F401

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
SSM_CHUNK, SSM_MAX_STATE = 16, 64

EXPORTS = (
    "themis_ssm_checkpoints", "themis_ssm_workspace_bytes", "themis_ssm_forward", "themis_ssm_backward", "themis_ssm_step",
    "themis_linear_workspace_bytes", "themis_linear_forward", "themis_linear_backward",
)

_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class SsmProblem(ctypes.Structure):
    """Mirror of ``themis_ssm_problem_t``."""
    _fields_ = ([(k, _i32) for k in ("batch", "length", "channels", "state", "groups", "conv_width", "dtype")]
                + [("flags", ctypes.c_uint32)]
                + [(k, _i64) for k in ("x_row", "x_time", "dt_row", "dt_time", "z_row", "z_time",
                                       "b_row", "b_time", "b_group", "c_row", "c_time", "c_group")])


class SsmInputs(ctypes.Structure):
    """Mirror of ``themis_ssm_inputs_t``."""
    _fields_ = [(k, _vp) for k in ("x", "dt", "z", "b", "c", "a", "conv_weight", "conv_bias", "skip", "dt_bias",
                                   "conv_state", "ssm_state", "lengths")]


class SsmOutputs(ctypes.Structure):
    """Mirror of ``themis_ssm_outputs_t``."""
    _fields_ = [(k, _vp) for k in ("y", "conv_state", "ssm_state", "checkpoints")]


class SsmGrads(ctypes.Structure):
    """Mirror of ``themis_ssm_grads_t``."""
    _fields_ = [(k, _vp) for k in ("x", "dt", "z", "b", "c", "a", "conv_weight", "conv_bias", "skip", "dt_bias")]


class LinearProblem(ctypes.Structure):
    """Mirror of ``themis_linear_problem_t``."""
    _fields_ = ([(k, _i32) for k in ("rows", "out_features", "in_features", "dtype", "activation")]
                + [("flags", ctypes.c_uint32)] + [(k, _i64) for k in ("x_row", "weight_row", "residual_row", "dy_row")])


# The calls pack these records with ``struct`` (a ctypes structure costs microseconds to fill); the
# classes above are their layout.
_PROBLEM, _INPUTS, _OUTPUTS, _GRADS = struct.Struct("@7iI12q"), struct.Struct("@13P"), struct.Struct("@4P"), struct.Struct("@10P")
_LINEAR = struct.Struct("@5iI4q")


def _bind(lib):
    sz = ctypes.c_size_t
    lib.themis_ssm_checkpoints.argtypes = [_vp, ctypes.POINTER(_i32)]
    lib.themis_ssm_workspace_bytes.argtypes = [_vp, ctypes.c_int, ctypes.POINTER(sz)]
    lib.themis_ssm_forward.argtypes = [_vp, _vp, _vp, _vp, sz, _vp]
    lib.themis_ssm_backward.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, sz, _vp]
    lib.themis_ssm_step.argtypes = [_vp, _vp, _vp, _vp]
    lib.themis_linear_workspace_bytes.argtypes = [_vp, ctypes.c_int, ctypes.c_int, ctypes.POINTER(sz)]
    lib.themis_linear_forward.argtypes = [_vp] * 8 + [_vp, sz, _vp]
    lib.themis_linear_backward.argtypes = [_vp] * 9 + [_vp, sz, _vp]
    for name in EXPORTS:
        getattr(lib, name).restype = ctypes.c_int
    return lib


_lib = _bind(ctypes.CDLL(solver.LIB_PATH))


def _check(rc: int, where: str) -> None:
    if rc != OK:
        raise ThemisError(rc, where)


class WaitExpired(RuntimeError):
    """A bounded on-device wait of an earlier product ran out: its outputs are void."""


# The word that products report to when their caller gives none: pinned host memory, which the device writes
# and the host reads without a synchronisation.
_status_memory: Optional[torch.Tensor] = None
_status_word = _i32(0)


def _default_status() -> int:
    """Its address; 0 if it would have to be allocated inside a stream capture."""
    global _status_memory, _status_word
    if _status_memory is None:
        if torch.cuda.is_current_stream_capturing():
            return 0
        _status_memory = torch.zeros(1, dtype=torch.int32, pin_memory=True)
        _status_word = _i32.from_address(_status_memory.data_ptr())
    return _status_memory.data_ptr()


def check_status() -> None:
    """Raises ``WaitExpired`` if a product that was given no ``status`` ran out of a wait and has reported it by now.  Does not
    synchronise: after a synchronisation it answers for everything before.  Every ``linear`` and ``linear_backward`` call
    begins with this check."""
    if _status_word.value:
        _status_word.value = 0
        raise WaitExpired("a bounded wait of an earlier linear or linear_backward call ran out; its outputs are void")


def _status(status: Optional[torch.Tensor], dev: int) -> int:
    """Pointer of the word that a call reports to."""
    check_status()
    return _default_status() if status is None else _full(status, (1,), torch.int32, dev, "status")


def _stream(x: torch.Tensor) -> int:
    """The current stream of the current device, which has to be the tensors'."""
    dev = x.get_device()
    if dev < 0:
        raise ValueError(f"expected CUDA tensors, got {x.device}")
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"tensors are on cuda:{dev}, the current device is cuda:{torch._C._cuda_getDevice()}")
    return torch._C._cuda_getCurrentRawStream(dev)


def _seq(t: torch.Tensor, shape, dtype: torch.dtype, dev: int, what: str) -> int:
    """Pointer of a sequence tensor: last axis contiguous, any other strides."""
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape:
        raise TypeError(f"{what}: expected {tuple(shape)} of {dtype} on {'cuda:%d' % dev if dev >= 0 else 'a CUDA device'}, "
                        f"got {tuple(t.shape)} of {t.dtype} on {t.device}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise TypeError(f"{what}: the last axis has to be contiguous")
    return t.data_ptr()


def _full(t: Optional[torch.Tensor], shape, dtype: torch.dtype, dev: int, what: str) -> int:
    """Pointer of a contiguous tensor, 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape or not t.is_contiguous():
        raise TypeError(f"{what}: expected a contiguous {tuple(shape)} tensor of {dtype} on {'cuda:%d' % dev if dev >= 0 else 'a CUDA device'}, "
                        f"got {tuple(t.shape)} of {t.dtype} on {t.device}")
    return t.data_ptr()


def _workspace(need: int, workspace: Optional[torch.Tensor], like: torch.Tensor):
    """(tensor to keep alive, pointer, bytes)"""
    if workspace is None:
        if need == 0:
            return None, None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=like.device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != like.device:
        raise TypeError(f"workspace: expected a contiguous uint8 tensor on {like.device}")
    return workspace, workspace.data_ptr(), workspace.numel()


# --- selective scan ------------------------------------------------------------------------------

def _ssm_args(x, dt, A, B, C, conv_weight, conv_bias, skip, dt_bias, z, conv_state, ssm_state, lengths, step: bool):
    """(problem, inputs, state size, conv width) of a call, arguments checked."""
    dtype, dev, shape = x.dtype, x.get_device(), x.shape
    if dtype not in DTYPES:
        raise TypeError(f"x: unsupported type {dtype}")
    dims = len(shape)
    if dims != (2 if step else 3) or A.dim() != 2 or conv_weight.dim() != 2:
        raise TypeError("x has to be [batch, channels] in a step, else [batch, length, channels]; "
                        "A [channels, state]; conv_weight [channels, width]")
    rows, channels, state, width = shape[0], shape[-1], A.shape[1], conv_weight.shape[1]
    if B.dim() == dims:             # one group, without its axis
        B, C = B.unsqueeze(-2), C.unsqueeze(-2)
    if B.dim() != dims + 1:
        raise TypeError("B: expected [..., groups, state]")
    groups = B.shape[-2]
    per_state = (rows, groups, state) if step else (rows, shape[1], groups, state)
    f32, per_channel = torch.float32, (channels,)
    inputs = _INPUTS.pack(
        _seq(x, shape, dtype, dev, "x"), _seq(dt, shape, dtype, dev, "dt"), 0 if z is None else _seq(z, shape, dtype, dev, "z"),
        _seq(B, per_state, dtype, dev, "B"), _seq(C, per_state, dtype, dev, "C"), _full(A, (channels, state), f32, dev, "A"),
        _full(conv_weight, (channels, width), f32, dev, "conv_weight"), _full(conv_bias, per_channel, f32, dev, "conv_bias"),
        _full(skip, per_channel, f32, dev, "skip"), _full(dt_bias, per_channel, f32, dev, "dt_bias"),
        _full(conv_state, (rows, width - 1, channels), dtype, dev, "conv_state"),
        _full(ssm_state, (rows, channels, state), f32, dev, "ssm_state"), _full(lengths, (rows,), torch.int32, dev, "lengths"))
    sx, sd, sb, sc = x.stride(), dt.stride(), B.stride(), C.stride()
    sz = sx if z is None else z.stride()
    if step:
        problem = _PROBLEM.pack(rows, 1, channels, state, groups, width, DTYPES[dtype], 0, sx[0], 0, sd[0], 0, sz[0], 0,
                                sb[0], 0, sb[1], sc[0], 0, sc[1])
    else:
        problem = _PROBLEM.pack(rows, shape[1], channels, state, groups, width, DTYPES[dtype], 0, sx[0], sx[1], sd[0], sd[1],
                                sz[0], sz[1], sb[0], sb[1], sb[2], sc[0], sc[1], sc[2])
    return problem, inputs, state, width


def themis_ssm_workspace_bytes(problem, backward: bool) -> int:
    """``problem``: an ``SsmProblem`` or its bytes."""
    n = ctypes.c_size_t()
    _check(_lib.themis_ssm_workspace_bytes(bytes(problem), int(backward), ctypes.byref(n)), "themis_ssm_workspace_bytes")
    return n.value


def themis_ssm_checkpoints(problem) -> int:
    n = _i32()
    _check(_lib.themis_ssm_checkpoints(bytes(problem), ctypes.byref(n)), "themis_ssm_checkpoints")
    return n.value


class ScanResult(NamedTuple):
    y: torch.Tensor                                 # [batch, length, channels]
    conv_state: Optional[torch.Tensor]              # [batch, conv_width - 1, channels]
    ssm_state: Optional[torch.Tensor]               # [batch, channels, state] float32
    checkpoints: Optional[torch.Tensor]             # [batch, ceil(length / 16), channels, state] float32


def ssm_scan(x, dt, A, B, C, conv_weight, conv_bias=None, skip=None, dt_bias=None, z=None, conv_state=None, ssm_state=None,
             lengths=None, states: bool = True, save: bool = False, workspace=None) -> ScanResult:
    """``themis_ssm_forward`` over whole histories.

    ``x``, ``dt``, ``z``: [batch, length, channels]; ``B``, ``C``: [batch, length, groups, state] (or without the
    groups' axis); ``A``: [channels, state]; ``lengths``: int32 [batch].  ``states``: return the states after every
    row's last time; ``save``: return the checkpoints that ``ssm_scan_backward`` needs."""
    problem, inputs, state, width = _ssm_args(x, dt, A, B, C, conv_weight, conv_bias, skip, dt_bias, z, conv_state, ssm_state,
                                              lengths, False)
    stream = _stream(x)
    rows, length, channels = x.shape
    y = torch.empty((rows, length, channels), dtype=x.dtype, device=x.device)
    new_conv = new_ssm = checkpoints = None
    if states:
        new_conv = torch.empty((rows, width - 1, channels), dtype=x.dtype, device=x.device)
        new_ssm = torch.empty((rows, channels, state), dtype=torch.float32, device=x.device)
    if save:
        checkpoints = torch.empty((rows, -(-length // SSM_CHUNK), channels, state), dtype=torch.float32, device=x.device)
    keep, ws, n = _workspace(themis_ssm_workspace_bytes(problem, False), workspace, x)
    out = _OUTPUTS.pack(y.data_ptr(), new_conv.data_ptr() if states else 0, new_ssm.data_ptr() if states else 0,
                        checkpoints.data_ptr() if save else 0)
    _check(_lib.themis_ssm_forward(problem, inputs, out, ws, n, stream), "themis_ssm_forward")
    return ScanResult(y, new_conv, new_ssm, checkpoints)


def ssm_scan_backward(dy, checkpoints, x, dt, A, B, C, conv_weight, conv_bias=None, skip=None, dt_bias=None, z=None,
                      conv_state=None, ssm_state=None, lengths=None, workspace=None) -> dict:
    """``themis_ssm_backward``: the gradients of ``sum(dy * y)`` for the inputs of an ``ssm_scan(..., save=True)`` call, as a
    dict ("dx", "ddt", "dA", "dB", "dC", "dconv_weight" and, for what was given, "dz", "dconv_bias", "dskip", "ddt_bias").
    Initial states are constants."""
    problem, inputs, state, width = _ssm_args(x, dt, A, B, C, conv_weight, conv_bias, skip, dt_bias, z, conv_state, ssm_state,
                                              lengths, False)
    stream, dev = _stream(x), x.get_device()
    rows, length, channels = x.shape
    saved = _full(checkpoints, (rows, -(-length // SSM_CHUNK), channels, state), torch.float32, dev, "checkpoints")
    p_dy = _full(dy, x.shape, x.dtype, dev, "dy")
    grads = {"dx": torch.empty(x.shape, dtype=x.dtype, device=x.device), "ddt": torch.empty(x.shape, dtype=x.dtype, device=x.device)}
    if z is not None:
        grads["dz"] = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    grads["dB"] = torch.empty(B.shape, dtype=x.dtype, device=x.device)
    grads["dC"] = torch.empty(C.shape, dtype=x.dtype, device=x.device)
    grads["dA"], grads["dconv_weight"] = torch.empty_like(A), torch.empty_like(conv_weight)
    for name, v in (("dconv_bias", conv_bias), ("dskip", skip), ("ddt_bias", dt_bias)):
        if v is not None:
            grads[name] = torch.empty_like(v)
    keep, ws, n = _workspace(themis_ssm_workspace_bytes(problem, True), workspace, x)
    g = _GRADS.pack(*(grads[k].data_ptr() if k in grads else 0 for k in
                      ("dx", "ddt", "dz", "dB", "dC", "dA", "dconv_weight", "dconv_bias", "dskip", "ddt_bias")))
    _check(_lib.themis_ssm_backward(problem, inputs, saved, p_dy, g, ws, n, stream), "themis_ssm_backward")
    return grads


def ssm_step(x, dt, A, B, C, conv_weight, conv_bias=None, skip=None, dt_bias=None, z=None, *, conv_state, ssm_state,
             new_conv_state=None, new_ssm_state=None, active=None) -> torch.Tensor:
    """``themis_ssm_step``: one time of every row; returns y [batch, channels].

    ``x``, ``dt``, ``z``: [batch, channels]; ``B``, ``C``: [batch, groups, state].  The states are updated in place unless
    ``new_conv_state`` / ``new_ssm_state`` are given.  ``active``: int32 [batch]; rows with 0 keep their states, y is 0."""
    problem, inputs, state, width = _ssm_args(x, dt, A, B, C, conv_weight, conv_bias, skip, dt_bias, z, conv_state, ssm_state,
                                              active, True)
    stream, dev = _stream(x), x.get_device()
    y = x.new_empty(x.shape)
    out = _OUTPUTS.pack(
        y.data_ptr(), conv_state.data_ptr() if new_conv_state is None else _full(new_conv_state, conv_state.shape, x.dtype, dev, "new_conv_state"),
        ssm_state.data_ptr() if new_ssm_state is None else _full(new_ssm_state, ssm_state.shape, torch.float32, dev, "new_ssm_state"), 0)
    _check(_lib.themis_ssm_step(problem, inputs, out, stream), "themis_ssm_step")
    return y


class _FirstOrderOnly(torch.autograd.Function):
    """A gradient as it is; differentiating it raises."""

    @staticmethod
    def forward(ctx, anchor, grad):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("the gradients of SsmScan and Linear cannot be differentiated again")


def _first_order(grads):
    """Gradients made by kernels, which autograd cannot see into: with ``create_graph=True`` they depend on a node that
    raises, so that a second derivative is refused instead of being taken as 0."""
    if not torch.is_grad_enabled():
        return grads
    anchor = torch.empty(0, requires_grad=True)
    return tuple(None if g is None else _FirstOrderOnly.apply(anchor, g) for g in grads)


class SsmScan(torch.autograd.Function):
    """``SsmScan.apply(x, dt, A, B, C, conv_weight, conv_bias, skip, dt_bias, z, lengths)`` -> y, from zero states.  Has first
    derivatives only."""

    @staticmethod
    def forward(ctx, x, dt, A, B, C, conv_weight, conv_bias=None, skip=None, dt_bias=None, z=None, lengths=None):
        args = (x, dt, A, B, C, conv_weight, conv_bias, skip, dt_bias, z)
        r = ssm_scan(*args, lengths=lengths, states=False, save=True)
        ctx.save_for_backward(r.checkpoints, lengths, *args)
        return r.y

    @staticmethod
    def backward(ctx, dy):
        checkpoints, lengths, *args = ctx.saved_tensors
        g = ssm_scan_backward(dy.contiguous(), checkpoints, *args, lengths=lengths)
        names = ("dx", "ddt", "dA", "dB", "dC", "dconv_weight", "dconv_bias", "dskip", "ddt_bias", "dz")
        return _first_order(tuple(g.get(k) for k in names)) + (None,)


# --- linear ----------------------------------------------------------------------------------------

def _rows(t: torch.Tensor, m: int, n: int, dtype: torch.dtype, dev: int, what: str):
    """(pointer, elements from one row to the next); a single row has no such number of its own"""
    p = _seq(t, (m, n), dtype, dev, what)
    if m <= 1:
        return p, n
    pitch = t.stride(0)
    if pitch < n:
        raise TypeError(f"{what}: rows overlap")
    return p, pitch


def _linear_dims(x, weight, activation: str):
    dtype = x.dtype
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        raise TypeError(f"x: unsupported type {dtype} (bfloat16 or float16)")
    if x.dim() != 2 or weight.dim() != 2:
        raise TypeError("x has to be [rows, in_features], weight [out_features, in_features]")
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation: {activation!r} is not one of {tuple(ACTIVATIONS)}")
    (m, k), n = x.shape, weight.shape[0]
    return dtype, x.get_device(), m, n, k, act


def themis_linear_workspace_bytes(problem, backward: bool, unaligned: bool = False) -> int:
    """``problem``: a ``LinearProblem`` or its bytes."""
    n = ctypes.c_size_t()
    _check(_lib.themis_linear_workspace_bytes(bytes(problem), int(backward), int(unaligned), ctypes.byref(n)),
           "themis_linear_workspace_bytes")
    return n.value


def linear(x, weight, bias=None, activation: str = "none", residual=None, save_pre: bool = False, status=None, workspace=None):
    """``themis_linear_forward``: ``act(x @ weight.T + bias) + residual``.

    ``x``: [rows, in]; ``weight``: [out, in]; ``bias``: float32 [out]; ``residual``: [rows, out].  With ``save_pre`` returns
    ``(y, pre)``, ``pre`` being what ``linear_backward`` needs of an activation.  ``status``: int32 [1], see the header; without
    it a wait that runs out is raised by a later call (``check_status``)."""
    dtype, dev, m, n, k, act = _linear_dims(x, weight, activation)
    (px, sx), (pw, sw) = _rows(x, m, k, dtype, dev, "x"), _rows(weight, n, k, dtype, dev, "weight")
    pr, sr = (None, n) if residual is None else _rows(residual, m, n, dtype, dev, "residual")
    pb = _full(bias, (n,), torch.float32, dev, "bias")
    stream, word = _stream(x), _status(status, dev)
    problem = _LINEAR.pack(m, n, k, DTYPES[dtype], act, 0, sx, sw, sr, n)
    y = x.new_empty((m, n))
    pre = x.new_empty((m, n)) if save_pre else None
    # (aligned operands need no workspace)
    unaligned = bool((px | pw) & 15)
    need = themis_linear_workspace_bytes(problem, False, unaligned) if unaligned or (sx | sw) & 7 else 0
    keep, ws, size = _workspace(need, workspace, x)
    _check(_lib.themis_linear_forward(problem, px, pw, pb, pr, y.data_ptr(), pre.data_ptr() if save_pre else None,
                                      word, ws, size, stream), "themis_linear_forward")
    return (y, pre) if save_pre else y


def linear_backward(dy, x, weight, pre=None, activation: str = "none", bias: bool = True, need_dx: bool = True,
                    need_dweight: bool = True, status=None, workspace=None) -> dict:
    """``themis_linear_backward``: "dx" and "dweight" (the type of x), "dbias" (float32) as a dict.  The residual's gradient
    is ``dy``.  ``status``: as for ``linear``."""
    dtype, dev, m, n, k, act = _linear_dims(x, weight, activation)
    (px, sx), (pw, sw) = _rows(x, m, k, dtype, dev, "x"), _rows(weight, n, k, dtype, dev, "weight")
    pd, sd = _rows(dy, m, n, dtype, dev, "dy")
    if act and pre is None:
        raise TypeError("pre: an activation's gradient needs it")
    pp = _full(pre, (m, n), dtype, dev, "pre") if act else None
    stream, word = _stream(x), _status(status, dev)
    problem = _LINEAR.pack(m, n, k, DTYPES[dtype], act, 0, sx, sw, n, sd)
    grads = {}
    if need_dx:
        grads["dx"] = x.new_empty((m, k))
    if need_dweight:
        grads["dweight"] = x.new_empty((n, k))
    if bias:
        grads["dbias"] = torch.empty((n,), dtype=torch.float32, device=x.device)
    keep, ws, size = _workspace(themis_linear_workspace_bytes(problem, True, bool((pd | px | pw) & 15)), workspace, x)
    _check(_lib.themis_linear_backward(
        problem, pd, px, pw, pp, *(grads[g].data_ptr() if g in grads else None for g in ("dx", "dweight", "dbias")),
        word, ws, size, stream), "themis_linear_backward")
    return grads


class Linear(torch.autograd.Function):
    """``Linear.apply(x, weight, bias, activation, residual)`` -> y.  Has first derivatives only."""

    @staticmethod
    def forward(ctx, x, weight, bias=None, activation="none", residual=None):
        y, pre = (linear(x, weight, bias, activation, residual, save_pre=True) if activation != "none"
                  else (linear(x, weight, bias, activation, residual), None))
        ctx.save_for_backward(x, weight, pre)
        ctx.activation, ctx.has_bias, ctx.has_residual = activation, bias is not None, residual is not None
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, pre = ctx.saved_tensors
        residual = dy if ctx.has_residual else None
        if dy.stride(-1) != 1 or (dy.shape[0] > 1 and dy.stride(0) < dy.shape[1]):
            dy = dy.contiguous()
        need = ctx.needs_input_grad
        g = linear_backward(dy, x, weight, pre, ctx.activation, bias=ctx.has_bias and need[2], need_dx=need[0], need_dweight=need[1])
        return _first_order((g.get("dx"), g.get("dweight"), g.get("dbias"))) + (None, residual)
