"""The operators on channels-last sequences: a short causal convolution, a selective scan and a group norm with an activation.

Like the rest of the binding this only marshals arguments: every function has the name of the C entry point that it calls
(include/sysconv.h has the formulas), tensors are torch CUDA tensors used as device memory, the stream is torch's current one unless
one is given, and what is wrong with the arguments is refused before anything runs.  Outputs that are not given are made with
torch.  With ``stream`` (a hipStream_t) outputs and workspaces are allocated on that stream; the inputs must be ready on it and live until it
is done with them.

Types, shapes and strides are checked and packed once for every combination that a program calls with (a "plan": what the C entry point is
told, and the workspace's size); a later call with the same ones finds it by them, which takes a third off the host time of a small call.

Outputs carry no autograd graph, also where inputs require gradients: a model that trains calls the ``_backward`` functions, as the
``torch.autograd.Function`` classes of examples/state_space_layer.py do.

The functions are reached through ``binding`` (``binding.sys_causal_conv1d`` and so on).
"""
from __future__ import annotations

import contextlib
import ctypes
import struct
from typing import NamedTuple, Optional

from . import binding as _b

SYS_F32, SYS_F16, SYS_BF16 = range(3)
SYS_ACT_NONE, SYS_ACT_SILU, SYS_ACT_RELU = range(3)
ACTIVATIONS = {"NONE": SYS_ACT_NONE, "SILU": SYS_ACT_SILU, "RELU": SYS_ACT_RELU}
SYS_MAX_CAUSAL_WIDTH = 8
SYS_MAX_STATES = 64

# sys_causal_conv1d_t, sys_selective_scan_t, sys_group_norm_t: passed as bytes, whose buffer ctypes hands on as it is
_CONV = struct.Struct("=8i4q")
_SCAN = struct.Struct("=8i12q")
_NORM = struct.Struct("=6ifi5q")

_POINTERS = {"sys_causal_conv1d": 7, "sys_causal_conv1d_backward": 12, "sys_causal_conv1d_update": 7, "sys_selective_scan": 13,
             "sys_selective_scan_backward": 22, "sys_selective_scan_update": 12, "sys_group_norm": 7, "sys_group_norm_backward": 10}
_WORKSPACES = ("sys_causal_conv1d_backward_workspace", "sys_selective_scan_workspace", "sys_selective_scan_backward_workspace",
               "sys_group_norm_workspace", "sys_group_norm_backward_workspace")
EXPORTS = [*_POINTERS, *_WORKSPACES]

_calls = None


class _EntryPoints:
    def __init__(self):
        import torch
        _b.lib()
        own = ctypes.CDLL(_b.LIB_PATH)
        for name, pointers in _POINTERS.items():
            f = getattr(own, name)
            f.argtypes, f.restype = [ctypes.c_char_p] + [ctypes.c_void_p] * (pointers + 1), ctypes.c_int      # ..., stream
            setattr(self, name, f)
        for name in _WORKSPACES:
            f = getattr(own, name)
            f.argtypes, f.restype = [ctypes.c_char_p], ctypes.c_size_t
            setattr(self, name, f)
        self.empty, self.float32 = torch.empty, torch.float32
        self.stream, self.external = torch.cuda.stream, torch.cuda.ExternalStream
        self.device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _entry_points() -> _EntryPoints:
    global _calls
    if _calls is None:
        _calls = _EntryPoints()
    return _calls


class ScanGradients(NamedTuple):
    """What sys_selective_scan_backward returns; None where the forward call had no such input."""
    du: object
    ddelta: object
    dA: object
    dB: object
    dC: object
    dD: Optional[object]
    dz: Optional[object]
    ddelta_bias: Optional[object]
    dstate: Optional[object]


_codes = {}


def _code(t, what) -> int:
    """The sys_dtype_t of a CUDA tensor."""
    if not _codes:
        import torch
        _codes.update({torch.float32: SYS_F32, torch.float16: SYS_F16, torch.bfloat16: SYS_BF16})
        _codes["tensor"], _codes["int32"] = torch.Tensor, torch.int32
    if not isinstance(t, _codes["tensor"]) or not t.is_cuda or t.dtype not in _codes:
        raise TypeError(f"{what} must be a float32, float16 or bfloat16 CUDA tensor")
    return _codes[t.dtype]


def _like(t, first, what, shape, dtype=None):
    """t is a CUDA tensor on first's device, of this type (first's) and shape, its last axis contiguous."""
    _code(t, what)
    if t.dtype != (first.dtype if dtype is None else dtype):
        raise TypeError(f"{what} must be {first.dtype if dtype is None else dtype}")
    if t.get_device() != first.get_device():
        raise ValueError(f"{what} must be on the device of the other tensors")
    if t.shape != shape:
        raise ValueError(f"{what} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{what} must have a contiguous last axis")
    return t


def _packed(t, first, what, shape, dtype=None):
    """The same, contiguous as a whole; None passes."""
    if t is None:
        return None
    _like(t, first, what, shape, dtype)
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t


def _ints(t, first, what, n):
    if t is None:
        return None
    if not isinstance(t, _codes["tensor"]) or not t.is_cuda or t.dtype != _codes["int32"]:
        raise TypeError(f"{what} must be an int32 CUDA tensor")
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous with {n} elements")
    if t.get_device() != first.get_device():
        raise ValueError(f"{what} must be on the device of the other tensors")
    return t


def _param(t, first, what, shape):
    """A parameter: contiguous, of first's type or float32.  Its sys_dtype_t."""
    code = _code(t, what)
    if code != SYS_F32 and t.dtype != first.dtype:
        raise TypeError(f"{what} must be float32 or of the type of the activations")
    _packed(t, first, what, shape, t.dtype)
    return code


def _activation(a) -> int:
    return ACTIVATIONS[a.upper()] if isinstance(a, str) else int(a)


def _ptr(t):
    return None if t is None else t.data_ptr()


_plans = {}


def _planned(make, options, *tensors):
    """make(*tensors, *options), kept by what it depends on: the types, devices, shapes and strides of the tensors, and the options."""
    try:
        key = (make, options, *[None if t is None else (t.dtype, t.get_device(), t.shape, t.stride()) for t in tensors])
        plan = _plans.get(key)
    except (AttributeError, TypeError, RuntimeError):          # what is no tensor is refused by make
        key = plan = None
    if plan is None:
        plan = make(*tensors, *options)
        if key is not None:
            if len(_plans) >= 4096:
                _plans.clear()
            _plans[key] = plan
    return plan


def _allocated(t, stream, make):
    """Outputs and workspace of a call, allocated on its stream."""
    if t.get_device() != _calls.device():
        raise ValueError("the tensors must be on the current device")
    if stream is None:
        return make(_calls.empty, t.device)
    with _calls.stream(_calls.external(int(stream), device=t.device)):
        return make(_calls.empty, t.device)


def _run(name, packed, stream, *pointers):
    status = getattr(_calls, name)(packed, *pointers, _b._stream_handle(stream))
    if status:
        _b._check(status)


def _floats(size):
    return (size + 3) // 4


def _packed_strides(shape):
    """Batch and row strides of a contiguous tensor of this shape."""
    return shape[1] * shape[2], shape[2]


# ---------------------------------------------------------------- causal convolution

def _conv_arguments(d_x, d_w, d_bias, activation, rows):
    code = _code(d_x, "d_x")
    if d_x.dim() != rows + 1:
        raise ValueError("d_x must be [batch, length, channels]" if rows == 2 else "d_x must be [requests, channels]")
    channels = d_x.shape[-1]
    if d_x.stride(-1) != 1 and channels > 1:
        raise ValueError("d_x must have a contiguous last axis")
    _code(d_w, "d_w")
    if d_w.dim() != 2:
        raise ValueError("d_w must be [channels, width]")
    params = _param(d_w, d_x, "d_w", (channels, d_w.shape[1]))
    if d_bias is not None and _param(d_bias, d_x, "d_bias", (channels,)) != params:
        raise TypeError("d_w and d_bias must have one type")
    return code, params, channels, d_w.shape[1], _activation(activation)


def _conv_plan(d_x, d_w, d_bias, d_state, d_lengths, d_other, d_state_out, activation, backward):
    code, params, channels, width, act = _conv_arguments(d_x, d_w, d_bias, activation, 2)
    batch, length = d_x.shape[0], d_x.shape[1]
    states = (batch, width - 1, channels)
    _packed(d_state, d_x, "d_state", states)
    _packed(d_state_out, d_x, "d_dstate_out" if backward else "d_state_out", states)
    _ints(d_lengths, d_x, "d_lengths", batch)
    if d_other is not None or backward:
        _like(d_other, d_x, "d_dy" if backward else "d_y", d_x.shape)
    c = _calls or _entry_points()
    other = _packed_strides(d_x.shape) if d_other is None else (d_other.stride(0), d_other.stride(1))
    packed = _CONV.pack(code, params, act, width, batch, length, channels, 0, d_x.stride(0), d_x.stride(1), *other)
    return packed, _floats(c.sys_causal_conv1d_backward_workspace(packed)) if backward else 0


def sys_causal_conv1d(d_x, d_w, d_bias=None, d_y=None, activation="NONE", d_state=None, d_state_out=None, d_lengths=None, stream=None):
    """y[b,t,c] = act(bias[c] + sum_j w[c,j] x[b, t-(width-1)+j, c]).  d_x: [batch, length, channels] (any batch and row strides);
    d_w: [channels, width]; d_state, d_state_out: [batch, width-1, channels]; d_lengths: int32 [batch].  Returns d_y."""
    packed, _ = _planned(_conv_plan, (activation, False), d_x, d_w, d_bias, d_state, d_lengths, d_y, d_state_out)
    d_y = _allocated(d_x, stream, lambda empty, device: empty(d_x.shape, dtype=d_x.dtype, device=device) if d_y is None else d_y)
    _run("sys_causal_conv1d", packed, stream, d_x.data_ptr(), d_w.data_ptr(), _ptr(d_bias), _ptr(d_state), _ptr(d_lengths), d_y.data_ptr(),
         _ptr(d_state_out))
    return d_y


def sys_causal_conv1d_backward(d_dy, d_x, d_w, d_bias=None, activation="NONE", d_state=None, d_lengths=None, d_dstate_out=None, stream=None):
    """Gradients of sys_causal_conv1d: (dx, dw, dbias, dstate), the last two None where the call had no bias or state."""
    packed, floats = _planned(_conv_plan, (activation, True), d_x, d_w, d_bias, d_state, d_lengths, d_dy, d_dstate_out)

    def make(empty, device):
        like = lambda t: None if t is None else empty(t.shape, dtype=t.dtype, device=device)  # noqa: E731
        return like(d_x), like(d_w), like(d_bias), like(d_state), empty(floats, dtype=_calls.float32, device=device) if floats else None
    dx, dw, dbias, dstate, workspace = _allocated(d_x, stream, make)
    _run("sys_causal_conv1d_backward", packed, stream, d_dy.data_ptr(), d_x.data_ptr(), d_w.data_ptr(), _ptr(d_bias), _ptr(d_state),
         _ptr(d_lengths), _ptr(d_dstate_out), dx.data_ptr(), dw.data_ptr(), _ptr(dbias), _ptr(dstate), _ptr(workspace))
    return dx, dw, dbias, dstate


def _conv_step_plan(d_x, d_w, d_bias, d_state, d_slots, d_y, d_state_out, activation):
    code, params, channels, width, act = _conv_arguments(d_x, d_w, d_bias, activation, 1)
    requests = d_x.shape[0]
    _code(d_state, "d_state")
    slots = d_state.shape[0] if d_state.dim() else 0
    _packed(d_state, d_x, "d_state", (slots, width - 1, channels))
    _packed(d_state_out, d_x, "d_state_out", d_state.shape)
    _ints(d_slots, d_x, "d_slots", requests)
    if d_y is not None:
        _like(d_y, d_x, "d_y", d_x.shape)
    _calls or _entry_points()
    return _CONV.pack(code, params, act, width, requests, 1, channels, slots, d_x.stride(0), 0, channels if d_y is None else d_y.stride(0), 0)


def sys_causal_conv1d_update(d_x, d_w, d_bias, d_state, d_y=None, activation="NONE", d_slots=None, d_state_out=None, stream=None):
    """One token a request: d_x [requests, channels], d_state [slots, width-1, channels], updated in place (or into d_state_out) at
    the slots of d_slots (int32; request i has slot i without it; a slot that is not there skips its request).  Returns d_y."""
    packed = _planned(_conv_step_plan, (activation,), d_x, d_w, d_bias, d_state, d_slots, d_y, d_state_out)
    d_y = _allocated(d_x, stream, lambda empty, device: empty(d_x.shape, dtype=d_x.dtype, device=device) if d_y is None else d_y)
    _run("sys_causal_conv1d_update", packed, stream, d_x.data_ptr(), d_w.data_ptr(), _ptr(d_bias), d_state.data_ptr(), _ptr(d_slots),
         d_y.data_ptr(), _ptr(d_state if d_state_out is None else d_state_out))
    return d_y


# ---------------------------------------------------------------- selective scan

def _scan_arguments(d_u, d_delta, d_A, d_B, d_C, d_D, d_z, d_delta_bias, rows):
    code = _code(d_u, "d_u")
    if d_u.dim() != rows + 1:
        raise ValueError("d_u must be [batch, length, channels]" if rows == 2 else "d_u must be [requests, channels]")
    import torch
    f32, channels = torch.float32, d_u.shape[-1]
    _like(d_u, d_u, "d_u", d_u.shape)
    _like(d_delta, d_u, "d_delta", d_u.shape)
    if d_z is not None:
        _like(d_z, d_u, "d_z", d_u.shape)
    _code(d_A, "d_A")
    if d_A.dim() != 2:
        raise ValueError("d_A must be [channels, states]")
    states = d_A.shape[1]
    _packed(d_A, d_u, "d_A", (channels, states), f32)
    _packed(d_D, d_u, "d_D", (channels,), f32)
    _packed(d_delta_bias, d_u, "d_delta_bias", (channels,), f32)
    _code(d_B, "d_B")
    if d_B.dim() != rows + 2:
        raise ValueError("d_B must be [batch, length, groups, states]" if rows == 2 else "d_B must be [requests, groups, states]")
    groups = d_B.shape[-2]
    for t, what in ((d_B, "d_B"), (d_C, "d_C")):
        _like(t, d_u, what, (*d_u.shape[:-1], groups, states))
        if groups > 1 and t.stride(-2) != states:
            raise ValueError(f"the groups of a row of {what} must be contiguous")
    return code, channels, states, groups, f32


def _strides(t):
    return (t.stride(0), t.stride(1)) if t is not None else (0, 0)


def _scan_plan(d_u, d_delta, d_A, d_B, d_C, d_D, d_z, d_delta_bias, d_state, d_lengths, d_other, d_state_out, softplus, backward):
    code, channels, states, groups, f32 = _scan_arguments(d_u, d_delta, d_A, d_B, d_C, d_D, d_z, d_delta_bias, 2)
    batch, length = d_u.shape[0], d_u.shape[1]
    _packed(d_state, d_u, "d_state", (batch, channels, states), f32)
    _packed(d_state_out, d_u, "d_dstate_out" if backward else "d_state_out", (batch, channels, states), f32)
    _ints(d_lengths, d_u, "d_lengths", batch)
    if d_other is not None or backward:
        _like(d_other, d_u, "d_dy" if backward else "d_y", d_u.shape)
    c = _calls or _entry_points()
    packed = _SCAN.pack(code, bool(softplus), batch, length, channels, states, groups, 0, *_strides(d_u), *_strides(d_delta), *_strides(d_z),
                        *_strides(d_B), *_strides(d_C), *(_packed_strides(d_u.shape) if d_other is None else _strides(d_other)))
    return packed, _floats(c.sys_selective_scan_backward_workspace(packed) if backward else c.sys_selective_scan_workspace(packed))


def sys_selective_scan(d_u, d_delta, d_A, d_B, d_C, d_D=None, d_z=None, d_delta_bias=None, d_y=None, softplus=False, d_state=None,
                       d_state_out=None, d_lengths=None, stream=None):
    """h_t = e^(s_t A) h_{t-1} + s_t u_t B_t, y_t = (C_t . h_t + D u_t) silu(z_t), s_t = delta_t + delta_bias (its softplus with
    ``softplus``).  d_u, d_delta, d_z: [batch, length, channels]; d_B, d_C: [batch, length, groups, states]; d_A [channels,
    states], d_D, d_delta_bias [channels] and the states [batch, channels, states] are float32.  Returns d_y."""
    packed, floats = _planned(_scan_plan, (softplus, False), d_u, d_delta, d_A, d_B, d_C, d_D, d_z, d_delta_bias, d_state, d_lengths, d_y, d_state_out)
    d_y, workspace = _allocated(d_u, stream, lambda empty, device: (empty(d_u.shape, dtype=d_u.dtype, device=device) if d_y is None else d_y,
                                                                    empty(floats, dtype=_calls.float32, device=device) if floats else None))
    _run("sys_selective_scan", packed, stream, d_u.data_ptr(), d_delta.data_ptr(), d_A.data_ptr(), d_B.data_ptr(), d_C.data_ptr(), _ptr(d_D),
         _ptr(d_z), _ptr(d_delta_bias), _ptr(d_state), _ptr(d_lengths), d_y.data_ptr(), _ptr(d_state_out), _ptr(workspace))
    return d_y


def sys_selective_scan_backward(d_dy, d_u, d_delta, d_A, d_B, d_C, d_D=None, d_z=None, d_delta_bias=None, softplus=False, d_state=None,
                                d_lengths=None, d_dstate_out=None, stream=None) -> ScanGradients:
    """Gradients of sys_selective_scan, computed from its inputs; those of B and C are summed over the channels of a group."""
    packed, floats = _planned(_scan_plan, (softplus, True), d_u, d_delta, d_A, d_B, d_C, d_D, d_z, d_delta_bias, d_state, d_lengths, d_dy, d_dstate_out)

    def make(empty, device):
        like = lambda t: None if t is None else empty(t.shape, dtype=t.dtype, device=device)  # noqa: E731
        return (ScanGradients(like(d_u), like(d_u), like(d_A), like(d_B), like(d_B), like(d_D), like(d_z), like(d_delta_bias), like(d_state)),
                empty(floats, dtype=_calls.float32, device=device) if floats else None)
    g, workspace = _allocated(d_u, stream, make)
    _run("sys_selective_scan_backward", packed, stream, d_dy.data_ptr(), d_u.data_ptr(), d_delta.data_ptr(), d_A.data_ptr(), d_B.data_ptr(),
         d_C.data_ptr(), _ptr(d_D), _ptr(d_z), _ptr(d_delta_bias), _ptr(d_state), _ptr(d_lengths), _ptr(d_dstate_out), g.du.data_ptr(),
         g.ddelta.data_ptr(), g.dA.data_ptr(), g.dB.data_ptr(), g.dC.data_ptr(), _ptr(g.dD), _ptr(g.dz), _ptr(g.ddelta_bias), _ptr(g.dstate),
         _ptr(workspace))
    return g


def _scan_step_plan(d_u, d_delta, d_A, d_B, d_C, d_D, d_z, d_delta_bias, d_state, d_slots, d_y, d_state_out, softplus):
    code, channels, states, groups, f32 = _scan_arguments(d_u, d_delta, d_A, d_B, d_C, d_D, d_z, d_delta_bias, 1)
    requests = d_u.shape[0]
    _code(d_state, "d_state")
    slots = d_state.shape[0] if d_state.dim() else 0
    _packed(d_state, d_u, "d_state", (slots, channels, states), f32)
    _packed(d_state_out, d_u, "d_state_out", d_state.shape, f32)
    _ints(d_slots, d_u, "d_slots", requests)
    if d_y is not None:
        _like(d_y, d_u, "d_y", d_u.shape)
    _calls or _entry_points()
    return _SCAN.pack(code, bool(softplus), requests, 1, channels, states, groups, slots, d_u.stride(0), 0, d_delta.stride(0), 0,
                      0 if d_z is None else d_z.stride(0), 0, d_B.stride(0), 0, d_C.stride(0), 0, channels if d_y is None else d_y.stride(0), 0)


def sys_selective_scan_update(d_u, d_delta, d_A, d_B, d_C, d_state, d_D=None, d_z=None, d_delta_bias=None, d_y=None, softplus=False,
                              d_slots=None, d_state_out=None, stream=None):
    """One token a request: d_u, d_delta, d_z [requests, channels], d_B, d_C [requests, groups, states], d_state float32 [slots,
    channels, states], updated in place (or into d_state_out); slots as sys_causal_conv1d_update.  Returns d_y."""
    packed = _planned(_scan_step_plan, (softplus,), d_u, d_delta, d_A, d_B, d_C, d_D, d_z, d_delta_bias, d_state, d_slots, d_y, d_state_out)
    d_y = _allocated(d_u, stream, lambda empty, device: empty(d_u.shape, dtype=d_u.dtype, device=device) if d_y is None else d_y)
    _run("sys_selective_scan_update", packed, stream, d_u.data_ptr(), d_delta.data_ptr(), d_A.data_ptr(), d_B.data_ptr(), d_C.data_ptr(),
         _ptr(d_D), _ptr(d_z), _ptr(d_delta_bias), d_state.data_ptr(), _ptr(d_slots), d_y.data_ptr(),
         _ptr(d_state if d_state_out is None else d_state_out))
    return d_y


# ---------------------------------------------------------------- group norm

def _norm_plan(d_x, d_w, d_b, d_mean, d_rstd, d_other, groups, eps, activation, backward):
    code = _code(d_x, "d_x")
    if d_x.dim() != 3:
        raise ValueError("d_x must be [batch, rows, channels]")
    batch, rows, channels = d_x.shape
    groups = int(groups)
    _like(d_x, d_x, "d_x", d_x.shape)
    params = code
    if d_w is not None:
        params = _param(d_w, d_x, "d_w", (channels,))
    if d_b is not None:
        got = _param(d_b, d_x, "d_b", (channels,))
        if d_w is not None and got != params:
            raise TypeError("d_w and d_b must have one type")
        params = got
    import torch
    for t, what in ((d_mean, "d_mean"), (d_rstd, "d_rstd")):
        if backward:
            _code(t, what)
        _packed(t, d_x, what, (batch, groups), torch.float32)
    if d_other is not None or backward:
        _like(d_other, d_x, "d_dy" if backward else "d_y", d_x.shape)
    c = _calls or _entry_points()
    packed = _NORM.pack(code, params, _activation(activation), groups, batch, channels, float(eps), 0, rows, d_x.stride(0), d_x.stride(1),
                        *(_packed_strides(d_x.shape) if d_other is None else _strides(d_other)))
    return packed, _floats(c.sys_group_norm_backward_workspace(packed) if backward else c.sys_group_norm_workspace(packed))


def sys_group_norm(d_x, groups, d_w=None, d_b=None, eps=1e-5, activation="NONE", d_y=None, d_mean=None, d_rstd=None, stream=None):
    """y = act((x - mean) * rstd * w + b), statistics over the rows of a batch entry and the channels of a group.  d_x: [batch, rows,
    channels] (rows = 1: token by token); d_mean, d_rstd: float32 [batch, groups], written where given.  Returns d_y."""
    packed, floats = _planned(_norm_plan, (groups, eps, activation, False), d_x, d_w, d_b, d_mean, d_rstd, d_y)
    d_y, workspace = _allocated(d_x, stream, lambda empty, device: (empty(d_x.shape, dtype=d_x.dtype, device=device) if d_y is None else d_y,
                                                                    empty(floats, dtype=_calls.float32, device=device) if floats else None))
    _run("sys_group_norm", packed, stream, d_x.data_ptr(), _ptr(d_w), _ptr(d_b), d_y.data_ptr(), _ptr(d_mean), _ptr(d_rstd), _ptr(workspace))
    return d_y


def sys_group_norm_backward(d_dy, d_x, groups, d_mean, d_rstd, d_w=None, d_b=None, activation="NONE", stream=None):
    """Gradients of sys_group_norm from its inputs and statistics: (dx, dw, db), the last two None without w or b."""
    packed, floats = _planned(_norm_plan, (groups, 0.0, activation, True), d_x, d_w, d_b, d_mean, d_rstd, d_dy)

    def make(empty, device):
        like = lambda t: None if t is None else empty(t.shape, dtype=t.dtype, device=device)  # noqa: E731
        return like(d_x), like(d_w), like(d_b), empty(floats, dtype=_calls.float32, device=device) if floats else None
    dx, dw, db, workspace = _allocated(d_x, stream, make)
    _run("sys_group_norm_backward", packed, stream, d_dy.data_ptr(), d_x.data_ptr(), _ptr(d_w), _ptr(d_b), d_mean.data_ptr(), d_rstd.data_ptr(),
         dx.data_ptr(), _ptr(dw), _ptr(db), _ptr(workspace))
    return dx, dw, db
