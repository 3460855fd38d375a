"""Python entry points of include/snn_ops.h: the causal convolution along time, the selective scan, the gated linear
recurrence, group norm, gated units, and AdamW.

Marshalling only, as in binding.py: PyTorch gives device memory (outputs, workspaces) and the stream, which is the
current one of the tensors' device.  Nothing here waits for the GPU, and there is no other path: without the built
library or a device the calls raise.  Tensors are time-major, [T, B, D] with the channels dense; any strides between
steps and between sequences are taken as they are.  Streamed tensors are float32 or bfloat16, all of one call alike;
parameters and scan states are float32.  What does not fit raises SnnError before anything is launched.

Gradients are explicit calls, as snn_backward is: `causal_conv_backward`, `selective_scan_backward` and their like take what
the forward call took and return a tuple of gradients with names.  (No autograd node is recorded; a caller who wants one
wraps the pair in a torch.autograd.Function.)
"""
from __future__ import annotations

import ctypes as C
import operator
import struct
from typing import NamedTuple, Optional, Sequence

import numpy as np

from . import binding
from .binding import SnnError

BLOCK = 128                       # SNN_ADAMW_BLOCK
MAX_TAPS, MAX_STATES = 8, 64
ACTS = {"silu": 0, "gelu": 1}     # snn_act
ERR_ARG, ERR_SHAPE = 2, 3
_DTYPE, _SHAPE = operator.attrgetter("dtype"), operator.attrgetter("shape")


class _Rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("stride_t", C.c_int64), ("stride_b", C.c_int64)]


class _ConvArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("T", "B", "D", "W", "type", "silu")] + [("x", _Rows), ("y", _Rows)] + \
               [(n, C.c_void_p) for n in ("weight", "bias", "init", "lengths", "state")]


class _ConvGrads(C.Structure):
    _fields_ = [("dy", _Rows), ("dx", _Rows)] + [(n, C.c_void_p) for n in ("d_state", "dweight", "dbias", "dinit")]


class _ScanArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("T", "B", "D", "N", "groups", "type", "softplus")] + \
               [(n, _Rows) for n in ("x", "dt", "z", "bv", "cv", "y")] + \
               [(n, C.c_void_p) for n in ("A", "skip", "dt_bias", "init", "lengths", "state")]


class _ScanGrads(C.Structure):
    _fields_ = [("dy", _Rows), ("d_state", C.c_void_p)] + [(n, _Rows) for n in ("dx", "ddt", "dz", "dbv", "dcv")] + \
               [(n, C.c_void_p) for n in ("dA", "dskip", "ddt_bias", "dinit")]


class _RecArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("T", "B", "D", "type")] + [("sharpness", C.c_float)] + [(n, _Rows) for n in ("x", "i", "r", "y")] + \
               [(n, C.c_void_p) for n in ("decay", "init", "lengths", "state")]


class _RecGrads(C.Structure):
    _fields_ = [("dy", _Rows), ("d_state", C.c_void_p)] + [(n, _Rows) for n in ("dx", "di", "dr")] + [(n, C.c_void_p) for n in ("ddecay", "dinit")]


class _NormArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("T", "B", "D", "groups", "type", "silu", "per_step")] + [("eps", C.c_float)] + \
               [(n, _Rows) for n in ("x", "y")] + [(n, C.c_void_p) for n in ("weight", "bias", "lengths")]


class _NormGrads(C.Structure):
    _fields_ = [("dy", _Rows), ("dx", _Rows), ("dweight", C.c_void_p), ("dbias", C.c_void_p)]


class _UnitsArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("T", "B", "D", "F", "type", "act")] + [(n, _Rows) for n in ("x", "y")] + \
               [(n, C.c_void_p) for n in ("gate", "up", "lengths")]


class _UnitsGrads(C.Structure):
    _fields_ = [("dy", _Rows), ("dx", _Rows), ("dgate", C.c_void_p), ("dup", C.c_void_p)]


class _AdamTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("copy", C.c_void_p), ("n", C.c_int64), ("at", C.c_int64),
                ("weight_decay", C.c_double)]


class _AdamArgs(C.Structure):
    _fields_ = [("bits", C.c_int32), ("grad_type", C.c_int32)] + [(n, C.c_void_p) for n in ("m", "v", "m_scale", "v_scale")] + \
               [("step", C.c_int64), ("seed", C.c_uint32)] + [(n, C.c_double) for n in ("lr", "beta1", "beta2", "eps", "grad_scale")]


class ConvOutput(NamedTuple):
    y: object
    state: object                 # [W - 1, B, D]: the last inputs of every sequence


class ConvGrads(NamedTuple):
    dx: object
    dweight: object
    dbias: object
    dinit: object


class ScanOutput(NamedTuple):
    y: object
    state: object                 # [B, D, N] after the last step of every sequence
    saved: object                 # for selective_scan_backward (save=True), else None


class ScanGrads(NamedTuple):
    dx: object
    ddt: object
    dA: object
    dB: object
    dC: object
    dD: object
    dz: object
    ddt_bias: object
    dinit: object


class RecurrenceOutput(NamedTuple):
    y: object
    state: object                 # [B, D] after the last step of every sequence
    saved: object                 # for gated_recurrence_backward (save=True), else None


class RecurrenceGrads(NamedTuple):
    dx: object
    di: object
    dr: object
    ddecay: object
    dinit: object


class NormOutput(NamedTuple):
    y: object
    saved: object                 # for group_norm_backward (save=True), else None


class NormGrads(NamedTuple):
    dx: object
    dweight: object
    dbias: object


class UnitsOutput(NamedTuple):
    y: object
    saved: object                 # for gated_units_backward (save=True), else None


class UnitsGrads(NamedTuple):
    dx: object
    dgate: object
    dup: object


torch = None                      # bound by _lib(), so that importing the package does not import torch
_declared = None
_types = None
_stream_of = None

# The argument structures are packed in one go: a call spends its host time on checks, not on fields.
_CONV = struct.Struct("6i" + "3q" * 2 + "5q")
_CONV_GRADS = struct.Struct("3q" * 2 + "4q")
_SCAN = struct.Struct("7i4x" + "3q" * 6 + "6q")
_SCAN_GRADS = struct.Struct("3qq" + "3q" * 5 + "4q")
_REC = struct.Struct("4if4x" + "3q" * 4 + "4q")
_REC_GRADS = struct.Struct("3qq" + "3q" * 3 + "2q")
_NORM = struct.Struct("7if" + "3q" * 2 + "3q")
_NORM_GRADS = struct.Struct("3q" * 2 + "2q")
_UNITS = struct.Struct("6i" + "3q" * 2 + "3q")
_UNITS_GRADS = struct.Struct("3q" * 2 + "2q")
_ADAM = struct.Struct("2i4qqI4x5d")
assert [s.size for s in (_CONV, _CONV_GRADS, _SCAN, _SCAN_GRADS, _REC, _REC_GRADS, _NORM, _NORM_GRADS, _UNITS, _UNITS_GRADS, _ADAM)] == \
    [C.sizeof(c) for c in (_ConvArgs, _ConvGrads, _ScanArgs, _ScanGrads, _RecArgs, _RecGrads, _NormArgs, _NormGrads, _UnitsArgs, _UnitsGrads, _AdamArgs)]


def _lib():
    """The built library with the signatures of these entry points (structures go in by address)."""
    global _declared, _types, _stream_of, torch
    if _declared is None:
        import torch as torch_
        torch = torch_
        lib = binding.load_library()
        vp, sz = C.c_void_p, C.c_size_t
        for name, args in (("conv_forward", [vp, vp]), ("conv_workspace_bytes", [vp, vp]), ("conv_backward", [vp, vp, vp, sz, vp]),
                           ("conv_step", [vp, vp]), ("scan_workspace_bytes", [vp, C.c_int32, vp]), ("scan_saved_bytes", [vp, vp]),
                           ("scan_forward", [vp, vp, vp, sz, vp]), ("scan_backward", [vp, vp, vp, vp, sz, vp]), ("scan_step", [vp, vp]),
                           ("recurrence_workspace_bytes", [vp, C.c_int32, vp]), ("recurrence_saved_bytes", [vp, vp]),
                           ("recurrence_forward", [vp, vp, vp, sz, vp]), ("recurrence_backward", [vp, vp, vp, vp, sz, vp]), ("recurrence_step", [vp, vp]),
                           ("norm_workspace_bytes", [vp, C.c_int32, vp]), ("norm_saved_bytes", [vp, vp]),
                           ("norm_forward", [vp, vp, vp, sz, vp]), ("norm_backward", [vp, vp, vp, vp, sz, vp]),
                           ("units_workspace_bytes", [vp, C.c_int32, vp]), ("units_saved_bytes", [vp, vp]),
                           ("units_forward", [vp, vp, vp, sz, vp]), ("units_backward", [vp, vp, vp, vp, sz, vp]),
                           ("adamw_step", [vp, vp, C.c_int32, vp]), ("adamw_network_elements", [vp, vp]),
                           ("adamw_network_step", [vp, vp, C.c_double])):
            f = getattr(lib, "snn_" + name)
            f.argtypes, f.restype = args, C.c_int32
        _types = {torch.float32: 0, torch.bfloat16: 1}
        # the handle of a device's current stream, without a Stream object around it where torch offers that
        _stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        _declared = lib
    return _declared


def _refuse(text, status=ERR_ARG):
    raise SnnError(status, text)


def _need(ok, text, status=ERR_ARG):
    if not ok:
        raise SnnError(status, text)


def _start(x):
    """snn_type and device number of a call's first tensor."""
    if _declared is None:
        _lib()
    kind = _types.get(x.dtype)
    if kind is None:
        _refuse(f"streamed tensors are float32 or bfloat16, not {x.dtype}")
    dev = x.get_device()
    if dev < 0:
        _refuse("tensors have to be on a HIP device")
    return kind, dev


def _first(x, shape):
    """The fields of the snn_rows of a call's first tensor, which the others are compared with."""
    s = x.stride()
    if s[-1] != 1 and shape[-1] > 1:
        _refuse("the channels of x have to be dense")
    return (x.data_ptr(), s[0], s[1]) if len(s) == 3 else (x.data_ptr(), 0, s[0])


def _rows(t, dtype, dev, shape, name):
    """The same of another [T, B, D] or, for one step, [B, D] tensor, which has to be like the first."""
    if t.shape != shape:
        _refuse(f"{name} is {tuple(t.shape)}, {tuple(shape)} is needed", ERR_SHAPE)
    if t.dtype is not dtype or t.get_device() != dev:
        _refuse(f"{name} has another type or device than x")
    s = t.stride()
    if s[-1] != 1 and shape[-1] > 1:
        _refuse(f"the channels of {name} have to be dense")
    return (t.data_ptr(), s[0], s[1]) if len(s) == 3 else (t.data_ptr(), 0, s[0])


def _vectors(t, dtype, dev, lead, N, name):
    """The fields of the snn_rows of a [*lead, G, N] tensor, or [*lead, N] for one group, and G."""
    k, s, shape = len(lead), t.stride(), t.shape
    grouped = len(shape) == k + 2
    g = shape[k] if grouped else 1
    if shape != ((*lead, g, N) if grouped else (*lead, N)):
        _refuse(f"{name} is {tuple(shape)}, {(*lead, g, N)} is needed", ERR_SHAPE)
    if t.dtype is not dtype or t.get_device() != dev:
        _refuse(f"{name} has another type or device than x")
    if (s[-1] != 1 and N > 1) or (grouped and g > 1 and s[k] != N):
        _refuse(f"the vectors of {name} have to be dense")
    return (t.data_ptr(), s[0], s[1]) if k == 2 else (t.data_ptr(), 0, s[0]), g


def _dense(t, dev, shape, dtype, name):
    """The address of a dense tensor, 0 for none."""
    if t is None:
        return 0
    if t.shape != shape:
        _refuse(f"{name} is {tuple(t.shape)}, {tuple(shape)} is needed", ERR_SHAPE)
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        _refuse(f"{name} has to be dense, {dtype}, on the device of x")
    return t.data_ptr()


def _call(f, dev, *args):
    """f(*args, stream): on the current stream of the device, with that device current for the launch."""
    if torch.cuda.current_device() == dev:
        rc = f(*args, _stream_of(dev))
    else:
        with torch.cuda.device(dev):
            rc = f(*args, _stream_of(dev))
    if rc:
        _check(rc)


def _check(rc):
    if rc:
        raise SnnError(rc, _declared.snn_last_error(None).decode())


def _bytes_of(f, *args):
    n = C.c_size_t(0)
    _check(f(*args, C.byref(n)))
    return n.value


def _space(n, x):
    return torch.empty(n, dtype=torch.uint8, device=x.device) if n else None


# ---------------------------------------------------------------------------------------------- convolution

def _conv_args(x, weight, bias, init, lengths, silu, step=False):
    """-> the device number, W, and the packer of the call's structure: f(y's address, the state's address)."""
    kind, dev = _start(x)
    shape = x.shape
    if len(shape) != (2 if step else 3):
        _refuse("x has to be [B, D]" if step else "x has to be [T, B, D]", ERR_SHAPE)
    *_, B, D = shape
    if B == 0 or D == 0:
        _refuse("there has to be a sequence and a channel", ERR_SHAPE)
    if weight.dim() != 2 or weight.shape[0] != D or not 1 <= weight.shape[1] <= MAX_TAPS:
        _refuse(f"weight has to be [D, W], W from 1 to {MAX_TAPS}", ERR_SHAPE)
    W, f32 = weight.shape[1], torch.float32
    T = 1 if step else shape[0]
    head = (T, B, D, W, kind, 1 if silu else 0, *_first(x, shape))
    tail = (_dense(weight, dev, (D, W), f32, "weight"), _dense(bias, dev, (D,), f32, "bias"), _dense(init, dev, (W - 1, B, D), x.dtype, "init"),
            _dense(lengths, dev, (B,), torch.int32, "lengths"))
    return dev, W, lambda y, state: _CONV.pack(*head, y, B * D, D, *tail, state)


def causal_conv(x, weight, bias=None, init=None, lengths=None, silu: bool = True) -> ConvOutput:
    """y[t] = f(bias + sum_k weight[:, k] x[t - (W-1) + k]) per channel, f = SiLU or nothing (snn_conv_forward).

    x [T, B, D]; weight [D, W] and bias [D] float32; init [W-1, B, D], the inputs before the first step (zeros without
    it); lengths [B] int32: steps beyond a sequence's length give zeros and are not looked at.  Returns y and the last
    W-1 inputs of every sequence, which `causal_conv_step` or the next call's `init` goes on from."""
    dev, W, pack = _conv_args(x, weight, bias, init, lengths, silu)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    state = torch.empty((W - 1, *x.shape[1:]), dtype=x.dtype, device=x.device)
    _call(_declared.snn_conv_forward, dev, pack(y.data_ptr(), state.data_ptr()))
    return ConvOutput(y, state)


def causal_conv_backward(dy, x, weight, bias=None, init=None, lengths=None, silu: bool = True, d_state=None) -> ConvGrads:
    """Gradients of causal_conv for dy = dL/dy and (optionally) d_state = dL/dstate; dbias and dinit are None where
    the forward call had no bias or init."""
    dev, W, pack = _conv_args(x, weight, bias, init, lengths, silu)
    a, (_, B, D) = pack(0, 0), x.shape
    dx, dweight = torch.empty_like(x, memory_format=torch.contiguous_format), torch.empty_like(weight)
    dbias = torch.empty_like(bias) if bias is not None else None
    dinit = torch.empty_like(init) if init is not None else None
    g = _CONV_GRADS.pack(*_rows(dy, x.dtype, dev, x.shape, "dy"), dx.data_ptr(), B * D, D, _dense(d_state, dev, (W - 1, B, D), x.dtype, "d_state"),
                         dweight.data_ptr(), dbias.data_ptr() if bias is not None else 0, dinit.data_ptr() if init is not None else 0)
    n = _bytes_of(_declared.snn_conv_workspace_bytes, a)
    ws = _space(n, x)
    _call(_declared.snn_conv_backward, dev, a, g, ws.data_ptr(), n)
    return ConvGrads(dx, dweight, dbias, dinit)


def causal_conv_step(x, state, weight, bias=None, silu: bool = True):
    """One step of every sequence: x [B, D] -> y [B, D]; `state` [W-1, B, D] is moved on in place."""
    dev, W, pack = _conv_args(x, weight, bias, None, None, silu, step=True)
    _need(state is not None, "state is needed")
    at = _dense(state, dev, (W - 1, *x.shape), x.dtype, "state")
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    _call(_declared.snn_conv_step, dev, pack(y.data_ptr(), at))
    return y


# --------------------------------------------------------------------------------------------- selective scan

def _scan_args(x, dt, A, B, Cv, D, z, dt_bias, softplus, init, lengths, step=False):
    """-> the device number, (N, groups), and the packer of the call's structure: f(y's address, the state's address)."""
    kind, dev = _start(x)
    shape = x.shape
    if len(shape) != (2 if step else 3):
        _refuse("x has to be [B, D]" if step else "x has to be [T, B, D]", ERR_SHAPE)
    *_, nb, nd = shape
    if nb == 0 or nd == 0:
        _refuse("there has to be a sequence and a channel", ERR_SHAPE)
    if A.dim() != 2 or A.shape[0] != nd or not 1 <= A.shape[1] <= MAX_STATES:
        _refuse(f"A has to be [D, N], N from 1 to {MAX_STATES}", ERR_SHAPE)
    N, f32, dtype, lead = A.shape[1], torch.float32, x.dtype, (nb,) if step else (shape[0], nb)
    bv, g = _vectors(B, dtype, dev, lead, N, "B")
    cv, gc = _vectors(Cv, dtype, dev, lead, N, "C")
    if g != gc or g < 1 or nd % g:
        _refuse("B and C have to have the same number of groups, which divides D", ERR_SHAPE)
    head = (1 if step else shape[0], nb, nd, N, g, kind, 1 if softplus else 0, *_first(x, shape), *_rows(dt, dtype, dev, shape, "dt"),
            *(_rows(z, dtype, dev, shape, "z") if z is not None else (0, 0, 0)), *bv, *cv)
    tail = (_dense(A, dev, (nd, N), f32, "A"), _dense(D, dev, (nd,), f32, "D"), _dense(dt_bias, dev, (nd,), f32, "dt_bias"),
            _dense(init, dev, (nb, nd, N), f32, "init"), _dense(lengths, dev, (nb,), torch.int32, "lengths"))
    return dev, (N, g), lambda y, state: _SCAN.pack(*head, y, nb * nd, nd, *tail, state)


def selective_scan(x, dt, A, B, C_, D=None, z=None, dt_bias=None, softplus: bool = True, init=None, lengths=None,
                   save: bool = False) -> ScanOutput:
    """delta = softplus(dt + dt_bias); h_t = exp(delta A) h_(t-1) + delta x B; y = (C h + D x) silu(z) (snn_scan_forward).

    x, dt, z [T, B, D]; B, C [T, B, G, N] (or [T, B, N]), channels d // (D // G) share a group's vectors; A [D, N] (any sign; -inf
    forgets at once), D, dt_bias [D] and init [B, D, N] float32; lengths [B] int32: steps beyond a sequence's length give zeros, leave its
    state alone and are not looked at.  `save` keeps the state before every 16th step for selective_scan_backward."""
    dev, (N, _), pack = _scan_args(x, dt, A, B, C_, D, z, dt_bias, softplus, init, lengths)
    lib, saved = _declared, None
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    state = torch.empty((*x.shape[1:], N), dtype=torch.float32, device=x.device)
    a = pack(y.data_ptr(), state.data_ptr())
    n = _bytes_of(lib.snn_scan_workspace_bytes, a, 0)
    ws = _space(n, x)
    if save:
        saved = torch.empty(_bytes_of(lib.snn_scan_saved_bytes, a) // 4, dtype=torch.float32, device=x.device)
    _call(lib.snn_scan_forward, dev, a, saved.data_ptr() if save else 0, ws.data_ptr() if n else 0, n)
    return ScanOutput(y, state, saved)


def selective_scan_backward(dy, saved, x, dt, A, B, C_, D=None, z=None, dt_bias=None, softplus: bool = True, init=None,
                            lengths=None, d_state=None) -> ScanGrads:
    """Gradients of selective_scan(..., save=True) for dy = dL/dy and (optionally) d_state = dL/dstate.  dD, dz,
    ddt_bias and dinit are None where the forward call had no such argument; dB and dC have B's and C's shape."""
    dev, (N, groups), pack = _scan_args(x, dt, A, B, C_, D, z, dt_bias, softplus, init, lengths)
    lib, a, (_, nb, nd) = _declared, pack(0, 0), x.shape
    _need(saved is not None, "saved is needed: call selective_scan with save=True")
    saved_at = _dense(saved, dev, (_bytes_of(lib.snn_scan_saved_bytes, a) // 4,), torch.float32, "saved")

    def like(t):
        return torch.empty_like(t, memory_format=torch.contiguous_format) if t is not None else None

    def at(t):
        return t.data_ptr() if t is not None else 0

    out = ScanGrads(like(x), like(x), like(A), like(B), like(C_), like(D), like(z), like(dt_bias), like(init))
    full, row = (nb * nd, nd), (nb * groups * N, groups * N)
    g = _SCAN_GRADS.pack(*_rows(dy, x.dtype, dev, x.shape, "dy"), _dense(d_state, dev, (nb, nd, N), torch.float32, "d_state"), at(out.dx), *full,
                         at(out.ddt), *full, at(out.dz), *full, at(out.dB), *row, at(out.dC), *row, at(out.dA), at(out.dD), at(out.ddt_bias), at(out.dinit))
    n = _bytes_of(lib.snn_scan_workspace_bytes, a, 1)
    ws = _space(n, x)
    _call(lib.snn_scan_backward, dev, a, g, saved_at, ws.data_ptr(), n)
    return out


def selective_scan_step(x, dt, state, A, B, C_, D=None, z=None, dt_bias=None, softplus: bool = True):
    """One step of every sequence: x, dt, z [B, D], B, C [B, G, N] or [B, N] -> y [B, D]; `state` [B, D, N] (float32) is
    moved on in place."""
    dev, (N, _), pack = _scan_args(x, dt, A, B, C_, D, z, dt_bias, softplus, None, None, step=True)
    _need(state is not None, "state is needed")
    at = _dense(state, dev, (*x.shape, N), torch.float32, "state")
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    _call(_declared.snn_scan_step, dev, pack(y.data_ptr(), at))
    return y


# ------------------------------------------------------------------------------------ gated linear recurrence

def _sizes(x, step):
    """The shape of a call's first tensor, [T, B, D] or, for a step, [B, D]."""
    shape = x.shape
    if len(shape) != (2 if step else 3):
        _refuse("x has to be [B, D]" if step else "x has to be [T, B, D]", ERR_SHAPE)
    if shape[-2] == 0 or shape[-1] == 0:
        _refuse("there has to be a sequence and a channel", ERR_SHAPE)
    return shape


def _like(t):
    return torch.empty_like(t, memory_format=torch.contiguous_format) if t is not None else None


def _at(t):
    return t.data_ptr() if t is not None else 0


def _saved(f, a, x):
    """A buffer for what a forward call leaves to its backward one, float32."""
    return torch.empty(_bytes_of(f, a) // 4, dtype=torch.float32, device=x.device)


def _saved_at(f, a, saved, dev, name):
    _need(saved is not None, f"saved is needed: call {name} with save=True")
    return _dense(saved, dev, (_bytes_of(f, a) // 4,), torch.float32, "saved")


def _rec_args(x, i, r, decay, sharpness, init, lengths, step=False):
    """-> the device number and the packer of the call's structure: f(y's address, the state's address)."""
    kind, dev = _start(x)
    shape, dtype, f32 = _sizes(x, step), x.dtype, torch.float32
    *_, B, D = shape
    if not 0 < sharpness <= 3e38:
        _refuse("sharpness has to be positive and finite")
    head = (1 if step else shape[0], B, D, kind, sharpness, *_first(x, shape), *_rows(i, dtype, dev, shape, "i"), *_rows(r, dtype, dev, shape, "r"))
    _need(decay is not None, "decay is needed")
    tail = (_dense(decay, dev, (D,), f32, "decay"), _dense(init, dev, (B, D), f32, "init"), _dense(lengths, dev, (B,), torch.int32, "lengths"))
    return dev, lambda y, state: _REC.pack(*head, y, B * D, D, *tail, state)


def gated_recurrence(x, i, r, decay, sharpness: float = 8.0, init=None, lengths=None, save: bool = False) -> RecurrenceOutput:
    """a = exp(-sharpness softplus(decay) sigmoid(r)); y_t = h_t = a h_(t-1) + sqrt(1 - a^2) sigmoid(i) x (snn_recurrence_forward).

    x, i, r [T, B, D]; decay [D] and init [B, D] float32; lengths [B] int32: steps beyond a sequence's length give zeros, leave its
    state alone and are not looked at.  `save` keeps the state before every 8th step for gated_recurrence_backward."""
    dev, pack = _rec_args(x, i, r, decay, sharpness, init, lengths)
    lib, y = _declared, _like(x)
    state = torch.empty(x.shape[1:], dtype=torch.float32, device=x.device)
    a = pack(y.data_ptr(), state.data_ptr())
    n = _bytes_of(lib.snn_recurrence_workspace_bytes, a, 0)
    ws = _space(n, x)
    saved = _saved(lib.snn_recurrence_saved_bytes, a, x) if save else None
    _call(lib.snn_recurrence_forward, dev, a, _at(saved), _at(ws), n)
    return RecurrenceOutput(y, state, saved)


def gated_recurrence_backward(dy, saved, x, i, r, decay, sharpness: float = 8.0, init=None, lengths=None, d_state=None) -> RecurrenceGrads:
    """Gradients of gated_recurrence(..., save=True) for dy = dL/dy and (optionally) d_state = dL/dstate; dinit is None where
    the forward call had no init."""
    dev, pack = _rec_args(x, i, r, decay, sharpness, init, lengths)
    lib, a, (_, B, D) = _declared, pack(0, 0), x.shape
    at = _saved_at(lib.snn_recurrence_saved_bytes, a, saved, dev, "gated_recurrence")
    out = RecurrenceGrads(_like(x), _like(x), _like(x), _like(decay), _like(init))
    g = _REC_GRADS.pack(*_rows(dy, x.dtype, dev, x.shape, "dy"), _dense(d_state, dev, (B, D), torch.float32, "d_state"), out.dx.data_ptr(), B * D, D,
                        out.di.data_ptr(), B * D, D, out.dr.data_ptr(), B * D, D, out.ddecay.data_ptr(), _at(out.dinit))
    n = _bytes_of(lib.snn_recurrence_workspace_bytes, a, 1)
    ws = _space(n, x)
    _call(lib.snn_recurrence_backward, dev, a, g, at, ws.data_ptr(), n)
    return out


def gated_recurrence_step(x, i, r, state, decay, sharpness: float = 8.0):
    """One step of every sequence: x, i, r [B, D] -> y [B, D]; `state` [B, D] (float32) is moved on in place."""
    dev, pack = _rec_args(x, i, r, decay, sharpness, None, None, step=True)
    _need(state is not None, "state is needed")
    at = _dense(state, dev, x.shape, torch.float32, "state")
    y = _like(x)
    _call(_declared.snn_recurrence_step, dev, pack(y.data_ptr(), at))
    return y


# ------------------------------------------------------------------------------------------------- group norm

def _norm_args(x, groups, weight, bias, silu, eps, per_step, lengths, step=False):
    """-> the device number and the packer of the call's structure: f(y's address)."""
    kind, dev = _start(x)
    shape, f32 = _sizes(x, step), torch.float32
    *_, B, D = shape
    if not isinstance(groups, int) or groups < 1 or D % groups:
        _refuse("groups has to be a whole number that divides D")
    if not 0 <= eps <= 3e38:
        _refuse("eps must not be negative and has to be finite")
    head = (1 if step else shape[0], B, D, groups, kind, 1 if silu else 0, 1 if per_step else 0, eps, *_first(x, shape))
    tail = (_dense(weight, dev, (D,), f32, "weight"), _dense(bias, dev, (D,), f32, "bias"), _dense(lengths, dev, (B,), torch.int32, "lengths"))
    return dev, lambda y: _NORM.pack(*head, y, B * D, D, *tail)


def group_norm(x, groups: int, weight=None, bias=None, silu: bool = True, eps: float = 1e-5, per_step: bool = False, lengths=None,
               save: bool = False) -> NormOutput:
    """y = f((x - mean) / sqrt(variance + eps) weight + bias), f = SiLU or nothing (snn_norm_forward).

    x [T, B, D]; weight and bias [D] float32, or None; channels d // (D // groups) form a group.  Statistics run over a group's channels
    and the steps of the sequence that exist, or with per_step over the group's channels of each step alone, as
    `group_norm_step` takes them.  lengths [B] int32: steps beyond a sequence's length give zeros and are not looked at."""
    dev, pack = _norm_args(x, groups, weight, bias, silu, eps, per_step, lengths)
    lib, y = _declared, _like(x)
    a = pack(y.data_ptr())
    n = _bytes_of(lib.snn_norm_workspace_bytes, a, 0)
    ws = _space(n, x)
    saved = _saved(lib.snn_norm_saved_bytes, a, x) if save else None
    _call(lib.snn_norm_forward, dev, a, _at(saved), _at(ws), n)
    return NormOutput(y, saved)


def group_norm_backward(dy, saved, x, groups: int, weight=None, bias=None, silu: bool = True, eps: float = 1e-5, per_step: bool = False,
                        lengths=None) -> NormGrads:
    """Gradients of group_norm(..., save=True) for dy = dL/dy; dweight and dbias are None where the forward call had no such
    argument."""
    dev, pack = _norm_args(x, groups, weight, bias, silu, eps, per_step, lengths)
    lib, a, D = _declared, pack(0), x.shape[-1]
    at = _saved_at(lib.snn_norm_saved_bytes, a, saved, dev, "group_norm")
    out = NormGrads(_like(x), _like(weight), _like(bias))
    g = _NORM_GRADS.pack(*_rows(dy, x.dtype, dev, x.shape, "dy"), out.dx.data_ptr(), x.shape[1] * D, D, _at(out.dweight), _at(out.dbias))
    n = _bytes_of(lib.snn_norm_workspace_bytes, a, 1)
    ws = _space(n, x)
    _call(lib.snn_norm_backward, dev, a, g, at, ws.data_ptr(), n)
    return out


def group_norm_step(x, groups: int, weight=None, bias=None, silu: bool = True, eps: float = 1e-5):
    """One step of every sequence, as group_norm with per_step takes it: x [B, D] -> y [B, D]."""
    dev, pack = _norm_args(x, groups, weight, bias, silu, eps, True, None, step=True)
    y = _like(x)
    a = pack(y.data_ptr())
    _call(_declared.snn_norm_forward, dev, a, 0, 0, 0)
    return y


# ------------------------------------------------------------------------------------------------ gated units

def _units_args(x, gate, up, act, lengths, step=False):
    """-> the device number, F, and the packer of the call's structure: f(y's address)."""
    kind, dev = _start(x)
    shape = _sizes(x, step)
    *_, B, D = shape
    _need(gate is not None and up is not None, "gate and up are needed")
    if gate.dim() != 2 or gate.shape[1] != D or gate.shape[0] == 0:
        _refuse("gate has to be [F, D]", ERR_SHAPE)
    if act not in ACTS:
        _refuse(f"act is one of {', '.join(ACTS)}, not {act!r}")
    F = gate.shape[0]
    head = (1 if step else shape[0], B, D, F, kind, ACTS[act], *_first(x, shape))
    tail = (_dense(gate, dev, (F, D), x.dtype, "gate"), _dense(up, dev, (F, D), x.dtype, "up"), _dense(lengths, dev, (B,), torch.int32, "lengths"))
    return dev, F, lambda y: _UNITS.pack(*head, y, B * F, F, *tail)


def _units_forward(x, gate, up, act, lengths, save, step):
    dev, F, pack = _units_args(x, gate, up, act, lengths, step)
    lib, y = _declared, torch.empty((*x.shape[:-1], F), dtype=x.dtype, device=x.device)
    a = pack(y.data_ptr())
    n = _bytes_of(lib.snn_units_workspace_bytes, a, 0)
    ws = _space(n, x)
    saved = _saved(lib.snn_units_saved_bytes, a, x) if save else None
    _call(lib.snn_units_forward, dev, a, _at(saved), _at(ws), n)
    return y, saved


def gated_units(x, gate, up, act: str = "silu", lengths=None, save: bool = False) -> UnitsOutput:
    """y = f(x gate^T) (x up^T), f = SiLU or GELU (the exact one): both products and what joins them in one kernel (snn_units_forward).

    x [T, B, D]; gate, up [F, D] of x's type; y [T, B, F].  lengths [B] int32: steps beyond a sequence's length give zeros and are
    not looked at.  `save` keeps both products (8 bytes a value) for gated_units_backward."""
    return UnitsOutput(*_units_forward(x, gate, up, act, lengths, save, False))


def gated_units_backward(dy, saved, x, gate, up, act: str = "silu", lengths=None) -> UnitsGrads:
    """Gradients of gated_units(..., save=True) for dy = dL/dy, all of x's type."""
    dev, F, pack = _units_args(x, gate, up, act, lengths)
    lib, a, (T, B, D) = _declared, pack(0), x.shape
    at = _saved_at(lib.snn_units_saved_bytes, a, saved, dev, "gated_units")
    out = UnitsGrads(_like(x), _like(gate), _like(up))
    g = _UNITS_GRADS.pack(*_rows(dy, x.dtype, dev, (T, B, F), "dy"), out.dx.data_ptr(), B * D, D, out.dgate.data_ptr(), out.dup.data_ptr())
    n = _bytes_of(lib.snn_units_workspace_bytes, a, 1)
    ws = _space(n, x)
    _call(lib.snn_units_backward, dev, a, g, at, _at(ws), n)
    return out


def gated_units_step(x, gate, up, act: str = "silu"):
    """One step of every sequence: x [B, D] -> y [B, F]."""
    return _units_forward(x, gate, up, act, None, False, True)[0]


# ------------------------------------------------------------------------------------------------------ AdamW

class AdamW:
    """AdamW over a list of dense float32 parameters, all tensors in one call (snn_adamw_step).

    `state_bits` 32 or 8; 8-bit moments take 2.06 bytes a parameter instead of 8 (see snn_ops.h for their format; `seed`
    is that of their rounding).  `weight_decay`: one value, or one per parameter.  `copies`: bfloat16 tensors (or None)
    that receive the updated parameters rounded, in the same pass.  Parameters and copies whose memory is replaced are followed;
    ones that no longer fit, or that share memory, are refused by the step.  The moments of all parameters lie in one
    buffer each, parameter i from element `at[i]` on; state_dict and load_state_dict carry them and the number of steps.  Rates
    and seed are the constructor's: a run that is resumed repeats one that went on if they are the same."""

    def __init__(self, params: Sequence, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01,
                 state_bits: int = 32, seed: int = 0, copies: Optional[Sequence] = None):
        _lib()
        self.params = list(params)
        _need(len(self.params) > 0, "there has to be a parameter")
        _need(state_bits in (32, 8), "state_bits has to be 32 or 8")
        self.device = dev = self.params[0].device
        _need(dev.type == "cuda", "parameters have to be on a HIP device")
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * len(self.params)
        self.copies = copies if copies is not None else [None] * len(self.params)
        _need(len(decay) == len(self.params), "weight_decay goes with the parameters", ERR_SHAPE)
        for p in self.params:
            _need(p.dtype == torch.float32 and p.device == dev and p.is_contiguous(), "parameters have to be dense, float32, on one device")
        self.lr, self.betas, self.eps, self.bits, self.seed, self.steps = float(lr), (float(betas[0]), float(betas[1])), float(eps), state_bits, int(seed), 0
        self.at, n = [], 0
        for p in self.params:
            self.at.append(n)
            n += -(-p.numel() // BLOCK) * BLOCK
        n = max(n, BLOCK)
        kind = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        self.m, self.v = (torch.zeros(n, dtype=torch.uint8 if state_bits == 8 else kind, device=dev).view(kind) for _ in range(2))
        self.m_scale = self.v_scale = None
        if state_bits == 8:
            self.m_scale, self.v_scale = (torch.ones(n // BLOCK, device=dev) for _ in range(2))
        self._shapes = [p.shape for p in self.params]
        # snn_adamw_tensor, one a row; the gradients' addresses are filled in by every step
        self._table = np.zeros((len(self.params), 6), np.int64)
        self._table[:, 3], self._table[:, 4] = [p.numel() for p in self.params], self.at
        self._table[:, 5] = np.array(decay, np.float64).view(np.int64)
        self._bind()
        self._bind_copies()

    def _bind(self):
        """Takes the parameters' memory as it is now.  The optimiser holds on to that memory and to how it is seen (`_held`:
        storage, offset, sizes, strides); a parameter that is still set to that, and of that type, need not be looked at again."""
        for p, shape in zip(self.params, self._shapes):
            if p.shape != shape or p.dtype != torch.float32 or p.device != self.device or not p.is_contiguous():
                _refuse("a parameter is not what it was when the optimiser was made")
        self._held = [p.detach() for p in self.params]
        self._table[:, 0] = [p.data_ptr() for p in self._held]

    def _bind_copies(self):
        """The same for the copies, whose list is a tuple from here on: one that is put in its place is seen."""
        copies = tuple(self.copies)
        _need(len(copies) == len(self.params), "copies go with the parameters", ERR_SHAPE)
        for c, shape in zip(copies, self._shapes):
            if c is not None and (c.shape != shape or c.dtype != torch.bfloat16 or c.device != self.device or not c.is_contiguous()):
                _refuse("copies have to be dense, bfloat16, of their parameters' shapes, on their device", ERR_SHAPE)
        self.copies = self._seen = copies
        self._copied = [c for c in copies if c is not None]
        self._held_copies = [c.detach() for c in self._copied]
        self._table[:, 2] = [0 if c is None else c.data_ptr() for c in copies]

    def step(self, grads: Sequence, lr: Optional[float] = None, grad_scale: float = 1.0) -> None:
        """One step with these gradients (dense, all float32 or all bfloat16, multiplied by `grad_scale` first).  Captured
        into a graph it is replayed with the step number and learning rate of the capture."""
        # (checks run over all tensors at C speed: with many small tensors they are what a step costs)
        tensor, params, dev = torch.Tensor, self.params, self.device.index
        if list(map(_SHAPE, grads)) != self._shapes or not all(map(tensor.is_contiguous, grads)):
            _refuse("a dense gradient of its shape is needed for every parameter", ERR_SHAPE)
        kind = set(map(_DTYPE, grads))
        if len(kind) != 1 or not kind <= _types.keys() or set(map(tensor.get_device, grads)) != {dev}:
            _refuse("gradients have to be all float32 or all bfloat16, on the parameters' device")
        if not all(map(tensor.is_set_to, params, self._held)) or set(map(_DTYPE, params)) != {torch.float32}:
            self._bind()
        copies = self._copied
        if self.copies is not self._seen or not all(map(tensor.is_set_to, copies, self._held_copies)) or not set(map(_DTYPE, copies)) <= {torch.bfloat16}:
            self._bind_copies()
        t = self._table
        t[:, 1] = list(map(tensor.data_ptr, grads))
        scales = (self.m_scale.data_ptr(), self.v_scale.data_ptr()) if self.bits == 8 else (0, 0)
        a = _ADAM.pack(self.bits, _types[kind.pop()], self.m.data_ptr(), self.v.data_ptr(), *scales, self.steps + 1, self.seed & 0xFFFFFFFF,
                       self.lr if lr is None else float(lr), *self.betas, self.eps, float(grad_scale))
        _call(_declared.snn_adamw_step, dev, a, t.ctypes.data, len(t))
        self.steps += 1

    def state_dict(self) -> dict:
        """The moments (the optimiser's own buffers, not copies) and the number of steps taken."""
        d = {"step": self.steps, "m": self.m, "v": self.v}
        return d | ({"m_scale": self.m_scale, "v_scale": self.v_scale} if self.bits == 8 else {})

    def load_state_dict(self, d: dict) -> None:
        names = ("m", "v") + (("m_scale", "v_scale") if self.bits == 8 else ())
        for k in names:
            own = getattr(self, k)
            _need(k in d and d[k].shape == own.shape and d[k].dtype == own.dtype, f"{k} does not fit this optimiser", ERR_SHAPE)
        _need(int(d["step"]) >= 0, "step must not be negative")
        for k in names:
            getattr(self, k).copy_(d[k])
        self.steps = int(d["step"])


class NetworkAdamW:
    """AdamW for an SNN (binding.py), in the place of its sgd_step: `step` after every `backward` (snn_adamw_network_step).
    Arguments as for AdamW; trained decays take part without weight decay."""

    def __init__(self, snn, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, state_bits: int = 32, seed: int = 0):
        lib = _lib()
        _need(state_bits in (32, 8), "state_bits has to be 32 or 8")
        self.snn, self.lr, self.betas, self.eps, self.weight_decay = snn, float(lr), (float(betas[0]), float(betas[1])), float(eps), float(weight_decay)
        self.bits, self.seed, self.steps = state_bits, int(seed), 0
        n = C.c_int64(0)
        _check(lib.snn_adamw_network_elements(snn.ctx, C.byref(n)))
        # (made in the network's stream, which the steps run on)
        with torch.cuda.stream(snn.stream):
            kind = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
            self.m, self.v = (torch.zeros(n.value, dtype=torch.uint8 if state_bits == 8 else kind, device=snn.device).view(kind) for _ in range(2))
            self.m_scale, self.v_scale = (torch.ones(n.value // BLOCK, device=snn.device) for _ in range(2)) if state_bits == 8 else (None, None)

    def step(self, lr: Optional[float] = None) -> None:
        scales = (self.m_scale.data_ptr(), self.v_scale.data_ptr()) if self.bits == 8 else (0, 0)
        a = _ADAM.pack(self.bits, 0, self.m.data_ptr(), self.v.data_ptr(), *scales, self.steps + 1, self.seed & 0xFFFFFFFF,
                       self.lr if lr is None else float(lr), *self.betas, self.eps, 1.0)
        rc = _declared.snn_adamw_network_step(self.snn.ctx, a, self.weight_decay)
        if rc:
            raise SnnError(rc, _declared.snn_last_error(self.snn.ctx).decode())
        self.steps += 1
