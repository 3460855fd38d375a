"""Python entry points of include/snn_ops.h: the causal convolution along time, the selective scan, and AdamW.

Marshalling only, as in binding.py: PyTorch gives device memory (outputs, workspaces) and the stream, which is the
current one of the tensors' device.  Nothing here waits for the GPU, and there is no other path: without the built
library or a device the calls raise.  Tensors are time-major, [T, B, D] with the channels dense; any strides between
steps and between sequences are taken as they are.  Streamed tensors are float32 or bfloat16, all of one call alike;
parameters and scan states are float32.  What does not fit raises SnnError before anything is launched.

Gradients are explicit calls, as snn_backward is: `causal_conv_backward` and `selective_scan_backward` take what the
forward call took and return a tuple of gradients with names.  (No autograd node is recorded; a caller who wants one
wraps the pair in a torch.autograd.Function.)
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence

from . import binding
from .binding import SnnError

BLOCK = 128                       # SNN_ADAMW_BLOCK
MAX_TAPS, MAX_STATES = 8, 64
TILE = 16                         # steps between saved states
ERR_ARG, ERR_SHAPE = 2, 3


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


_declared = None
_types = None


def _lib():
    """The built library with the signatures of these entry points."""
    global _declared, _types
    if _declared is None:
        import torch
        lib = binding.load_library()
        vp, sz, p = C.c_void_p, C.c_size_t, C.POINTER
        lib.snn_conv_forward.argtypes = [p(_ConvArgs), vp]
        lib.snn_conv_workspace_bytes.argtypes = [p(_ConvArgs), p(sz)]
        lib.snn_conv_backward.argtypes = [p(_ConvArgs), p(_ConvGrads), vp, sz, vp]
        lib.snn_conv_step.argtypes = [p(_ConvArgs), vp]
        lib.snn_scan_workspace_bytes.argtypes = [p(_ScanArgs), C.c_int32, p(sz)]
        lib.snn_scan_saved_bytes.argtypes = [p(_ScanArgs), p(sz)]
        lib.snn_scan_forward.argtypes = [p(_ScanArgs), vp, vp, sz, vp]
        lib.snn_scan_backward.argtypes = [p(_ScanArgs), p(_ScanGrads), vp, vp, sz, vp]
        lib.snn_scan_step.argtypes = [p(_ScanArgs), vp]
        lib.snn_adamw_step.argtypes = [p(_AdamArgs), p(_AdamTensor), C.c_int32, vp]
        for name in ("conv_forward", "conv_workspace_bytes", "conv_backward", "conv_step", "scan_workspace_bytes",
                     "scan_saved_bytes", "scan_forward", "scan_backward", "scan_step", "adamw_step"):
            getattr(lib, "snn_" + name).restype = C.c_int32
        _types = {torch.float32: 0, torch.bfloat16: 1}
        _declared = lib
    return _declared


def _check(rc):
    if rc:
        raise SnnError(rc, binding.load_library().snn_last_error(None).decode())


def _need(ok, text, status=ERR_ARG):
    if not ok:
        raise SnnError(status, text)


def _type(x):
    _lib()
    _need(x.dtype in _types, f"streamed tensors are float32 or bfloat16, not {x.dtype}")
    _need(x.is_cuda, "tensors have to be on a HIP device")
    return _types[x.dtype]


def _rows(t, like, shape, name):
    """snn_rows of a [T, B, D] tensor."""
    _need(t.shape == shape, f"{name} is {tuple(t.shape)}, {tuple(shape)} is needed", ERR_SHAPE)
    _need(t.dtype == like.dtype and t.device == like.device, f"{name} has another type or device than x")
    st, sb, sd = t.stride()
    _need(sd == 1 or shape[2] <= 1, f"the channels of {name} have to be dense")
    return _Rows(t.data_ptr(), st, sb)


def _vectors(t, like, T, B, D, N, name):
    """snn_rows of a [T, B, G, N] tensor, or [T, B, N] for one group."""
    g = t.shape[2] if t.dim() == 4 else 1
    _need(tuple(t.shape) in ((T, B, g, N), (T, B, N)), f"{name} is {tuple(t.shape)}, {(T, B, g, N)} is needed", ERR_SHAPE)
    _need(t.dtype == like.dtype and t.device == like.device, f"{name} has another type or device than x")
    s = t.stride()
    _need((s[-1] == 1 or N <= 1) and (t.dim() == 3 or g <= 1 or s[2] == N), f"the vectors of {name} have to be dense")
    return _Rows(t.data_ptr(), s[0], s[1]), g


def _dense(t, like, shape, dtype, name):
    """The address of a dense tensor, or None."""
    if t is None:
        return None
    _need(tuple(t.shape) == tuple(shape), f"{name} is {tuple(t.shape)}, {tuple(shape)} is needed", ERR_SHAPE)
    _need(t.dtype == dtype and t.device == like.device and t.is_contiguous(), f"{name} has to be dense, {dtype}, on the device of x")
    return t.data_ptr()


class _On:
    """The current stream of a tensor's device, with that device the current one for the launch."""

    def __init__(self, x):
        import torch
        self.stream = C.c_void_p(torch.cuda.current_stream(x.device).cuda_stream)
        self.guard = None if torch.cuda.current_device() == x.device.index else torch.cuda.device(x.device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return self.stream

    def __exit__(self, *e):
        if self.guard is not None:
            self.guard.__exit__(*e)


def _space(n, x):
    import torch
    return torch.empty(n, dtype=torch.uint8, device=x.device) if n else None


# ---------------------------------------------------------------------------------------------- convolution

def _conv_args(x, weight, bias, init, lengths, silu):
    import torch
    kind = _type(x)
    _need(x.dim() == 3, "x has to be [T, B, D]", ERR_SHAPE)
    T, B, D = x.shape
    _need(B > 0 and D > 0, "there has to be a sequence and a channel", ERR_SHAPE)
    _need(weight.dim() == 2 and weight.shape[0] == D and 1 <= weight.shape[1] <= MAX_TAPS, f"weight has to be [D, W], W from 1 to {MAX_TAPS}", ERR_SHAPE)
    W = weight.shape[1]
    f32 = torch.float32
    a = _ConvArgs(T, B, D, W, kind, int(bool(silu)), _rows(x, x, x.shape, "x"))
    a.weight = _dense(weight, x, (D, W), f32, "weight")
    a.bias = _dense(bias, x, (D,), f32, "bias")
    a.init = _dense(init, x, (W - 1, B, D), x.dtype, "init")
    a.lengths = _dense(lengths, x, (B,), torch.int32, "lengths")
    return a


def causal_conv(x, weight, bias=None, init=None, lengths=None, silu: bool = True) -> ConvOutput:
    """y[t] = f(bias + sum_k weight[:, k] x[t - (W-1) + k]) per channel, f = SiLU or nothing (snn_conv_forward).

    x [T, B, D]; weight [D, W] and bias [D] float32; init [W-1, B, D], the inputs before the first step (zeros without
    it); lengths [B] int32: steps beyond a sequence's length give zeros and are not looked at.  Returns y and the last
    W-1 inputs of every sequence, which `causal_conv_step` or the next call's `init` goes on from."""
    import torch
    a = _conv_args(x, weight, bias, init, lengths, silu)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    state = torch.empty((a.W - 1, a.B, a.D), dtype=x.dtype, device=x.device)
    a.y, a.state = _Rows(y.data_ptr(), a.B * a.D, a.D), state.data_ptr()
    with _On(x) as st:
        _check(_declared.snn_conv_forward(C.byref(a), st))
    return ConvOutput(y, state)


def causal_conv_backward(dy, x, weight, bias=None, init=None, lengths=None, silu: bool = True, d_state=None) -> ConvGrads:
    """Gradients of causal_conv for dy = dL/dy and (optionally) d_state = dL/dstate; dbias and dinit are None where
    the forward call had no bias or init."""
    import torch
    a = _conv_args(x, weight, bias, init, lengths, silu)
    g = _ConvGrads(_rows(dy, x, x.shape, "dy"))
    g.d_state = _dense(d_state, x, (a.W - 1, a.B, a.D), x.dtype, "d_state")
    dx, dweight = torch.empty(x.shape, dtype=x.dtype, device=x.device), torch.empty_like(weight)
    dbias = torch.empty_like(bias) if bias is not None else None
    dinit = torch.empty_like(init) if init is not None else None
    g.dx, g.dweight = _Rows(dx.data_ptr(), a.B * a.D, a.D), dweight.data_ptr()
    g.dbias = dbias.data_ptr() if bias is not None else None
    g.dinit = dinit.data_ptr() if init is not None else None
    n = C.c_size_t(0)
    _check(_declared.snn_conv_workspace_bytes(C.byref(a), C.byref(n)))
    ws = _space(n.value, x)
    with _On(x) as st:
        _check(_declared.snn_conv_backward(C.byref(a), C.byref(g), ws.data_ptr(), n.value, st))
    return ConvGrads(dx, dweight, dbias, dinit)


def causal_conv_step(x, state, weight, bias=None, silu: bool = True):
    """One step of every sequence: x [B, D] -> y [B, D]; `state` [W-1, B, D] is moved on in place."""
    import torch
    _need(x.dim() == 2, "x has to be [B, D]", ERR_SHAPE)
    a = _conv_args(x[None], weight, bias, None, None, silu)
    _need(state is not None, "state is needed")
    a.state = _dense(state, x, (a.W - 1, a.B, a.D), x.dtype, "state")
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    a.y = _Rows(y.data_ptr(), 0, a.D)
    with _On(x) as st:
        _check(_declared.snn_conv_step(C.byref(a), st))
    return y


# --------------------------------------------------------------------------------------------- selective scan

def _scan_args(x, dt, A, B, Cv, D, z, dt_bias, softplus, init, lengths):
    import torch
    kind = _type(x)
    _need(x.dim() == 3, "x has to be [T, B, D]", ERR_SHAPE)
    T, nb, nd = x.shape
    _need(nb > 0 and nd > 0, "there has to be a sequence and a channel", ERR_SHAPE)
    _need(A.dim() == 2 and A.shape[0] == nd and 1 <= A.shape[1] <= MAX_STATES, f"A has to be [D, N], N from 1 to {MAX_STATES}", ERR_SHAPE)
    N, f32 = A.shape[1], torch.float32
    bv, g = _vectors(B, x, T, nb, nd, N, "B")
    cv, gc = _vectors(Cv, x, T, nb, nd, N, "C")
    _need(g == gc and g >= 1 and nd % g == 0, "B and C have to have the same number of groups, which divides D", ERR_SHAPE)
    a = _ScanArgs(T, nb, nd, N, g, kind, int(bool(softplus)), _rows(x, x, x.shape, "x"), _rows(dt, x, x.shape, "dt"))
    if z is not None:
        a.z = _rows(z, x, x.shape, "z")
    a.bv, a.cv = bv, cv
    a.A = _dense(A, x, (nd, N), f32, "A")
    a.skip = _dense(D, x, (nd,), f32, "D")
    a.dt_bias = _dense(dt_bias, x, (nd,), f32, "dt_bias")
    a.init = _dense(init, x, (nb, nd, N), f32, "init")
    a.lengths = _dense(lengths, x, (nb,), torch.int32, "lengths")
    return a


def selective_scan(x, dt, A, B, C_, D=None, z=None, dt_bias=None, softplus: bool = True, init=None, lengths=None,
                   save: bool = False) -> ScanOutput:
    """delta = softplus(dt + dt_bias); h_t = exp(delta A) h_(t-1) + delta x B; y = (C h + D x) silu(z) (snn_scan_forward).

    x, dt, z [T, B, D]; B, C [T, B, G, N] (or [T, B, N]), channels d // (D // G) share a group's vectors; A [D, N], D,
    dt_bias [D] and init [B, D, N] float32; lengths [B] int32: steps beyond a sequence's length give zeros, leave its
    state alone and are not looked at.  `save` keeps the state before every 16th step for selective_scan_backward."""
    import torch
    a = _scan_args(x, dt, A, B, C_, D, z, dt_bias, softplus, init, lengths)
    lib, n, k = _declared, C.c_size_t(0), C.c_size_t(0)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    state = torch.empty((a.B, a.D, a.N), dtype=torch.float32, device=x.device)
    a.y, a.state = _Rows(y.data_ptr(), a.B * a.D, a.D), state.data_ptr()
    _check(lib.snn_scan_workspace_bytes(C.byref(a), 0, C.byref(n)))
    ws, saved = _space(n.value, x), None
    if save:
        _check(lib.snn_scan_saved_bytes(C.byref(a), C.byref(k)))
        saved = torch.empty(k.value // 4, dtype=torch.float32, device=x.device)
    with _On(x) as st:
        _check(lib.snn_scan_forward(C.byref(a), saved.data_ptr() if save else None, ws.data_ptr() if ws is not None else None, n.value, st))
    return ScanOutput(y, state, saved)


def selective_scan_backward(dy, saved, x, dt, A, B, C_, D=None, z=None, dt_bias=None, softplus: bool = True, init=None,
                            lengths=None, d_state=None) -> ScanGrads:
    """Gradients of selective_scan(..., save=True) for dy = dL/dy and (optionally) d_state = dL/dstate.  dD, dz,
    ddt_bias and dinit are None where the forward call had no such argument; dB and dC have B's and C's shape."""
    import torch
    a = _scan_args(x, dt, A, B, C_, D, z, dt_bias, softplus, init, lengths)
    lib, n, k = _declared, C.c_size_t(0), C.c_size_t(0)
    _check(lib.snn_scan_saved_bytes(C.byref(a), C.byref(k)))
    _need(saved is not None, "saved is needed: call selective_scan with save=True")
    saved_at = _dense(saved, x, (k.value // 4,), torch.float32, "saved")
    g = _ScanGrads(_rows(dy, x, x.shape, "dy"))
    g.d_state = _dense(d_state, x, (a.B, a.D, a.N), torch.float32, "d_state")

    def streamed(like):
        return torch.empty(like.shape, dtype=x.dtype, device=x.device)

    dx, ddt, dz = streamed(x), streamed(x), streamed(x) if z is not None else None
    dB, dC, dA = streamed(B), streamed(C_), torch.empty_like(A)
    dD = torch.empty_like(D) if D is not None else None
    ddt_bias = torch.empty_like(dt_bias) if dt_bias is not None else None
    dinit = torch.empty_like(init) if init is not None else None
    step, row = a.B * a.D, a.groups * a.N
    g.dx, g.ddt = _Rows(dx.data_ptr(), step, a.D), _Rows(ddt.data_ptr(), step, a.D)
    if z is not None:
        g.dz = _Rows(dz.data_ptr(), step, a.D)
    g.dbv, g.dcv = _Rows(dB.data_ptr(), a.B * row, row), _Rows(dC.data_ptr(), a.B * row, row)
    g.dA = dA.data_ptr()
    for name, t in (("dskip", dD), ("ddt_bias", ddt_bias), ("dinit", dinit)):
        if t is not None:
            setattr(g, name, t.data_ptr())
    _check(lib.snn_scan_workspace_bytes(C.byref(a), 1, C.byref(n)))
    ws = _space(n.value, x)
    with _On(x) as st:
        _check(lib.snn_scan_backward(C.byref(a), C.byref(g), saved_at, ws.data_ptr(), n.value, st))
    return ScanGrads(dx, ddt, dA, dB, dC, dD, dz, ddt_bias, dinit)


def selective_scan_step(x, dt, state, A, B, C_, D=None, z=None, dt_bias=None, softplus: bool = True):
    """One step of every sequence: x, dt, z [B, D], B, C [B, G, N] or [B, N] -> y [B, D]; `state` [B, D, N] (float32) is
    moved on in place."""
    import torch
    _need(x.dim() == 2, "x has to be [B, D]", ERR_SHAPE)
    a = _scan_args(x[None], dt[None], A, B[None], C_[None], D, z[None] if z is not None else None, dt_bias, softplus, None, None)
    _need(state is not None, "state is needed")
    a.state = _dense(state, x, (a.B, a.D, a.N), torch.float32, "state")
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    a.y = _Rows(y.data_ptr(), 0, a.D)
    with _On(x) as st:
        _check(_declared.snn_scan_step(C.byref(a), st))
    return y


# ------------------------------------------------------------------------------------------------------ AdamW

class AdamW:
    """AdamW over a list of dense float32 parameters, all tensors in one call (snn_adamw_step).

    `state_bits` 32 or 8; 8-bit moments take 2.06 bytes a parameter instead of 8 (see snn_ops.h for their format; `seed`
    is that of their rounding).  `weight_decay`: one value, or one per parameter.  `copies`: bfloat16 tensors (or None)
    that receive the updated parameters rounded, in the same pass.  The moments of all parameters lie in one buffer
    each, parameter i from element `at[i]` on; state_dict and load_state_dict carry them."""

    def __init__(self, params: Sequence, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01,
                 state_bits: int = 32, seed: int = 0, copies: Optional[Sequence] = None):
        import torch
        _lib()
        self.params = list(params)
        _need(len(self.params) > 0, "there has to be a parameter")
        _need(state_bits in (32, 8), "state_bits has to be 32 or 8")
        dev = self.params[0].device
        _need(dev.type == "cuda", "parameters have to be on a HIP device")
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * len(self.params)
        self.copies = list(copies) if copies is not None else [None] * len(self.params)
        _need(len(decay) == len(self.params) and len(self.copies) == len(self.params), "weight_decay and copies go with the parameters", ERR_SHAPE)
        self.lr, self.betas, self.eps, self.bits, self.seed, self.steps = float(lr), betas, float(eps), state_bits, int(seed), 0
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
        self._tensors = (_AdamTensor * len(self.params))()
        for e, p, at, wd, c in zip(self._tensors, self.params, self.at, decay, self.copies):
            _need(p.dtype == torch.float32 and p.device == dev and p.is_contiguous(), "parameters have to be dense, float32, on one device")
            _need(c is None or (c.dtype == torch.bfloat16 and c.device == dev and c.is_contiguous() and c.shape == p.shape),
                  "copies have to be dense, bfloat16, of their parameters' shapes")
            e.n, e.at, e.weight_decay = p.numel(), at, float(wd)

    def step(self, grads: Sequence, lr: Optional[float] = None, grad_scale: float = 1.0) -> None:
        """One step with these gradients (dense, all float32 or all bfloat16, multiplied by `grad_scale` first)."""
        _need(len(grads) == len(self.params), "a gradient for every parameter is needed", ERR_SHAPE)
        kind, dev = grads[0].dtype, self.m.device
        _need(kind in _types, f"gradients are float32 or bfloat16, not {kind}")
        for e, p, g, c in zip(self._tensors, self.params, grads, self.copies):
            _need(g.shape == p.shape, f"a gradient is {tuple(g.shape)}, its parameter {tuple(p.shape)}", ERR_SHAPE)
            _need(g.dtype == kind and g.device == dev and g.is_contiguous(), "gradients have to be dense and alike, on the parameters' device")
            _need(p.is_contiguous() and p.numel() == e.n, "a parameter is not what it was when the optimiser was made")
            e.param, e.grad = p.data_ptr(), g.data_ptr()
            e.copy = c.data_ptr() if c is not None else None
        a = _AdamArgs(self.bits, _types[kind], self.m.data_ptr(), self.v.data_ptr(),
                      self.m_scale.data_ptr() if self.bits == 8 else None, self.v_scale.data_ptr() if self.bits == 8 else None,
                      self.steps + 1, self.seed & 0xFFFFFFFF, self.lr if lr is None else float(lr), self.betas[0], self.betas[1],
                      self.eps, float(grad_scale))
        with _On(self.m) as st:
            _check(_declared.snn_adamw_step(C.byref(a), self._tensors, len(self.params), st))
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
