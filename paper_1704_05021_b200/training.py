"""The operators of a training step around the gradient exchange: ctypes binding of include/gd_train.h and the objects that hold
what its calls need between them.

`LinearSession` (a linear layer's shape and workspace), `cross_entropy` and `AdamWSession` (a list of tensors, their moments)
check the tensors they are given, marshal addresses and issue the calls.  All arithmetic happens inside libgd.so; there
is no other code path.  Tensors must live on the device the session was made for and be ready on the stream of the call: the current
stream, or the one passed as `stream`.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import struct
from typing import Optional, Sequence, Union

import torch

from . import binding as B

GD_DTYPE_FP32, GD_DTYPE_BF16, GD_DTYPE_FP16 = 0, 1, 2
GD_ACT_NONE, GD_ACT_RELU, GD_ACT_GELU, GD_ACT_SILU = 0, 1, 2, 3
GD_W_IN_OUT, GD_W_OUT_IN = 0, 1
GD_LINEAR_ACCUMULATE = 1

EXPORTS = ["gd_linear_forward", "gd_linear_backward", "gd_linear_workspace_bytes", "gd_linear_status", "gd_selftest_linear_wait", "gd_cross_entropy",
           "gd_adamw_step"]

_DTYPES = {torch.float32: GD_DTYPE_FP32, torch.bfloat16: GD_DTYPE_BF16, torch.float16: GD_DTYPE_FP16}
_ACTIVATIONS = {"none": GD_ACT_NONE, "relu": GD_ACT_RELU, "gelu": GD_ACT_GELU, "silu": GD_ACT_SILU}
_LAYOUTS = {"in_out": GD_W_IN_OUT, "out_in": GD_W_OUT_IN}
_SCALE_BLOCK = 128          # consecutive elements that share a scale in the 8-bit moments


class _LinearForwardArgs(C.Structure):
    _fields_ = [("m", C.c_uint64), ("n", C.c_uint64), ("k", C.c_uint64),
                ("dtype", C.c_int32), ("activation", C.c_int32), ("w_layout", C.c_int32), ("bias_dtype", C.c_int32),
                ("y_dtype", C.c_int32), ("reserved", C.c_int32),
                ("x", C.c_void_p), ("ldx", C.c_uint64), ("w", C.c_void_p), ("ldw", C.c_uint64), ("bias", C.c_void_p),
                ("residual", C.c_void_p), ("ld_residual", C.c_uint64), ("y", C.c_void_p), ("ldy", C.c_uint64),
                ("pre", C.c_void_p), ("ld_pre", C.c_uint64), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class _LinearBackwardArgs(C.Structure):
    _fields_ = [("m", C.c_uint64), ("n", C.c_uint64), ("k", C.c_uint64),
                ("dtype", C.c_int32), ("activation", C.c_int32), ("w_layout", C.c_int32), ("dw_dtype", C.c_int32),
                ("flags", C.c_uint32), ("reserved", C.c_int32),
                ("dy", C.c_void_p), ("ld_dy", C.c_uint64), ("pre", C.c_void_p), ("ld_pre", C.c_uint64),
                ("x", C.c_void_p), ("ldx", C.c_uint64), ("w", C.c_void_p), ("ldw", C.c_uint64),
                ("dx", C.c_void_p), ("ld_dx", C.c_uint64), ("dw", C.c_void_p), ("ld_dw", C.c_uint64), ("db", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class _CrossEntropyArgs(C.Structure):
    _fields_ = [("rows", C.c_uint64), ("classes", C.c_uint64), ("dtype", C.c_int32), ("target_bits", C.c_int32),
                ("logits", C.c_void_p), ("ld_logits", C.c_uint64), ("targets", C.c_void_p), ("ignore_index", C.c_int64),
                ("grad_scale", C.c_float), ("reserved", C.c_int32), ("grad_scale_dev", C.c_void_p),
                ("loss", C.c_void_p), ("lse", C.c_void_p), ("grad", C.c_void_p), ("ld_grad", C.c_uint64)]


class _AdamwTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("copy", C.c_void_p), ("n", C.c_uint64), ("weight_decay", C.c_double)]


class _AdamwArgs(C.Structure):
    _fields_ = [("tensors", C.POINTER(_AdamwTensor)), ("n_tensors", C.c_uint32), ("state_bits", C.c_int32),
                ("param_dtype", C.c_int32), ("grad_dtype", C.c_int32), ("copy_dtype", C.c_int32), ("seed", C.c_uint32),
                ("step", C.c_uint64), ("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("grad_scale", C.c_float), ("reserved", C.c_int32), ("grad_scale_dev", C.c_void_p)]


# The first three, written in one go (setting ctypes fields one by one costs more than the launch), anew for every call: the library reads
# them while other threads may run.
_FORWARD_FIELDS, _BACKWARD_FIELDS, _LOSS_FIELDS = struct.Struct("<3Q6i13Q"), struct.Struct("<3Q4iIi15Q"), struct.Struct("<2Q2i3Qqfi5Q")
assert _FORWARD_FIELDS.size == C.sizeof(_LinearForwardArgs) and _BACKWARD_FIELDS.size == C.sizeof(_LinearBackwardArgs)
assert _LOSS_FIELDS.size == C.sizeof(_CrossEntropyArgs)

_lib = None


def load_library():
    """libgd.so with the prototypes of gd_train.h (see binding.load_library)."""
    global _lib
    if _lib is None:
        lib = B.load_library()
        lib.gd_linear_forward.argtypes = [C.c_void_p, C.c_void_p]         # (the bytes of the arguments, or byref of a structure)
        lib.gd_linear_backward.argtypes = [C.c_void_p, C.c_void_p]
        lib.gd_linear_workspace_bytes.argtypes = [C.c_uint64, C.c_uint64, C.c_uint64, C.c_int, C.POINTER(C.c_size_t)]
        lib.gd_linear_status.argtypes = [C.c_void_p, C.c_void_p]
        lib.gd_selftest_linear_wait.argtypes = [C.c_void_p, C.c_size_t, C.c_uint64, C.c_void_p]
        lib.gd_cross_entropy.argtypes = [C.c_void_p, C.c_void_p]
        lib.gd_adamw_step.argtypes = [C.POINTER(_AdamwArgs), C.c_void_p]
        for name in EXPORTS:
            getattr(lib, name).restype = C.c_int
        _lib = lib
    return _lib


def _dtype_of(dtype: torch.dtype) -> int:
    if dtype not in _DTYPES:
        raise ValueError(f"{dtype} is not supported: float32, bfloat16 or float16")
    return _DTYPES[dtype]


# The checks below run on every call and cost more than the launch if done naively: one comparison each for the common case (a
# contiguous tensor of the right type, shape and device), everything else in the functions that explain.

def _matrix(t: torch.Tensor, name: str, rows: int, cols: int, dtype, index: int) -> int:
    """Checks a [rows, cols] tensor whose rows are contiguous and returns its leading dimension."""
    if t.dtype is not dtype or t.shape != (rows, cols) or t.get_device() != index:
        raise ValueError(f"{name}: expected {dtype} [{rows}, {cols}] on cuda:{index}, got {t.dtype} {list(t.shape)} on {t.device}")
    if t.is_contiguous():
        return cols
    ld, step = t.stride()
    if (step != 1 and cols > 1) or (rows > 1 and ld < cols):
        raise ValueError(f"{name}: the elements of a row must be neighbours and rows must not overlap (strides {ld}, {step})")
    return ld if rows > 1 else cols


def _vector(t: torch.Tensor, name: str, n: int, dtypes, index: int) -> None:
    if t.dtype not in dtypes or t.shape != (n,) or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name}: expected {n} contiguous {' or '.join(map(str, dtypes))} on cuda:{index}, got {t.dtype} {list(t.shape)} on {t.device}")


def _scalar(t: Optional[torch.Tensor], name: str, index: int) -> int:
    if t is None:
        return 0
    if t.numel() != 1 or t.dtype is not torch.float32 or t.get_device() != index:
        raise ValueError(f"{name} is one float32 on cuda:{index}")
    return t.data_ptr()


def _cuda_index(device) -> int:
    device = torch.device(device)
    if device.type != "cuda":
        raise RuntimeError("a CUDA device is needed: the library has no CPU path")
    return torch.cuda.current_device() if device.index is None else device.index


# the current stream's handle without a Stream object around it, and the current device without initialising anything
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _issue(call, args, stream, index: int) -> int:
    """call(args, stream's handle) with the tensors' device current: the library launches on the current device, and the handle of a default
    stream does not say which device's it is."""
    if _current_device() != index:
        with torch.cuda.device(index):
            return call(args, _raw_stream(index) if stream is None else B._stream_handle(stream))
    return call(args, _raw_stream(index) if stream is None else B._stream_handle(stream))


def _stream_object(stream, index: int):
    return stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=index)


class LinearSession:
    """One linear layer's shape - n_in inputs, n_out outputs, up to max_rows rows at a time - and its workspace.

    dtype is that of x, w, residual and pre (bfloat16 or float16).  The workspace is part of the session: calls on different
    streams must be ordered with respect to each other, or use sessions of their own.  any_layout=True makes
    room for operands that are not contiguous or start at odd addresses.
    """

    def __init__(self, n_in: int, n_out: int, max_rows: int, dtype=torch.bfloat16, activation: str = "none", w_layout: str = "in_out",
                 device="cuda", any_layout: bool = False):
        if dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("LinearSession takes bfloat16 or float16")
        if activation not in _ACTIVATIONS or w_layout not in _LAYOUTS:
            raise ValueError(f"activation is one of {sorted(_ACTIVATIONS)}, w_layout one of {sorted(_LAYOUTS)}")
        self._index = index = _cuda_index(device)
        self.device = torch.device("cuda", index)
        self.n_in, self.n_out, self.max_rows, self.dtype, self.activation, self.w_layout = int(n_in), int(n_out), int(max_rows), dtype, activation, w_layout
        self.w_shape = (self.n_in, self.n_out) if w_layout == "in_out" else (self.n_out, self.n_in)
        self._lib = load_library()
        size = C.c_size_t(0)
        B._check(self._lib.gd_linear_workspace_bytes(self.max_rows, self.n_out, self.n_in, int(any_layout), C.byref(size)), "gd_linear_workspace_bytes")
        self._bind(torch.empty(size.value, dtype=torch.uint8, device=self.device))
        self.workspace[:256].zero_()

    def _bind(self, workspace: torch.Tensor) -> None:
        """The arguments that stay the same from call to call."""
        self.workspace = workspace
        self._space = (workspace.data_ptr(), workspace.numel())
        self._codes = (self.n_out, self.n_in, _DTYPES[self.dtype], _ACTIVATIONS[self.activation], _LAYOUTS[self.w_layout])

    def _rows(self, t: torch.Tensor) -> int:
        m = t.shape[0] if t.dim() == 2 else -1
        if not 0 <= m <= self.max_rows:
            raise ValueError(f"at most {self.max_rows} rows of a matrix, got {list(t.shape)}")
        return m

    def forward(self, x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """act(x W + bias) + residual, into `out` (float32, or the session's type; made here, on the call's stream, if None) and, if `pre`
        is given, x W + bias."""
        m, n, dt, index = self._rows(x), self.n_out, self.dtype, self._index
        if out is None:
            # on the stream of the call: memory that other streams gave back may still be in use there
            with contextlib.nullcontext() if stream is None else torch.cuda.stream(_stream_object(stream, index)):
                out = torch.empty(m, n, dtype=dt, device=self.device)
        out_dt = out.dtype if out.dtype is torch.float32 else dt
        bias_at = bias_code = residual_at = ld_residual = pre_at = ld_pre = 0
        if bias is not None:
            _vector(bias, "bias", n, (torch.float32, dt), index)
            bias_at, bias_code = bias.data_ptr(), _DTYPES[bias.dtype]
        if residual is not None:
            residual_at, ld_residual = residual.data_ptr(), _matrix(residual, "residual", m, n, dt, index)
        if pre is not None:
            pre_at, ld_pre = pre.data_ptr(), _matrix(pre, "pre", m, n, dt, index)
        args = _FORWARD_FIELDS.pack(m, *self._codes, bias_code, _DTYPES[out_dt], 0, x.data_ptr(), _matrix(x, "x", m, self.n_in, dt, index),
                                    w.data_ptr(), _matrix(w, "w", *self.w_shape, dt, index), bias_at, residual_at, ld_residual,
                                    out.data_ptr(), _matrix(out, "out", m, n, out_dt, index), pre_at, ld_pre, *self._space)
        code = _issue(self._lib.gd_linear_forward, args, stream, index)
        if code:
            raise B.GdError(code, "gd_linear_forward")
        return out

    def backward(self, dy: torch.Tensor, x: Optional[torch.Tensor], w: Optional[torch.Tensor], pre: Optional[torch.Tensor] = None,
                 dx: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None, db: Optional[torch.Tensor] = None, accumulate: bool = False,
                 stream=None) -> None:
        """The gradients whose buffers are given, for dy, the gradient of forward's result (that of residual is dy itself).

        dw has w's shape, in float32 or the session's type; db is float32.  accumulate adds to dw (float32) and db.
        """
        m, n, k, dt, index = self._rows(dy), self.n_out, self.n_in, self.dtype, self._index
        if self.activation != "none" and pre is None:
            raise ValueError("backward needs the pre-activation that forward wrote")
        pre_at = ld_pre = x_at = ldx = w_at = ldw = dx_at = ld_dx = dw_at = ld_dw = db_at = dw_code = 0
        if pre is not None:
            pre_at, ld_pre = pre.data_ptr(), _matrix(pre, "pre", m, n, dt, index)
        if dx is not None:
            if w is None:
                raise ValueError("dx needs w")
            w_at, ldw = w.data_ptr(), _matrix(w, "w", *self.w_shape, dt, index)
            dx_at, ld_dx = dx.data_ptr(), _matrix(dx, "dx", m, k, dt, index)
        if dw is not None:
            if x is None:
                raise ValueError("dw needs x")
            dw_dt = dw.dtype if dw.dtype is torch.float32 else dt
            x_at, ldx = x.data_ptr(), _matrix(x, "x", m, k, dt, index)
            dw_at, ld_dw, dw_code = dw.data_ptr(), _matrix(dw, "dw", *self.w_shape, dw_dt, index), _DTYPES[dw_dt]
        if db is not None:
            _vector(db, "db", n, (torch.float32,), index)
            db_at = db.data_ptr()
        args = _BACKWARD_FIELDS.pack(m, *self._codes, dw_code, GD_LINEAR_ACCUMULATE if accumulate else 0, 0, dy.data_ptr(),
                                     _matrix(dy, "dy", m, n, dt, index), pre_at, ld_pre, x_at, ldx, w_at, ldw, dx_at, ld_dx, dw_at, ld_dw, db_at,
                                     *self._space)
        code = _issue(self._lib.gd_linear_backward, args, stream, index)
        if code:
            raise B.GdError(code, "gd_linear_backward")

    def status(self, stream=None) -> int:
        """GD_OK, or GD_ERR_DEVICE_TIMEOUT if a device-side wait of any call so far gave up (waits for the stream)."""
        return _issue(self._lib.gd_linear_status, self.workspace.data_ptr(), stream, self._index)


def cross_entropy(logits: torch.Tensor, targets: torch.Tensor, loss: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                  grad: Optional[torch.Tensor] = None, grad_scale: float = 1.0, grad_scale_dev: Optional[torch.Tensor] = None,
                  ignore_index: int = -100, stream=None) -> None:
    """Softmax cross-entropy of every row of logits [rows, classes] against targets (int32 or int64), into the buffers given:
    loss and lse (float32, rows) and grad (like logits; may be logits itself), the gradient of sum(loss) * grad_scale *
    grad_scale_dev.  Rows whose target is ignore_index have loss and gradient 0."""
    if logits.dim() != 2:
        raise ValueError(f"logits: expected a matrix, got {list(logits.shape)}")
    index = logits.get_device()
    if index < 0:
        raise RuntimeError("a CUDA device is needed: the library has no CPU path")
    rows, classes = logits.shape
    dtype = logits.dtype
    ld = _matrix(logits, "logits", rows, classes, dtype, index)
    _vector(targets, "targets", rows, (torch.int64, torch.int32), index)
    if loss is not None:
        _vector(loss, "loss", rows, (torch.float32,), index)
    if lse is not None:
        _vector(lse, "lse", rows, (torch.float32,), index)
    args = _LOSS_FIELDS.pack(rows, classes, _dtype_of(dtype), 64 if targets.dtype is torch.int64 else 32, logits.data_ptr(), ld, targets.data_ptr(),
                             ignore_index, grad_scale, 0, _scalar(grad_scale_dev, "grad_scale_dev", index), 0 if loss is None else loss.data_ptr(),
                             0 if lse is None else lse.data_ptr(), 0 if grad is None else grad.data_ptr(),
                             0 if grad is None else _matrix(grad, "grad", rows, classes, dtype, index))
    code = _issue(load_library().gd_cross_entropy, args, stream, index)
    if code:
        raise B.GdError(code, "gd_cross_entropy")


class AdamWSession:
    """A list of tensors under one AdamW update, with their moments.

    params and grads are lists of contiguous tensors of one type each (float32, bfloat16 or float16; any starting address).  m and v are
    lists of float32 tensors, or - the 8-bit form - of float8_e4m3fn tensors (v holds the root of the second moment) with
    m_scale and v_scale, ceil(n / 128) float32 each; without them the session makes zero moments of state_bits.  copies: 16-bit (or
    float32) tensors that receive the updated parameters, or None.  weight_decay: one number or one per tensor.  Addresses are
    taken once and the memory behind them is kept: a tensor that is pointed at other memory later (`t.data = ...`) needs a new session.
    """

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], m: Optional[Sequence[torch.Tensor]] = None,
                 v: Optional[Sequence[torch.Tensor]] = None, m_scale: Optional[Sequence[torch.Tensor]] = None,
                 v_scale: Optional[Sequence[torch.Tensor]] = None, copies: Optional[Sequence[torch.Tensor]] = None,
                 weight_decay: Union[float, Sequence[float]] = 0.0, state_bits: int = 32):
        self.params = list(params)
        if not self.params:
            raise ValueError("AdamWSession needs at least one tensor")
        if (m is None) != (v is None) or (m_scale is None) != (v_scale is None) or (m is None and m_scale is not None):
            raise ValueError("give both moments, and the scales of both or of neither")
        self._index = _cuda_index(self.params[0].device)
        dev = self.params[0].device
        sizes = [p.numel() for p in self.params]
        if m is not None:
            state_bits = 32 if m_scale is None else 8
        if state_bits not in (8, 32):
            raise ValueError("state_bits is 8 or 32")
        held = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        if m is None:
            m, v = ([torch.zeros(n, dtype=torch.float32 if state_bits == 32 else torch.uint8, device=dev).view(held) for n in sizes] for _ in range(2))
            if state_bits == 8:
                m_scale, v_scale = ([torch.ones(-(-n // _SCALE_BLOCK), dtype=torch.float32, device=dev) for n in sizes] for _ in range(2))
        self.m, self.v, self.state_bits = list(m), list(v), state_bits
        self.m_scale, self.v_scale = (None, None) if state_bits == 32 else (list(m_scale), list(v_scale))
        self.copies = None if copies is None else list(copies)
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [float(weight_decay)] * len(sizes)
        lists = [self.m, self.v, decay] + [t for t in (self.m_scale, self.v_scale, self.copies) if t is not None]
        if any(len(t) != len(sizes) for t in lists):
            raise ValueError("one entry per tensor is needed in every list")
        self._device = dev
        self._tensors = (_AdamwTensor * len(sizes))()
        a = self._args = _AdamwArgs()
        a.tensors, a.n_tensors, a.state_bits = self._tensors, len(sizes), state_bits
        a.param_dtype = _dtype_of(self.params[0].dtype)
        a.copy_dtype = GD_DTYPE_FP32 if self.copies is None else _dtype_of(self.copies[0].dtype)
        self._held = []
        for i, n in enumerate(sizes):
            t = self._tensors[i]
            t.n, t.weight_decay = n, float(decay[i])
            t.param = self._take(self.params[i], "params", n, self.params[0].dtype)
            t.m, t.v = (self._take(s[i], name, n, held) for s, name in ((self.m, "m"), (self.v, "v")))
            if state_bits == 8:
                t.m_scale, t.v_scale = (self._take(s[i], name, -(-n // _SCALE_BLOCK), torch.float32)
                                        for s, name in ((self.m_scale, "m_scale"), (self.v_scale, "v_scale")))
            if self.copies is not None:
                t.copy = self._take(self.copies[i], "copies", n, self.copies[0].dtype)
        self.set_grads(grads)

    def _flat(self, t: torch.Tensor, name: str, n: int, dtype) -> torch.Tensor:
        """The checked tensor's memory under a name of its own, which lives whatever becomes of the tensor."""
        if t.numel() != n or t.dtype != dtype or t.device != self._device or not t.is_contiguous():
            raise ValueError(f"{name}: expected {n} contiguous {dtype} on {self._device}, got {t.dtype} {list(t.shape)} on {t.device}")
        return t.detach()

    def _take(self, *what) -> int:
        self._held.append(self._flat(*what))
        return self._held[-1].data_ptr()

    def set_grads(self, grads: Sequence[torch.Tensor]) -> None:
        """The gradients the next steps read (the same buffers are read every step until other ones are set)."""
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError("one gradient per tensor is needed")
        grad_dtype = _dtype_of(grads[0].dtype)
        held = [self._flat(g, "grads", t.n, grads[0].dtype) for g, t in zip(grads, self._tensors)]
        self._args.grad_dtype = grad_dtype            # (all of them or, where one is refused, none: their type is one for all)
        for t, g in zip(self._tensors, held):
            t.grad = g.data_ptr()
        self.grads, self._held_grads = grads, held

    def step(self, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, grad_scale: float = 1.0,
             grad_scale_dev: Optional[torch.Tensor] = None, seed: int = 0, stream=None) -> None:
        """Update number `step` (from 1).  seed: another one every step for the 8-bit moments' rounding; not used with 32 bits."""
        if step < 0:                         # (would reach the library as a step near 2^64; 0 is refused there)
            raise ValueError(f"steps count from 1, got {step}")
        a = self._args
        a.step, a.lr, a.beta1, a.beta2, a.eps = step, lr, beta1, beta2, eps
        a.grad_scale, a.seed = grad_scale, seed & 0xFFFFFFFF
        a.grad_scale_dev = _scalar(grad_scale_dev, "grad_scale_dev", self._index)
        code = _issue(load_library().gd_adamw_step, C.byref(a), stream, self._index)
        if code:
            raise B.GdError(code, "gd_adamw_step")
