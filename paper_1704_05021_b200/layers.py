"""The layers of a language model around the linear layer and the loss: ctypes binding of include/gd_layers.h and the objects that hold what its
calls need between them.

`EmbeddingSession` (a table's shape, and the workspace of its gradient), `LayerNormSession`, `recurrence_forward` and `recurrence_backward`, and
`GatedLinearSession` check the tensors they are given, marshal addresses and issue the calls, as training.py does: all
arithmetic happens inside libgd.so.  Tensors must live on the device of the call and be ready on its stream: the current stream, or the
one passed as `stream`.  A session's workspace is part of it: calls on different streams must be ordered with respect to each other, or use
sessions of their own; a captured graph uses the workspace of the session that was called.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import struct
from typing import Optional

import torch

from . import binding as B
from . import training as T
from .training import _ACTIVATIONS, _DTYPES, _LAYOUTS, _cuda_index, _dtype_of, _issue, _matrix, _stream_object, _vector

GD_EMBEDDING_ACCUMULATE = 1
GD_LAYER_NORM_ACCUMULATE = 1

EXPORTS = ["gd_embedding_forward", "gd_embedding_backward", "gd_embedding_workspace_bytes", "gd_layer_norm_forward", "gd_layer_norm_backward",
           "gd_layer_norm_workspace_bytes", "gd_recurrence_forward", "gd_recurrence_backward", "gd_recurrence_marks_rows",
           "gd_selftest_recurrence_wait", "gd_gated_forward", "gd_gated_backward", "gd_gated_workspace_bytes", "gd_selftest_gated_wait"]


class _EmbeddingForwardArgs(C.Structure):
    _fields_ = [("tokens", C.c_uint64), ("vocab", C.c_uint64), ("width", C.c_uint64), ("table_dtype", C.c_int32), ("y_dtype", C.c_int32),
                ("id_bits", C.c_int32), ("scale", C.c_float), ("ignore_index", C.c_int64), ("table", C.c_void_p), ("ld_table", C.c_uint64),
                ("ids", C.c_void_p), ("y", C.c_void_p), ("ld_y", C.c_uint64)]


class _EmbeddingBackwardArgs(C.Structure):
    _fields_ = [("tokens", C.c_uint64), ("vocab", C.c_uint64), ("width", C.c_uint64), ("dtype", C.c_int32), ("dtable_dtype", C.c_int32),
                ("id_bits", C.c_int32), ("scale", C.c_float), ("ignore_index", C.c_int64), ("flags", C.c_uint32), ("reserved", C.c_int32),
                ("dy", C.c_void_p), ("ld_dy", C.c_uint64), ("ids", C.c_void_p), ("dtable", C.c_void_p), ("ld_dtable", C.c_uint64),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class _LayerNormForwardArgs(C.Structure):
    _fields_ = [("rows", C.c_uint64), ("width", C.c_uint64), ("dtype", C.c_int32), ("param_dtype", C.c_int32), ("eps", C.c_float), ("reserved", C.c_int32),
                ("x", C.c_void_p), ("ldx", C.c_uint64), ("weight", C.c_void_p), ("bias", C.c_void_p), ("y", C.c_void_p), ("ldy", C.c_uint64),
                ("mean", C.c_void_p), ("rstd", C.c_void_p)]


class _LayerNormBackwardArgs(C.Structure):
    _fields_ = [("rows", C.c_uint64), ("width", C.c_uint64), ("dtype", C.c_int32), ("param_dtype", C.c_int32), ("flags", C.c_uint32), ("reserved", C.c_int32),
                ("dy", C.c_void_p), ("ld_dy", C.c_uint64), ("x", C.c_void_p), ("ldx", C.c_uint64), ("weight", C.c_void_p), ("mean", C.c_void_p),
                ("rstd", C.c_void_p), ("add", C.c_void_p), ("ld_add", C.c_uint64), ("dx", C.c_void_p), ("ld_dx", C.c_uint64),
                ("dweight", C.c_void_p), ("dbias", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class _RecurrenceForwardArgs(C.Structure):
    _fields_ = [("rows", C.c_uint64), ("sequences", C.c_uint64), ("width", C.c_uint64), ("dtype", C.c_int32), ("offset_bits", C.c_int32),
                ("offsets", C.c_void_p), ("gate", C.c_void_p), ("ld_gate", C.c_uint64), ("value", C.c_void_p), ("ld_value", C.c_uint64),
                ("y", C.c_void_p), ("ld_y", C.c_uint64), ("h0", C.c_void_p), ("h_last", C.c_void_p), ("marks", C.c_void_p)]


class _RecurrenceBackwardArgs(C.Structure):
    _fields_ = [("rows", C.c_uint64), ("sequences", C.c_uint64), ("width", C.c_uint64), ("dtype", C.c_int32), ("offset_bits", C.c_int32),
                ("offsets", C.c_void_p), ("dy", C.c_void_p), ("ld_dy", C.c_uint64), ("gate", C.c_void_p), ("ld_gate", C.c_uint64),
                ("value", C.c_void_p), ("ld_value", C.c_uint64), ("marks", C.c_void_p), ("dgate", C.c_void_p), ("ld_dgate", C.c_uint64),
                ("dvalue", C.c_void_p), ("ld_dvalue", C.c_uint64), ("dh_last", C.c_void_p), ("dh0", C.c_void_p)]


class _GatedForwardArgs(C.Structure):
    _fields_ = [("m", C.c_uint64), ("n", C.c_uint64), ("k", C.c_uint64), ("dtype", C.c_int32), ("activation", C.c_int32), ("w_layout", C.c_int32),
                ("bias_dtype", C.c_int32), ("x", C.c_void_p), ("ldx", C.c_uint64), ("w", C.c_void_p), ("ldw", C.c_uint64), ("bias", C.c_void_p),
                ("y", C.c_void_p), ("ldy", C.c_uint64), ("pre", C.c_void_p), ("ld_pre", C.c_uint64), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t)]


class _GatedBackwardArgs(C.Structure):
    _fields_ = [("m", C.c_uint64), ("n", C.c_uint64), ("k", C.c_uint64), ("dtype", C.c_int32), ("activation", C.c_int32), ("w_layout", C.c_int32),
                ("dw_dtype", C.c_int32), ("flags", C.c_uint32), ("reserved", C.c_int32), ("dy", C.c_void_p), ("ld_dy", C.c_uint64),
                ("pre", C.c_void_p), ("ld_pre", C.c_uint64), ("x", C.c_void_p), ("ldx", C.c_uint64), ("w", C.c_void_p), ("ldw", C.c_uint64),
                ("dx", C.c_void_p), ("ld_dx", C.c_uint64), ("dw", C.c_void_p), ("ld_dw", C.c_uint64), ("db", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


# written in one go for every call, as in training.py
_FIELDS = {_EmbeddingForwardArgs: struct.Struct("<3Q3ifq5Q"), _EmbeddingBackwardArgs: struct.Struct("<3Q3ifqIi7Q"),
           _LayerNormForwardArgs: struct.Struct("<2Q2ifi8Q"), _LayerNormBackwardArgs: struct.Struct("<2Q2iIi15Q"),
           _RecurrenceForwardArgs: struct.Struct("<3Q2i10Q"), _RecurrenceBackwardArgs: struct.Struct("<3Q2i14Q"),
           _GatedForwardArgs: struct.Struct("<3Q4i11Q"), _GatedBackwardArgs: struct.Struct("<3Q4iIi15Q")}
assert all(fields.size == C.sizeof(args) for args, fields in _FIELDS.items())
_EMBED, _EMBED_BACK, _NORM, _NORM_BACK, _SCAN, _SCAN_BACK, _GATED, _GATED_BACK = _FIELDS.values()

_lib = None


def load_library():
    """libgd.so with the prototypes of gd_layers.h (see binding.load_library)."""
    global _lib
    if _lib is None:
        lib = T.load_library()
        for name in EXPORTS:
            function = getattr(lib, name)
            function.argtypes, function.restype = [C.c_void_p, C.c_void_p], C.c_int      # (the bytes of the arguments, or byref of a structure)
        lib.gd_embedding_workspace_bytes.argtypes = [C.c_uint64, C.c_uint64, C.c_uint64, C.POINTER(C.c_size_t)]
        lib.gd_layer_norm_workspace_bytes.argtypes = [C.c_uint64, C.c_uint64, C.POINTER(C.c_size_t)]
        lib.gd_gated_workspace_bytes.argtypes = [C.c_uint64, C.c_uint64, C.c_uint64, C.c_int, C.POINTER(C.c_size_t)]
        lib.gd_selftest_gated_wait.argtypes = [C.c_void_p, C.c_size_t, C.c_uint64, C.c_void_p]
        lib.gd_selftest_recurrence_wait.argtypes = [C.c_void_p, C.c_size_t, C.c_int, C.c_uint64, C.c_void_p]
        lib.gd_recurrence_marks_rows.argtypes = [C.c_uint64, C.c_uint64, C.POINTER(C.c_uint64)]
        _lib = lib
    return _lib


def _call(function, name: str, args: bytes, stream, index: int) -> None:
    code = _issue(function, args, stream, index)
    if code:
        raise B.GdError(code, name)


def _new(rows: int, cols: int, dtype, stream, index: int) -> torch.Tensor:
    """A result made by a call, from the call's stream: memory that other streams gave back may still be in use there."""
    with contextlib.nullcontext() if stream is None else torch.cuda.stream(_stream_object(stream, index)):
        return torch.empty(rows, cols, dtype=dtype, device=torch.device("cuda", index))


def _opt_matrix(t: Optional[torch.Tensor], name: str, rows: int, cols: int, dtype, index: int):
    return (0, 0) if t is None else (t.data_ptr(), _matrix(t, name, rows, cols, dtype, index))


def _opt_vector(t: Optional[torch.Tensor], name: str, n: int, dtypes, index: int) -> int:
    if t is None:
        return 0
    _vector(t, name, n, dtypes, index)
    return t.data_ptr()


def _opt_state(t: Optional[torch.Tensor], name: str, rows: int, cols: int, index: int) -> int:
    if t is None:
        return 0
    if t.dtype is not torch.float32 or t.shape != (rows, cols) or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous torch.float32 [{rows}, {cols}] on cuda:{index}, got {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


_F32 = (torch.float32,)
_MARK_ROWS = 64             # rows from one of the recurrence's marks to the next
_INTS = (torch.int64, torch.int32)


class EmbeddingSession:
    """The shape of an embedding table - vocab rows of width elements - and the workspace that its gradient for up to max_tokens positions takes
    (gradient=False: none, for a program that only looks up).  A lookup takes any number of them.

    ids are vectors of int32 or int64.  A position whose id is ignore_index is padding: its row is zeros and its gradient counts nowhere.  An
    id that is not in the table gives a row of NaN and has no part in the gradient.
    """

    def __init__(self, vocab: int, width: int, max_tokens: int, device="cuda", gradient: bool = True):
        self._index = index = _cuda_index(device)
        self.device = torch.device("cuda", index)
        self.vocab, self.width, self.max_tokens = int(vocab), int(width), int(max_tokens)
        self._lib = load_library()
        size = C.c_size_t(0)
        B._check(self._lib.gd_embedding_workspace_bytes(self.max_tokens, self.vocab, self.width, C.byref(size)), "gd_embedding_workspace_bytes")
        self.workspace = torch.empty(size.value, dtype=torch.uint8, device=self.device) if gradient else None

    def _ids(self, ids: torch.Tensor) -> int:
        n = ids.numel()
        _vector(ids, "ids", n, _INTS, self._index)
        return n

    def forward(self, table: torch.Tensor, ids: torch.Tensor, out: Optional[torch.Tensor] = None, scale: float = 1.0, ignore_index: int = -100,
                stream=None) -> torch.Tensor:
        """scale * table[ids], into `out` (the table's type, or float32; from a float32 table any; made here if None)."""
        n, index, width = self._ids(ids), self._index, self.width
        ld = _matrix(table, "table", self.vocab, width, table.dtype, index)
        if out is None:
            out = _new(n, width, table.dtype, stream, index)
        args = _EMBED.pack(n, self.vocab, width, _dtype_of(table.dtype), _dtype_of(out.dtype), 64 if ids.dtype is torch.int64 else 32, scale, ignore_index,
                           table.data_ptr(), ld, ids.data_ptr(), out.data_ptr(), _matrix(out, "out", n, width, out.dtype, index))
        _call(self._lib.gd_embedding_forward, "gd_embedding_forward", args, stream, index)
        return out

    def backward(self, dy: torch.Tensor, ids: torch.Tensor, dtable: torch.Tensor, scale: float = 1.0, accumulate: bool = False, ignore_index: int = -100,
                 stream=None) -> None:
        """dtable (float32, or dy's type) receives scale times the sums of dy's rows of equal ids, zeros elsewhere; accumulate adds them to what a
        float32 dtable holds and leaves the other rows as they are."""
        n, index, width = self._ids(ids), self._index, self.width
        if self.workspace is None:
            raise ValueError("a session made with gradient=False has no workspace for backward")
        if n > self.max_tokens:
            raise ValueError(f"the workspace is for at most {self.max_tokens} positions, got {n}")
        args = _EMBED_BACK.pack(n, self.vocab, width, _dtype_of(dy.dtype), _dtype_of(dtable.dtype), 64 if ids.dtype is torch.int64 else 32, scale, ignore_index,
                                GD_EMBEDDING_ACCUMULATE if accumulate else 0, 0, dy.data_ptr(), _matrix(dy, "dy", n, width, dy.dtype, index),
                                ids.data_ptr(), dtable.data_ptr(), _matrix(dtable, "dtable", self.vocab, width, dtable.dtype, index),
                                self.workspace.data_ptr(), self.workspace.numel())
        _call(self._lib.gd_embedding_backward, "gd_embedding_backward", args, stream, index)


class LayerNormSession:
    """Layer norm over rows of `width` elements of one type (float32, bfloat16 or float16), up to max_rows at a time, and the workspace for the sums
    of its parameters' gradients.  weight and bias are float32 or of the rows' type, both the same."""

    def __init__(self, width: int, max_rows: int, dtype=torch.bfloat16, eps: float = 1e-5, device="cuda"):
        self._index = index = _cuda_index(device)
        self.device = torch.device("cuda", index)
        self._code = _dtype_of(dtype)
        if not eps >= 0:
            raise ValueError(f"eps is not negative, got {eps}")
        self.width, self.max_rows, self.dtype, self.eps = int(width), int(max_rows), dtype, float(eps)
        self._lib = load_library()
        size = C.c_size_t(0)
        B._check(self._lib.gd_layer_norm_workspace_bytes(self.max_rows, self.width, C.byref(size)), "gd_layer_norm_workspace_bytes")
        self.workspace = torch.empty(size.value, dtype=torch.uint8, device=self.device)

    def _rows(self, t: torch.Tensor) -> int:
        rows = t.shape[0] if t.dim() == 2 else -1
        if not 0 <= rows <= self.max_rows:
            raise ValueError(f"at most {self.max_rows} rows of a matrix, got {list(t.shape)}")
        return rows

    def _param(self, p: Optional[torch.Tensor], name: str, other: Optional[torch.Tensor]) -> int:
        """The address of a parameter, float32 or of the rows' type and of the other one's."""
        if p is None:
            return 0
        if p.dtype is not torch.float32 and p.dtype is not self.dtype or other is not None and other.dtype is not p.dtype:
            raise ValueError(f"weight and bias are both float32 or both {self.dtype}, got {p.dtype}" + ("" if other is None else f" and {other.dtype}"))
        _vector(p, name, self.width, (p.dtype,), self._index)
        return p.data_ptr()

    def forward(self, x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """(x - mean) * rstd * weight + bias into `out` (may be x; made here if None), and each row's mean and rstd (float32) if given."""
        rows, width, dt, index = self._rows(x), self.width, self.dtype, self._index
        ldx = _matrix(x, "x", rows, width, dt, index)
        if out is None:
            out = _new(rows, width, dt, stream, index)
        given = bias if weight is None else weight
        args = _NORM.pack(rows, width, self._code, 0 if given is None else _DTYPES.get(given.dtype, -1), self.eps, 0, x.data_ptr(), ldx,
                          self._param(weight, "weight", bias), self._param(bias, "bias", weight), out.data_ptr(),
                          _matrix(out, "out", rows, width, dt, index), _opt_vector(mean, "mean", rows, _F32, index), _opt_vector(rstd, "rstd", rows, _F32, index))
        _call(self._lib.gd_layer_norm_forward, "gd_layer_norm_forward", args, stream, index)
        return out

    def backward(self, dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor,
                 dx: Optional[torch.Tensor] = None, add: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None,
                 dbias: Optional[torch.Tensor] = None, accumulate: bool = False, stream=None) -> None:
        """The gradients whose buffers are given.  add is the gradient that reaches x past the norm and is added to dx; dx may be dy or add itself.
        dweight and dbias are float32; accumulate adds to what they hold."""
        rows, width, dt, index = self._rows(dy), self.width, self.dtype, self._index
        sums = [_opt_vector(t, name, width, _F32, index) for t, name in ((dweight, "dweight"), (dbias, "dbias"))]
        _vector(mean, "mean", rows, _F32, index)
        _vector(rstd, "rstd", rows, _F32, index)
        args = _NORM_BACK.pack(rows, width, self._code, 0 if weight is None else _DTYPES.get(weight.dtype, -1), GD_LAYER_NORM_ACCUMULATE if accumulate else 0, 0, dy.data_ptr(),
                               _matrix(dy, "dy", rows, width, dt, index), x.data_ptr(), _matrix(x, "x", rows, width, dt, index), self._param(weight, "weight", None), mean.data_ptr(),
                               rstd.data_ptr(), *_opt_matrix(add, "add", rows, width, dt, index), *_opt_matrix(dx, "dx", rows, width, dt, index), *sums,
                               self.workspace.data_ptr(), self.workspace.numel())
        _call(self._lib.gd_layer_norm_backward, "gd_layer_norm_backward", args, stream, index)


def _spans(rows: int, offsets: Optional[torch.Tensor], sequences: int, index: int):
    """offset_bits and the address of offsets."""
    if offsets is None:
        if sequences < 1 or rows % sequences:
            raise ValueError(f"without offsets {rows} rows are equal parts for {sequences} sequences")
        return 64, 0
    _vector(offsets, "offsets", sequences + 1, _INTS, index)
    return 64 if offsets.dtype is torch.int64 else 32, offsets.data_ptr()


def _matrix_index(t: torch.Tensor, name: str) -> int:
    if t.dim() != 2:
        raise ValueError(f"{name}: expected a matrix, got {list(t.shape)}")
    if t.get_device() < 0:
        raise RuntimeError("a CUDA device is needed: the library has no CPU path")
    return t.get_device()


def recurrence_marks(rows: int, sequences: int, width: int, device="cuda") -> torch.Tensor:
    """Room for the states that recurrence_forward keeps for recurrence_backward, for up to this many rows and sequences."""
    count = C.c_uint64(0)
    B._check(load_library().gd_recurrence_marks_rows(rows, sequences, C.byref(count)), "gd_recurrence_marks_rows")
    return torch.empty(count.value, width, dtype=torch.float32, device=torch.device("cuda", _cuda_index(device)))


def _marks(marks: Optional[torch.Tensor], rows: int, sequences: int, width: int, index: int) -> int:
    if marks is None:
        return 0
    count = rows // _MARK_ROWS + sequences             # (what gd_recurrence_marks_rows says, without the call)
    if marks.dtype is not torch.float32 or marks.dim() != 2 or marks.shape[1] != width or marks.shape[0] < count or marks.get_device() != index or \
            not marks.is_contiguous():
        raise ValueError(f"marks: expected contiguous torch.float32 [{count}, {width}] on cuda:{index}, got {marks.dtype} {list(marks.shape)} on {marks.device}")
    return marks.data_ptr()


def recurrence_forward(gate: torch.Tensor, value: torch.Tensor, out: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
                       sequences: int = 1, h0: Optional[torch.Tensor] = None, h_last: Optional[torch.Tensor] = None,
                       marks: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """h[t] = f h[t-1] + (1 - f) value[t] with f = sigmoid(gate[t]), per column, over sequences that lie one behind the other in the rows.

    offsets (int32 or int64, sequences + 1, ascending): where each begins and the last one ends; None: equal parts.  h0 and h_last: [sequences, width]
    float32, the states before and after; they may be one tensor, as in a model that answers token by token (one row per sequence).
    `out` (of value's type; made here if None) receives the states; rows that belong to no sequence are left as they are.  marks (from
    recurrence_marks) are what recurrence_backward takes.
    """
    index = _matrix_index(value, "value")
    rows, width = value.shape
    dt = value.dtype
    code = _dtype_of(dt)
    bits, offsets_at = _spans(rows, offsets, sequences, index)
    gate_ld, value_ld = _matrix(gate, "gate", rows, width, dt, index), _matrix(value, "value", rows, width, dt, index)
    if out is None:
        out = _new(rows, width, dt, stream, index)
    args = _SCAN.pack(rows, sequences, width, code, bits, offsets_at, gate.data_ptr(), gate_ld, value.data_ptr(), value_ld, out.data_ptr(),
                      _matrix(out, "out", rows, width, dt, index), _opt_state(h0, "h0", sequences, width, index),
                      _opt_state(h_last, "h_last", sequences, width, index), _marks(marks, rows, sequences, width, index))
    _call(load_library().gd_recurrence_forward, "gd_recurrence_forward", args, stream, index)
    return out


def recurrence_backward(dy: torch.Tensor, gate: torch.Tensor, value: torch.Tensor, marks: torch.Tensor, dgate: torch.Tensor, dvalue: torch.Tensor,
                        offsets: Optional[torch.Tensor] = None, sequences: int = 1, dh_last: Optional[torch.Tensor] = None,
                        dh0: Optional[torch.Tensor] = None, stream=None) -> None:
    """Gradients of recurrence_forward for dy and dh_last (the gradients of its result and of h_last), with the marks, offsets and sequences of that
    call.  dgate may be gate or dy itself, dvalue value."""
    index = _matrix_index(value, "value")
    rows, width = value.shape
    dt = value.dtype
    code = _dtype_of(dt)
    bits, offsets_at = _spans(rows, offsets, sequences, index)
    matrices = []
    for t, name in ((dy, "dy"), (gate, "gate"), (value, "value"), (dgate, "dgate"), (dvalue, "dvalue")):
        matrices += (t.data_ptr(), _matrix(t, name, rows, width, dt, index))
    args = _SCAN_BACK.pack(rows, sequences, width, code, bits, offsets_at, *matrices[:6], _marks(marks, rows, sequences, width, index), *matrices[6:],
                           _opt_state(dh_last, "dh_last", sequences, width, index), _opt_state(dh0, "dh0", sequences, width, index))
    _call(load_library().gd_recurrence_backward, "gd_recurrence_backward", args, stream, index)


class GatedLinearSession:
    """The gated feed-forward block's two projections - n_in inputs, n_out outputs each, up to max_rows rows at a time - and its workspace.

    W is one matrix, [n_in, 2 n_out] or [2 n_out, n_in] (w_layout): the first n_out outputs are the gate, the others are multiplied by it.  dtype is
    that of x, w, the result and pre (bfloat16 or float16).  any_layout=True makes room for operands that are not contiguous or start at odd
    addresses.  The block's last projection is a LinearSession.
    """

    def __init__(self, n_in: int, n_out: int, max_rows: int, dtype=torch.bfloat16, activation: str = "silu", w_layout: str = "in_out", device="cuda",
                 any_layout: bool = False):
        if dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("GatedLinearSession takes bfloat16 or float16")
        if activation not in _ACTIVATIONS or w_layout not in _LAYOUTS:
            raise ValueError(f"activation is one of {sorted(_ACTIVATIONS)}, w_layout one of {sorted(_LAYOUTS)}")
        self._index = index = _cuda_index(device)
        self.device = torch.device("cuda", index)
        self.n_in, self.n_out, self.max_rows, self.dtype, self.activation, self.w_layout = int(n_in), int(n_out), int(max_rows), dtype, activation, w_layout
        self.w_shape = (self.n_in, 2 * self.n_out) if w_layout == "in_out" else (2 * self.n_out, self.n_in)
        self._lib = load_library()
        size = C.c_size_t(0)
        B._check(self._lib.gd_gated_workspace_bytes(self.max_rows, self.n_out, self.n_in, int(any_layout), C.byref(size)), "gd_gated_workspace_bytes")
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

    def forward(self, x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                pre: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """act(z[:, :n_out]) * z[:, n_out:] with z = x W + bias (float32 or the session's type), into `out` (made here if None) and, if `pre`
        ([rows, 2 n_out]) is given, z."""
        m, n, dt, index = self._rows(x), self.n_out, self.dtype, self._index
        if out is None:
            out = _new(m, n, dt, stream, index)
        bias_at = _opt_vector(bias, "bias", 2 * n, (torch.float32, dt), index)
        args = _GATED.pack(m, *self._codes, 0 if bias is None else _DTYPES[bias.dtype], x.data_ptr(), _matrix(x, "x", m, self.n_in, dt, index), w.data_ptr(),
                           _matrix(w, "w", *self.w_shape, dt, index), bias_at, out.data_ptr(), _matrix(out, "out", m, n, dt, index),
                           *_opt_matrix(pre, "pre", m, 2 * n, dt, index), *self._space)
        _call(self._lib.gd_gated_forward, "gd_gated_forward", args, stream, index)
        return out

    def backward(self, dy: torch.Tensor, x: Optional[torch.Tensor], w: Optional[torch.Tensor], pre: torch.Tensor, dx: Optional[torch.Tensor] = None,
                 dw: Optional[torch.Tensor] = None, db: Optional[torch.Tensor] = None, accumulate: bool = False, stream=None) -> None:
        """The gradients whose buffers are given, for dy, the gradient of forward's result, and the pre that it wrote.

        dw has w's shape, in float32 or the session's type; db is float32, 2 n_out.  accumulate adds to dw (float32) and db.
        """
        m, n, k, dt, index = self._rows(dy), self.n_out, self.n_in, self.dtype, self._index
        if dx is not None and w is None:
            raise ValueError("dx needs w")
        if dw is not None and x is None:
            raise ValueError("dw needs x")
        dw_dt = dt if dw is None or dw.dtype is not torch.float32 else torch.float32
        args = _GATED_BACK.pack(m, *self._codes, _DTYPES[dw_dt], T.GD_LINEAR_ACCUMULATE if accumulate else 0, 0, dy.data_ptr(),
                                _matrix(dy, "dy", m, n, dt, index), pre.data_ptr(), _matrix(pre, "pre", m, 2 * n, dt, index),
                                *_opt_matrix(x if dw is not None else None, "x", m, k, dt, index),
                                *_opt_matrix(w if dx is not None else None, "w", *self.w_shape, dt, index), *_opt_matrix(dx, "dx", m, k, dt, index),
                                *_opt_matrix(dw, "dw", *self.w_shape, dw_dt, index), _opt_vector(db, "db", 2 * n, _F32, index), *self._space)
        _call(self._lib.gd_gated_backward, "gd_gated_backward", args, stream, index)

    def status(self, stream=None) -> int:
        """GD_OK, or GD_ERR_DEVICE_TIMEOUT if a device-side wait of any call so far gave up (waits for the stream)."""
        return _issue(self._lib.gd_linear_status, self.workspace.data_ptr(), stream, self._index)
