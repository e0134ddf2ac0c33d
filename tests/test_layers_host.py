"""Host-side checks of the layers of include/gd_layers.h that need no GPU: exports, structures, sizing, refusals before anything runs."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import build as gd_build
from paper_1704_05021_b200 import layers as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, LARGE, SPACE = B.GD_ERR_INVALID_ARG, B.GD_ERR_TOO_LARGE, B.GD_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    gd_build.build_library()
    return L.load_library()


def test_every_declared_symbol_is_exported(lib):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gd_layers.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(gd_[a-z_]+)\s*\(", header))
    assert declared == set(L.EXPORTS)
    for name in declared:
        assert getattr(lib, name) is not None


def test_header_is_plain_c_and_structures_agree(lib, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler here")
    structures = list(L._FIELDS)
    names = ["gd" + re.sub("([A-Z])", lambda m: "_" + m.group(1).lower(), s.__name__[1:]) for s in structures]
    src = tmp_path / "use_gd_layers.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"gd_layers.h\"\nint main(void) {\n" +
                   "".join(f'  printf("%zu\\n", sizeof({n}));\n' for n in names) +
                   "".join(f'  printf("%zu\\n", offsetof({n}, {f[0]}));\n' for n, s in zip(names, structures) for f in s._fields_) +
                   "  return gd_layer_norm_forward(NULL, NULL) == GD_ERR_INVALID_ARG ? 0 : 1;\n}\n")
    exe, libdir = tmp_path / "use_gd_layers", os.path.dirname(gd_build.LIB_PATH)
    res = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-L", libdir,
                          "-l:libgd.so", "-Wl,-rpath," + libdir, "-o", str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, (out.returncode, out.stderr)
    ours = [C.sizeof(s) for s in structures] + [getattr(s, f[0]).offset for s in structures for f in s._fields_]
    assert [int(x) for x in out.stdout.split()] == ours


def _embedding():
    a = L._EmbeddingForwardArgs()
    a.tokens, a.vocab, a.width, a.table_dtype, a.y_dtype, a.id_bits, a.scale = 4, 10, 8, 1, 1, 64, 1.0
    a.table, a.ld_table, a.ids, a.y, a.ld_y = 0x1000, 8, 0x2000, 0x3000, 8
    return a


def _embedding_back():
    a = L._EmbeddingBackwardArgs()
    a.tokens, a.vocab, a.width, a.dtype, a.dtable_dtype, a.id_bits, a.scale = 4, 10, 8, 1, 0, 64, 1.0
    a.dy, a.ld_dy, a.ids, a.dtable, a.ld_dtable, a.workspace, a.workspace_bytes = 0x1000, 8, 0x2000, 0x3000, 8, 0x4000, 1 << 20
    return a


def _norm():
    a = L._LayerNormForwardArgs()
    a.rows, a.width, a.dtype, a.eps = 4, 8, 1, 1e-5
    a.x, a.ldx, a.weight, a.bias, a.y, a.ldy, a.mean, a.rstd = 0x1000, 8, 0x2000, 0x3000, 0x4000, 8, 0x5000, 0x6000
    return a


def _norm_back():
    a = L._LayerNormBackwardArgs()
    a.rows, a.width, a.dtype = 4, 8, 1
    a.dy, a.ld_dy, a.x, a.ldx, a.weight, a.mean, a.rstd, a.add, a.ld_add = 0x1000, 8, 0x2000, 8, 0x3000, 0x4000, 0x5000, 0x6000, 8
    a.dx, a.ld_dx, a.dweight, a.dbias, a.workspace, a.workspace_bytes = 0x7000, 8, 0x8000, 0x9000, 0xa000, 1 << 20
    return a


def _scan():
    a = L._RecurrenceForwardArgs()
    a.rows, a.sequences, a.width, a.dtype, a.offset_bits, a.offsets = 6, 2, 8, 1, 64, 0x1000
    a.gate, a.ld_gate, a.value, a.ld_value, a.y, a.ld_y, a.h0, a.h_last, a.marks = 0x2000, 8, 0x3000, 8, 0x4000, 8, 0x5000, 0x6000, 0x7000
    return a


def _scan_back():
    a = L._RecurrenceBackwardArgs()
    a.rows, a.sequences, a.width, a.dtype, a.offset_bits, a.offsets = 6, 2, 8, 1, 64, 0x1000
    a.dy, a.ld_dy, a.gate, a.ld_gate, a.value, a.ld_value, a.marks = 0x2000, 8, 0x3000, 8, 0x4000, 8, 0x5000
    a.dgate, a.ld_dgate, a.dvalue, a.ld_dvalue, a.dh_last, a.dh0 = 0x6000, 8, 0x7000, 8, 0x8000, 0x9000
    return a


def _gated():
    a = L._GatedForwardArgs()
    a.m, a.n, a.k, a.dtype, a.activation = 4, 8, 16, 1, 3
    a.x, a.ldx, a.w, a.ldw, a.bias, a.y, a.ldy, a.pre, a.ld_pre, a.workspace, a.workspace_bytes = 0x1000, 16, 0x2000, 16, 0x3000, 0x4000, 8, 0x5000, 16, 0x6000, 256
    return a


def _gated_back():
    a = L._GatedBackwardArgs()
    a.m, a.n, a.k, a.dtype, a.activation = 4, 8, 16, 1, 3
    a.dy, a.ld_dy, a.pre, a.ld_pre, a.x, a.ldx, a.w, a.ldw = 0x1000, 8, 0x2000, 16, 0x3000, 16, 0x4000, 16
    a.dx, a.ld_dx, a.dw, a.ld_dw, a.db, a.workspace, a.workspace_bytes = 0x5000, 16, 0x6000, 16, 0x7000, 0x8000, 512
    return a


@pytest.mark.parametrize("call, make, changes, code", [
    ("gd_gated_forward", _gated, dict(dtype=0), INVALID), ("gd_gated_forward", _gated, dict(activation=4), INVALID),
    ("gd_gated_forward", _gated, dict(w_layout=2), INVALID), ("gd_gated_forward", _gated, dict(bias_dtype=2), INVALID),
    ("gd_gated_forward", _gated, dict(x=None), INVALID), ("gd_gated_forward", _gated, dict(w=0x2001), INVALID), ("gd_gated_forward", _gated, dict(ldw=15), INVALID),
    ("gd_gated_forward", _gated, dict(y=None), INVALID), ("gd_gated_forward", _gated, dict(ld_pre=15), INVALID), ("gd_gated_forward", _gated, dict(m=1 << 30), LARGE),
    ("gd_gated_forward", _gated, dict(workspace=None), SPACE), ("gd_gated_forward", _gated, dict(workspace_bytes=255), SPACE),
    ("gd_gated_forward", _gated, dict(ldx=17), SPACE), ("gd_gated_forward", _gated, dict(ldw=17), SPACE), ("gd_gated_forward", _gated, dict(w=0x2002), SPACE),
    ("gd_gated_forward", _gated, dict(n=0), 0), ("gd_gated_backward", _gated_back, dict(dtype=0), INVALID),
    ("gd_gated_backward", _gated_back, dict(flags=2), INVALID), ("gd_gated_backward", _gated_back, dict(reserved=1), INVALID),
    ("gd_gated_backward", _gated_back, dict(dw_dtype=2), INVALID), ("gd_gated_backward", _gated_back, dict(flags=1, dw_dtype=1), INVALID),
    ("gd_gated_backward", _gated_back, dict(dy=None), INVALID), ("gd_gated_backward", _gated_back, dict(pre=None), INVALID),
    ("gd_gated_backward", _gated_back, dict(x=None), INVALID), ("gd_gated_backward", _gated_back, dict(w=None), INVALID),
    ("gd_gated_backward", _gated_back, dict(db=0x7002), INVALID), ("gd_gated_backward", _gated_back, dict(ld_dw=15), INVALID),
    ("gd_gated_backward", _gated_back, dict(workspace_bytes=511 - 128), SPACE), ("gd_gated_backward", _gated_back, dict(ldx=19), SPACE),
    ("gd_gated_backward", _gated_back, dict(k=1 << 30), LARGE), ("gd_gated_backward", _gated_back, dict(dx=None, dw=None, db=None), 0),
    ("gd_embedding_forward", _embedding, dict(table_dtype=3), INVALID), ("gd_embedding_forward", _embedding, dict(y_dtype=2), INVALID),
    ("gd_embedding_forward", _embedding, dict(id_bits=16), INVALID), ("gd_embedding_forward", _embedding, dict(table=None), INVALID),
    ("gd_embedding_forward", _embedding, dict(table=0x1001), INVALID), ("gd_embedding_forward", _embedding, dict(ld_table=7), INVALID),
    ("gd_embedding_forward", _embedding, dict(ids=None), INVALID), ("gd_embedding_forward", _embedding, dict(ids=0x2004), INVALID),
    ("gd_embedding_forward", _embedding, dict(y=None), INVALID), ("gd_embedding_forward", _embedding, dict(ld_y=3), INVALID),
    ("gd_embedding_forward", _embedding, dict(tokens=1 << 31), LARGE), ("gd_embedding_forward", _embedding, dict(width=1 << 20), LARGE),
    ("gd_embedding_forward", _embedding, dict(tokens=0, table=None), 0),
    ("gd_embedding_backward", _embedding_back, dict(dtype=-1), INVALID), ("gd_embedding_backward", _embedding_back, dict(dtable_dtype=2), INVALID),
    ("gd_embedding_backward", _embedding_back, dict(flags=2), INVALID), ("gd_embedding_backward", _embedding_back, dict(flags=1, dtable_dtype=1), INVALID),
    ("gd_embedding_backward", _embedding_back, dict(reserved=1), INVALID), ("gd_embedding_backward", _embedding_back, dict(dy=None), INVALID),
    ("gd_embedding_backward", _embedding_back, dict(dtable=0x3002), INVALID), ("gd_embedding_backward", _embedding_back, dict(ld_dtable=5), INVALID),
    ("gd_embedding_backward", _embedding_back, dict(workspace=None), SPACE), ("gd_embedding_backward", _embedding_back, dict(workspace=0x4010), SPACE),
    ("gd_embedding_backward", _embedding_back, dict(workspace_bytes=255), SPACE), ("gd_embedding_backward", _embedding_back, dict(vocab=1 << 31), LARGE),
    ("gd_embedding_backward", _embedding_back, dict(vocab=0), 0), ("gd_embedding_backward", _embedding_back, dict(tokens=0, flags=1), 0),
    ("gd_layer_norm_forward", _norm, dict(dtype=5), INVALID), ("gd_layer_norm_forward", _norm, dict(param_dtype=2), INVALID),
    ("gd_layer_norm_forward", _norm, dict(eps=-1.0), INVALID), ("gd_layer_norm_forward", _norm, dict(eps=float("nan")), INVALID),
    ("gd_layer_norm_forward", _norm, dict(reserved=1), INVALID), ("gd_layer_norm_forward", _norm, dict(width=0), INVALID),
    ("gd_layer_norm_forward", _norm, dict(x=None), INVALID), ("gd_layer_norm_forward", _norm, dict(x=0x1001), INVALID),
    ("gd_layer_norm_forward", _norm, dict(y=0x1000, ldy=9), INVALID), ("gd_layer_norm_forward", _norm, dict(weight=0x2002), INVALID),
    ("gd_layer_norm_forward", _norm, dict(ldx=7), INVALID), ("gd_layer_norm_forward", _norm, dict(mean=0x5002), INVALID),
    ("gd_layer_norm_forward", _norm, dict(rows=1 << 31), LARGE), ("gd_layer_norm_forward", _norm, dict(rows=0, x=None), 0),
    ("gd_layer_norm_backward", _norm_back, dict(flags=4), INVALID), ("gd_layer_norm_backward", _norm_back, dict(dy=None), INVALID),
    ("gd_layer_norm_backward", _norm_back, dict(mean=None), INVALID), ("gd_layer_norm_backward", _norm_back, dict(rstd=None), INVALID),
    ("gd_layer_norm_backward", _norm_back, dict(dx=0x1000, ld_dx=9), INVALID), ("gd_layer_norm_backward", _norm_back, dict(ld_add=7), INVALID),
    ("gd_layer_norm_backward", _norm_back, dict(dweight=0x8002), INVALID), ("gd_layer_norm_backward", _norm_back, dict(workspace=None), SPACE),
    ("gd_layer_norm_backward", _norm_back, dict(workspace_bytes=4 * 2 * 8 * 4 - 1), SPACE),
    ("gd_layer_norm_backward", _norm_back, dict(dx=None, dweight=None, dbias=None), 0),
    ("gd_recurrence_forward", _scan, dict(dtype=3), INVALID), ("gd_recurrence_forward", _scan, dict(offset_bits=8), INVALID),
    ("gd_recurrence_forward", _scan, dict(offsets=0x1004), INVALID), ("gd_recurrence_forward", _scan, dict(offsets=None, sequences=4), INVALID),
    ("gd_recurrence_forward", _scan, dict(offsets=None, sequences=0), INVALID), ("gd_recurrence_forward", _scan, dict(gate=None), INVALID),
    ("gd_recurrence_forward", _scan, dict(ld_value=7), INVALID), ("gd_recurrence_forward", _scan, dict(y=0x4001), INVALID),
    ("gd_recurrence_forward", _scan, dict(h0=0x5002), INVALID), ("gd_recurrence_forward", _scan, dict(rows=1 << 31), LARGE),
    ("gd_recurrence_forward", _scan, dict(width=0, gate=None), 0), ("gd_recurrence_forward", _scan, dict(sequences=0), 0),
    ("gd_recurrence_backward", _scan_back, dict(marks=None), INVALID), ("gd_recurrence_backward", _scan_back, dict(dgate=None), INVALID),
    ("gd_recurrence_backward", _scan_back, dict(dgate=0x3000, ld_dgate=9), INVALID), ("gd_recurrence_backward", _scan_back, dict(dvalue=0x4000, ld_dvalue=10), INVALID),
    ("gd_recurrence_backward", _scan_back, dict(dh0=0x9001), INVALID), ("gd_recurrence_backward", _scan_back, dict(sequences=1 << 31), LARGE)])
def test_refused_on_the_host(lib, call, make, changes, code):
    a = make()
    for field, value in changes.items():
        setattr(a, field, value)
    assert getattr(lib, call)(C.byref(a), None) == code
    assert getattr(lib, call)(None, None) == INVALID


def test_workspaces_and_marks(lib):
    def embedding(tokens, vocab, width):
        size = C.c_size_t(0)
        assert lib.gd_embedding_workspace_bytes(tokens, vocab, width, C.byref(size)) == B.GD_OK
        return size.value

    assert 256 <= embedding(0, 10, 8) <= embedding(100, 10, 8) < embedding(9000, 10, 8) < embedding(9000, 10, 512)
    assert lib.gd_embedding_workspace_bytes(1, 1, 1 << 20, C.byref(C.c_size_t(0))) == LARGE and lib.gd_embedding_workspace_bytes(1, 1, 1, None) == INVALID
    size = C.c_size_t(0)
    assert lib.gd_layer_norm_workspace_bytes(4, 8, C.byref(size)) == B.GD_OK and size.value == 4 * 2 * 8 * 4
    assert lib.gd_layer_norm_workspace_bytes(1 << 31, 8, C.byref(size)) == LARGE and lib.gd_layer_norm_workspace_bytes(1, 1, None) == INVALID

    def gated(m, n, k, any_layout=0):
        assert lib.gd_gated_workspace_bytes(m, n, k, any_layout, C.byref(size)) == B.GD_OK
        return size.value

    assert 256 <= gated(0, 0, 0) < gated(80, 64, 64) < gated(80, 65, 64) < gated(80, 65, 65) and gated(80, 64, 64) < gated(80, 64, 64, 1)
    assert lib.gd_gated_workspace_bytes(1, 1 << 30, 1, 0, C.byref(size)) == LARGE and lib.gd_gated_workspace_bytes(1, 1, 1, 0, None) == INVALID
    count = C.c_uint64(0)
    assert lib.gd_recurrence_marks_rows(640, 3, C.byref(count)) == B.GD_OK and count.value == 13
    for rows, sequences in ((0, 1), (63, 2), (64, 2), (1000, 7)):
        assert lib.gd_recurrence_marks_rows(rows, sequences, C.byref(count)) == B.GD_OK and count.value == rows // L._MARK_ROWS + sequences
    assert lib.gd_recurrence_marks_rows(1, 1 << 31, C.byref(count)) == LARGE and lib.gd_recurrence_marks_rows(1, 1, None) == INVALID


def test_sessions_and_calls_want_a_gpu():
    x = torch.zeros(4, 8)
    for make in (lambda: L.EmbeddingSession(4, 8, 4, device="cpu"), lambda: L.LayerNormSession(8, 4, device="cpu"), lambda: L.GatedLinearSession(8, 8, 4, device="cpu"), lambda: L.recurrence_forward(x, x),
                 lambda: L.recurrence_marks(4, 1, 8, device="cpu"), lambda: L.recurrence_backward(x, x, x, x, x, x)):
        with pytest.raises(RuntimeError, match="CUDA device is needed"):
            make()


def _without_gpu(cls, **attributes):
    """A session as its constructor leaves it on a GPU, on tensors that claim to live there (nothing is launched: the checks come first)."""
    s = cls.__new__(cls)
    s._index, s.device, s._lib, s.workspace = -1, torch.device("cpu"), None, torch.empty(256, dtype=torch.uint8)
    for name, value in attributes.items():
        setattr(s, name, value)
    return s


def test_tensors_that_do_not_fit_are_refused():
    s = _without_gpu(L.EmbeddingSession, vocab=10, width=8, max_tokens=4)
    table, ids = torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64)
    for bad in (dict(table=torch.zeros(9, 8)), dict(ids=torch.zeros(5, dtype=torch.int64)), dict(ids=torch.zeros(4)), dict(ids=torch.zeros(2, 2, dtype=torch.int64)),
                dict(out=torch.zeros(3, 8)), dict(out=torch.zeros(4, 8, dtype=torch.float64)), dict(table=torch.zeros(8, 10).t())):
        with pytest.raises(ValueError):
            s.forward(**{**dict(table=table, ids=ids, out=torch.zeros(4, 8)), **bad})
    for bad in (dict(dy=torch.zeros(4, 7)), dict(dtable=torch.zeros(10, 9)), dict(ids=torch.zeros(3, dtype=torch.int64))):
        with pytest.raises(ValueError):
            s.backward(**{**dict(dy=torch.zeros(4, 8), ids=ids, dtable=torch.zeros(10, 8)), **bad})
    s.workspace = None
    with pytest.raises(ValueError, match="gradient=False"):
        s.backward(torch.zeros(4, 8), ids, torch.zeros(10, 8))

    n = _without_gpu(L.LayerNormSession, width=8, max_rows=4, dtype=torch.bfloat16, eps=1e-5, _code=1)
    x, half = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.float16)
    for bad in (dict(x=torch.zeros(4, 8)), dict(x=torch.zeros(5, 8, dtype=torch.bfloat16)), dict(weight=half), dict(weight=torch.zeros(8), bias=torch.zeros(8).bfloat16()),
                dict(weight=torch.zeros(7)), dict(mean=torch.zeros(3)), dict(rstd=torch.zeros(4).bfloat16()), dict(out=torch.zeros(4, 8))):
        with pytest.raises(ValueError):
            n.forward(**{**dict(x=x, out=torch.empty_like(x)), **bad})
    stats = torch.zeros(4)
    for bad in (dict(x=x[:3]), dict(mean=stats[:3]), dict(rstd=stats.bfloat16()), dict(dx=torch.zeros(4, 8)), dict(dweight=half), dict(dbias=torch.zeros(9)),
                dict(add=torch.zeros(8, 4, dtype=torch.bfloat16).t())):
        with pytest.raises(ValueError):
            n.backward(**{**dict(dy=x, x=x, weight=None, mean=stats, rstd=stats), **bad})


def test_gated_tensors_that_do_not_fit_are_refused():
    for wrong in (dict(dtype=torch.float32), dict(activation="sigmoid"), dict(w_layout="out")):
        with pytest.raises(ValueError):
            L.GatedLinearSession(8, 16, 4, **wrong)
    s = _without_gpu(L.GatedLinearSession, n_in=8, n_out=16, max_rows=4, dtype=torch.bfloat16, activation="silu", w_layout="in_out", w_shape=(8, 32))
    s._bind(s.workspace)
    x, w, y, pre = (torch.zeros(*shape, dtype=torch.bfloat16) for shape in ((4, 8), (8, 32), (4, 16), (4, 32)))
    for bad in (dict(x=x.float()), dict(x=torch.zeros(5, 8).bfloat16()), dict(w=w[:, :16]), dict(w=w.t()), dict(bias=torch.zeros(16)), dict(bias=torch.zeros(32).half()),
                dict(out=torch.zeros(4, 16)), dict(pre=y)):
        with pytest.raises(ValueError):
            s.forward(**{**dict(x=x, w=w, out=y), **bad})
    for bad in (dict(dy=x), dict(pre=y), dict(dx=x, w=None), dict(dw=w, x=None), dict(dw=w.half()), dict(db=torch.zeros(16)), dict(dx=y)):
        with pytest.raises(ValueError):
            s.backward(**{**dict(dy=y, x=x, w=w, pre=pre), **bad})


def test_recurrence_arguments_that_do_not_fit_are_refused(monkeypatch):
    monkeypatch.setattr(L, "_matrix_index", lambda t, name: -1)
    x, state = torch.zeros(6, 8), torch.zeros(2, 8)
    for bad in (dict(gate=torch.zeros(6, 7)), dict(gate=x.bfloat16()), dict(offsets=torch.zeros(4, dtype=torch.int64)), dict(offsets=torch.zeros(3)), dict(sequences=4),
                dict(sequences=0), dict(h0=torch.zeros(3, 8)), dict(h_last=state.double()), dict(h0=torch.zeros(8, 2).t()), dict(out=x.bfloat16()),
                dict(marks=torch.zeros(1, 8)), dict(marks=torch.zeros(2, 9))):
        with pytest.raises(ValueError):
            L.recurrence_forward(**{**dict(gate=x, value=x, out=torch.empty_like(x), sequences=2), **bad})
    for bad in (dict(dy=x[:5]), dict(dgate=x.half()), dict(dh_last=state[:1]), dict(dh0=state.half()), dict(marks=torch.zeros(1, 8))):
        with pytest.raises(ValueError):
            L.recurrence_backward(**{**dict(dy=x, gate=x, value=x, marks=torch.zeros(2, 8), dgate=x, dvalue=x, sequences=2), **bad})
