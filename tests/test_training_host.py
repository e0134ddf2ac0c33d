"""Host-side checks of the training-step operators that need no GPU: exports, structures, sizing, argument validation."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import build as gd_build
from paper_1704_05021_b200 import training as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    gd_build.build_library()
    return T.load_library()


def test_every_declared_symbol_is_exported(lib):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gd_train.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(gd_[a-z_]+)\s*\(", header))
    assert declared == set(T.EXPORTS)
    for name in declared:
        assert getattr(lib, name) is not None


def test_header_is_plain_c_and_structures_agree(lib, tmp_path):
    """include/gd_train.h compiles as C99, a C program links and calls it, and the binding's structures have the C sizes."""
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler here")
    src = tmp_path / "use_gd_train.c"
    src.write_text(r'''
#include <stdio.h>
#include "gd_train.h"
int main(void) {
  size_t ws = 0;
  if (gd_linear_workspace_bytes(80, 10, 4096, 0, &ws) != GD_OK || ws == 0) return 1;
  if (gd_linear_forward(NULL, NULL) != GD_ERR_INVALID_ARG || gd_adamw_step(NULL, NULL) != GD_ERR_INVALID_ARG) return 2;
  printf("%zu %zu %zu %zu %zu\n", sizeof(gd_linear_forward_args), sizeof(gd_linear_backward_args), sizeof(gd_cross_entropy_args),
         sizeof(gd_adamw_tensor), sizeof(gd_adamw_args));
  return 0;
}
''')
    exe, libdir = tmp_path / "use_gd_train", os.path.dirname(gd_build.LIB_PATH)
    res = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-L", libdir,
                          "-l:libgd.so", "-Wl,-rpath," + libdir, "-o", str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, (out.returncode, out.stderr)
    ours = (T._LinearForwardArgs, T._LinearBackwardArgs, T._CrossEntropyArgs, T._AdamwTensor, T._AdamwArgs)
    assert [int(x) for x in out.stdout.split()] == [C.sizeof(s) for s in ours]


def test_linear_workspace_grows_with_what_is_ragged(lib):
    def size(m, n, k, any_layout=0):
        out = C.c_size_t(0)
        assert lib.gd_linear_workspace_bytes(m, n, k, any_layout, C.byref(out)) == B.GD_OK
        return out.value

    even, odd, anything = size(80, 4096, 784), size(80, 4096, 785), size(80, 4096, 784, 1)
    assert 0 < even < odd and even < anything
    assert size(0, 0, 0) >= 256
    assert lib.gd_linear_workspace_bytes(1 << 31, 1, 1, 0, C.byref(C.c_size_t(0))) == B.GD_ERR_TOO_LARGE
    assert lib.gd_linear_workspace_bytes(1, 1, 1, 0, None) == B.GD_ERR_INVALID_ARG


def _forward_args():
    a = T._LinearForwardArgs()
    a.m, a.n, a.k, a.dtype, a.y_dtype = 4, 8, 16, T.GD_DTYPE_BF16, T.GD_DTYPE_BF16
    a.x, a.ldx, a.w, a.ldw, a.y, a.ldy = 0x1000, 16, 0x2000, 8, 0x3000, 8
    a.workspace, a.workspace_bytes = 0x4000, 4096
    return a


@pytest.mark.parametrize("field, value, code", [
    ("dtype", T.GD_DTYPE_FP32, B.GD_ERR_INVALID_ARG), ("dtype", 7, B.GD_ERR_INVALID_ARG), ("activation", 4, B.GD_ERR_INVALID_ARG),
    ("w_layout", 2, B.GD_ERR_INVALID_ARG), ("y_dtype", T.GD_DTYPE_FP16, B.GD_ERR_INVALID_ARG), ("reserved", 1, B.GD_ERR_INVALID_ARG),
    ("x", None, B.GD_ERR_INVALID_ARG), ("x", 0x1001, B.GD_ERR_INVALID_ARG), ("ldx", 15, B.GD_ERR_INVALID_ARG), ("w", None, B.GD_ERR_INVALID_ARG),
    ("ldw", 7, B.GD_ERR_INVALID_ARG), ("y", None, B.GD_ERR_INVALID_ARG), ("ldy", 3, B.GD_ERR_INVALID_ARG), ("m", 1 << 31, B.GD_ERR_TOO_LARGE),
    ("workspace", None, B.GD_ERR_WORKSPACE), ("workspace", 0x4010, B.GD_ERR_WORKSPACE), ("workspace_bytes", 255, B.GD_ERR_WORKSPACE)])
def test_linear_forward_refuses_on_the_host(lib, field, value, code):
    a = _forward_args()
    setattr(a, field, value)
    assert lib.gd_linear_forward(C.byref(a), None) == code


def test_linear_forward_refuses_a_workspace_without_room_before_anything_runs(lib):
    a = _forward_args()
    a.ldx, a.workspace_bytes = 17, 256                    # ragged rows, no room to lay them out
    assert lib.gd_linear_forward(C.byref(a), None) == B.GD_ERR_WORKSPACE
    a = _forward_args()
    a.ldw, a.workspace_bytes = 9, 256
    assert lib.gd_linear_forward(C.byref(a), None) == B.GD_ERR_WORKSPACE


def test_linear_backward_refuses_on_the_host(lib):
    def args():
        a = T._LinearBackwardArgs()
        a.m, a.n, a.k, a.dtype, a.dw_dtype = 4, 8, 16, T.GD_DTYPE_BF16, T.GD_DTYPE_FP32
        a.dy, a.ld_dy, a.x, a.ldx, a.w, a.ldw = 0x1000, 8, 0x2000, 16, 0x3000, 8
        a.dx, a.ld_dx, a.dw, a.ld_dw, a.db = 0x5000, 16, 0x6000, 8, 0x7000
        a.workspace, a.workspace_bytes = 0x8000, 256
        return a

    for field, value, code in [("dy", None, -1), ("flags", 2, -1), ("x", None, -1), ("w", None, -1), ("db", 0x7002, -1), ("dw_dtype", 2, -1), ("ld_dw", 7, -1),
                               ("activation", T.GD_ACT_GELU, -1), ("workspace", None, -3), ("ld_dy", 9, -3), ("ldx", 19, -3), ("ldw", 9, -3), ("k", 1 << 31, -2)]:
        a = args()
        setattr(a, field, value)
        assert lib.gd_linear_backward(C.byref(a), None) == code, field
    a = args()
    a.flags, a.dw_dtype = T.GD_LINEAR_ACCUMULATE, T.GD_DTYPE_BF16
    assert lib.gd_linear_backward(C.byref(a), None) == B.GD_ERR_INVALID_ARG
    a = args()
    a.dx = a.dw = a.db = None
    assert lib.gd_linear_backward(C.byref(a), None) == B.GD_OK            # nothing asked for


def test_cross_entropy_refuses_on_the_host(lib):
    def args():
        a = T._CrossEntropyArgs()
        a.rows, a.classes, a.target_bits = 4, 8, 64
        a.logits, a.ld_logits, a.targets, a.loss, a.grad, a.ld_grad = 0x1000, 8, 0x2000, 0x3000, 0x4000, 8
        return a

    for field, value, code in [("classes", 0, -1), ("dtype", 3, -1), ("target_bits", 16, -1), ("logits", None, -1), ("logits", 0x1002, -1),
                               ("targets", 0x2004, -1), ("ld_logits", 7, -1), ("ld_grad", 7, -1), ("loss", 0x3001, -1), ("rows", 1 << 31, -2)]:
        a = args()
        setattr(a, field, value)
        assert lib.gd_cross_entropy(C.byref(a), None) == code, field
    a = args()
    a.grad, a.ld_grad = a.logits, 9                                      # in place, but with other rows
    assert lib.gd_cross_entropy(C.byref(a), None) == B.GD_ERR_INVALID_ARG
    a = args()
    a.rows = 0
    assert lib.gd_cross_entropy(C.byref(a), None) == B.GD_OK
    assert lib.gd_cross_entropy(None, None) == B.GD_ERR_INVALID_ARG


def test_adamw_refuses_on_the_host(lib):
    def args(**tensor):
        t = (T._AdamwTensor * 1)()
        t[0].param, t[0].grad, t[0].m, t[0].v, t[0].n = 0x1000, 0x2000, 0x3000, 0x4000, 10
        for name, value in tensor.items():
            setattr(t[0], name, value)
        a = T._AdamwArgs()
        a.tensors, a.n_tensors, a.state_bits, a.step, a.beta1, a.beta2, a.eps, a.grad_scale = t, 1, 32, 1, 0.9, 0.999, 1e-8, 1.0
        return a

    for field, value in [("state_bits", 16), ("param_dtype", 3), ("grad_dtype", -1), ("copy_dtype", 9), ("step", 0), ("beta1", 1.0), ("beta2", float("nan")),
                         ("eps", -1e-9), ("lr", float("inf")), ("grad_scale_dev", 0x1002), ("reserved", 5), ("state_bits", 8)]:
        a = args()
        setattr(a, field, value)
        assert lib.gd_adamw_step(C.byref(a), None) == B.GD_ERR_INVALID_ARG, field     # (8 bits: the scales are missing)
    for tensor in (dict(param=None), dict(grad=0x2002), dict(m=None), dict(v=0x4001), dict(copy=0x5002), dict(weight_decay=float("nan"))):
        assert lib.gd_adamw_step(C.byref(args(**tensor)), None) == B.GD_ERR_INVALID_ARG, tensor
    assert lib.gd_adamw_step(C.byref(args(n=1 << 40)), None) == B.GD_ERR_TOO_LARGE
    assert lib.gd_adamw_step(C.byref(args(n=0, param=None)), None) == B.GD_OK          # an empty tensor needs nothing
    a = args()
    a.n_tensors = 0
    assert lib.gd_adamw_step(C.byref(a), None) == B.GD_OK
