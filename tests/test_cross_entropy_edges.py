"""The cross-entropy at its edges: slices of a row as long as shared memory without asking for more, rows in place, a masked target.

Bounds: exp of a difference d in fp32 is off by |d| 2^-23 for the argument and 2^-21 for the function, sums and the logarithm by a few
2^-23, a gradient rounds once to its type.
"""
import os
import subprocess
import sys

import pytest
import torch

from paper_1704_05021_b200 import training as T

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}


def check(rows, classes, dtype, in_place=False):
    gen = torch.Generator(device="cuda").manual_seed(classes)
    logits = (torch.randn(rows, classes, generator=gen, device="cuda") * 3).to(dtype)
    t = torch.randint(classes, (rows,), generator=gen, device="cuda")
    z = logits.double()
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    grad = logits if in_place else torch.empty_like(logits)
    T.cross_entropy(logits, t, loss=loss, lse=lse, grad=grad)
    want = torch.logsumexp(z, 1)
    top = z.max(1).values
    room = 2.0 ** -22 * (top.abs() + 2 * (want - top) + (want - z.gather(1, t[:, None])[:, 0]).abs()) + 2.0 ** -20
    assert bool(((lse.double() - want).abs() <= room).all()), (classes, "lse")
    assert bool(((loss.double() - (want - z.gather(1, t[:, None])[:, 0])).abs() <= room).all()), (classes, "loss")
    p = torch.softmax(z, 1)
    room = p * (2.0 ** -19 + (top[:, None] - z) * 2.0 ** -22)
    p.scatter_add_(1, t[:, None], torch.full_like(top, -1.0)[:, None])
    room += p.abs() * (ROUND[dtype] + 2.0 ** -23) + 2.0 ** -126 + TINY[dtype]
    assert bool(((grad.double() - p).abs() <= room).all()), (classes, "grad")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
def test_slices_as_long_as_shared_memory(cuda_device, dtype):
    """Slices of 48 KB and just below, in one CTA and in clusters of two to eight, in a process that has called nothing before."""
    first = 12288 if dtype is torch.float32 else 24576
    sizes = [n for c in (1, 2, 4, 8) for n in (first * c - 63 * c, first * c)]
    code = (f"import sys; sys.path[:0] = [{ROOT!r}, {os.path.dirname(os.path.abspath(__file__))!r}]\n"
            f"import torch, test_cross_entropy_edges as e\n"
            f"for n in {sizes}: e.check(200, n, {dtype})\n")
    res = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert res.returncode == 0, res.stderr[-2000:]


@pytest.mark.parametrize("rows, classes", [(3, 40000), (150, 85000), (1, 200000)], ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_in_place_with_the_target_in_any_slice(cuda_device, dtype, rows, classes):
    """Rows that several CTAs share, worked on in place, the target in every part of them: the bits of a call into another buffer.  (The
    CTA that writes the loss reads the target's logit from the slice of another, which overwrites it.)"""
    gen = torch.Generator(device=cuda_device).manual_seed(classes)
    logits = (torch.randn(rows, classes, generator=gen, device=cuda_device) * 3).to(dtype)
    for at in range(16):
        t = (torch.arange(rows, device=cuda_device) * 7919 + at * (classes // 16) + 13 * at) % classes
        apart, loss, inside = torch.empty_like(logits), [torch.empty(rows, device=cuda_device) for _ in range(2)], logits.clone()
        T.cross_entropy(logits, t, loss=loss[0], grad=apart)
        T.cross_entropy(inside, t, loss=loss[1], grad=inside)
        assert torch.equal(loss[0], loss[1]) and torch.equal(apart, inside)
    check(rows, classes, dtype, in_place=True)


@pytest.mark.parametrize("classes", [10, 700, 5000, 85000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
def test_a_masked_target(cuda_device, dtype, classes):
    """The target's own logit is -inf while other classes are not masked: loss +inf, the gradient that of the formula; ignored, the row is 0."""
    gen = torch.Generator(device=cuda_device).manual_seed(classes)
    x = torch.randn(90, classes, generator=gen, device=cuda_device).to(dtype)
    x[:, classes // 2:] = -float("inf")
    t = torch.full((90,), classes - 1, device=cuda_device)
    t[1::3], t[2::3] = 0, -100
    loss, lse, grad = torch.empty(90, device=cuda_device), torch.empty(90, device=cuda_device), torch.empty_like(x)
    T.cross_entropy(x, t, loss=loss, lse=lse, grad=grad, grad_scale=0.5)
    assert bool((loss[0::3] == float("inf")).all()) and bool(torch.isfinite(loss[1::3]).all()) and bool((loss[2::3] == 0).all())
    assert bool(((lse.double() - torch.logsumexp(x.double(), 1)).abs() <= 2.0 ** -18).all())
    p = torch.softmax(x.double(), 1) * 0.5
    room = p * (2.0 ** -18 + ROUND[dtype]) + 2.0 ** -126 + TINY[dtype]
    half = slice(0, classes // 2)
    assert bool(((grad[0::3, half].double() - p[0::3, half]).abs() <= room[0::3, half]).all())
    assert bool((grad[0::3, classes // 2:classes - 1] == 0).all()) and bool((grad[0::3, classes - 1] == -0.5).all())
    assert bool((grad[1::3, classes // 2:] == 0).all()) and bool((grad[2::3] == 0).all())
