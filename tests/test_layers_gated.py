"""The gated block of include/gd_layers.h on a GPU against plain implementations in 64 bits.

Tolerances are bounds on what the stated arithmetic can do, not observations:
  products     fp32 accumulation in steps of 16 products, each rounding (possibly truncating) once: at most (k / 16 + 8) 2^-22 of the sum of
               magnitudes
  activations  x Phi(x) and x sigmoid(x) and their slopes: 2^-20 and, for the exponential's argument, |x| 2^-23, of max(1, |x|)
  gradients    dz is rounded to 16 bits before the products (half a step of each entry); its sums are not
"""
import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import layers as L

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}
ACT = {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}
STEEP = {"none": 1.0, "relu": 1.0, "gelu": 1.13, "silu": 1.1}            # the largest slopes


def _gen(device, seed):
    return torch.Generator(device=device).manual_seed(seed)


def _rand(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen, device=gen.device) * scale).to(dtype)


def _within(got, ref, tol, what):
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - ref).abs() - tol
    assert bool((over <= 0).all()), f"{what}: {float(over.max())} past the bound at {int(over.argmax())}"


class Inset:
    """A matrix that starts `offset` elements into a buffer, its rows further apart than their length; the rest is a number nobody computes."""

    def __init__(self, rows, cols, dtype, device, strided, fill=-77.0):
        pitch, offset = (cols + 3, 5) if strided else (cols, 0)
        self.buf = torch.full((rows * pitch + 16,), fill, dtype=dtype, device=device)
        self.inside = torch.zeros_like(self.buf, dtype=torch.bool)
        self.t, mask = (b[offset:offset + rows * pitch].view(rows, pitch)[:, :cols] for b in (self.buf, self.inside))
        mask.fill_(True)
        self.fill = fill

    def check_around(self):
        assert bool((self.buf[~self.inside] == self.fill).all()), "written outside the matrix"


def _inset(x, strided):
    m = Inset(*x.shape, x.dtype, x.device, strided)
    m.t.copy_(x)
    return m.t


def _act_off(z, name):
    return torch.zeros_like(z) if name in ("none", "relu") else (2.0 ** -20 + z.abs() * 2.0 ** -23) * z.abs().clamp(min=1.0)


def _slope(z, name):
    z = z.clone().requires_grad_()
    return torch.autograd.grad(ACT[name](z).sum(), z)[0]


SHAPES = [(1, 1, 1), (1, 8, 16), (2, 24, 40), (17, 33, 65), (3, 10, 784), (80, 100, 500), (128, 64, 64), (129, 257, 191), (1, 4096, 2048), (16, 520, 4096),
          (300, 500, 250), (1000, 7, 96), (513, 264, 1031), (64, 72, 0), (260, 136, 8)]
LARGE = [(2500, 2048, 300), (4096, 1544, 512), (5000, 1003, 264), (1300, 4100, 200)]      # many tiles: the pairs' kernel


def _check_forward(device, m, n, k, dtype, act, layout, bias, pre, strided):
    gen = _gen(device, m + n)
    x, w = _rand(gen, m, k, dtype=dtype), _rand(gen, *((k, 2 * n) if layout == "in_out" else (2 * n, k)), dtype=dtype, scale=max(k, 1) ** -0.5)
    x, w = _inset(x, strided), _inset(w, strided)
    b = _rand(gen, 2 * n, dtype=bias) if bias else None
    y, z = Inset(m, n, dtype, device, strided), Inset(m, 2 * n, dtype, device, strided) if pre else None
    s = L.GatedLinearSession(k, n, m, dtype=dtype, activation=act, w_layout=layout, device=device, any_layout=strided)
    got = s.forward(x, w, b, out=y.t, pre=z.t if pre else None)
    assert got is y.t and s.status() == B.GD_OK
    w64 = w.double() if layout == "in_out" else w.double().T
    z64 = x.double() @ w64 + (b.double() if bias else 0.0)
    off = (k / 16 + 8) * 2.0 ** -22 * (x.double().abs() @ w64.abs() + (b.double().abs() if bias else 0.0))
    if pre:
        _within(z.t, z64, off + HALF_ULP[dtype] * (z64.abs() + off) + TINY[dtype], "pre")
        z.check_around()
    g, u, off_g, off_u = z64[:, :n], z64[:, n:], off[:, :n], off[:, n:]
    off_a = STEEP[act] * off_g + _act_off(g, act)
    ref, tol = ACT[act](g) * u, off_a * (u.abs() + off_u) + ACT[act](g).abs() * off_u
    _within(y.t, ref, tol + (HALF_ULP[dtype] + 2.0 ** -23) * (ref.abs() + tol) + TINY[dtype], "y")
    y.check_around()


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("m, n, k", SHAPES + LARGE)
def test_forward(cuda_device, m, n, k, layout, strided):
    _check_forward(cuda_device, m, n, k, torch.bfloat16, "silu", layout, torch.float32, True, strided)
    _check_forward(cuda_device, m, n, k, torch.float16, "gelu", layout, None, False, strided)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("m, n, k", [(5, 24, 72), (200, 130, 96), (2500, 2048, 136)])
def test_forward_activations(cuda_device, m, n, k, act):
    _check_forward(cuda_device, m, n, k, torch.bfloat16, act, "in_out", torch.bfloat16, False, False)
    _check_forward(cuda_device, m, n, k, torch.float16, act, "out_in", torch.float32, True, True)


def _check_backward(device, m, n, k, dtype, act, layout, grads, strided):
    gen = _gen(device, m + n + 1)
    x, w = _rand(gen, m, k, dtype=dtype), _rand(gen, *((k, 2 * n) if layout == "in_out" else (2 * n, k)), dtype=dtype, scale=max(k, 1) ** -0.5)
    dy, pre = _rand(gen, m, n, dtype=dtype), _rand(gen, m, 2 * n, dtype=dtype)
    x, w, dy, pre = (_inset(t, strided) for t in (x, w, dy, pre))
    dx, dw = Inset(m, k, dtype, device, strided), Inset(*w.shape, grads, device, strided)
    db = torch.full((2 * n,), 9.0, device=device)
    s = L.GatedLinearSession(k, n, m, dtype=dtype, activation=act, w_layout=layout, device=device, any_layout=strided)
    s.backward(dy, x, w, pre, dx=dx.t, dw=dw.t, db=db)
    assert s.status() == B.GD_OK
    g, u, d = pre[:, :n].double(), pre[:, n:].double(), dy.double()
    dz = torch.cat([d * u * _slope(g, act), d * ACT[act](g)], 1)
    off = torch.cat([(d * u).abs() * _act_off(g, act), d.abs() * _act_off(g, act)], 1) + 3 * 2.0 ** -24 * dz.abs()
    _within(db, dz.sum(0), off.sum(0) + (m / 64 + 64) * 2.0 ** -24 * dz.abs().sum(0) + TINY[torch.float32], "db")
    off = off + HALF_ULP[dtype] * dz.abs() + TINY[dtype]
    w64 = w.double() if layout == "in_out" else w.double().T
    ref, tol = dz @ w64.T, off @ w64.abs().T + (2 * n / 16 + 8) * 2.0 ** -22 * (dz.abs() @ w64.abs().T)
    _within(dx.t, ref, tol + HALF_ULP[dtype] * (ref.abs() + tol) + TINY[dtype], "dx")
    dx.check_around()
    ref, tol = x.double().T @ dz, x.double().abs().T @ off + (m / 16 + 8) * 2.0 ** -22 * (x.double().abs().T @ dz.abs())
    if layout == "out_in":
        ref, tol = ref.T, tol.T
    _within(dw.t, ref, tol + HALF_ULP[grads] * (ref.abs() + tol) + TINY[grads], "dw")
    dw.check_around()
    if grads is torch.float32:
        first = dw.t.clone(), db.clone()
        held_w, held_b = _rand(gen, *w.shape), _rand(gen, 2 * n)
        dw.t.copy_(held_w), db.copy_(held_b)
        s.backward(dy, x, w, pre, dw=dw.t, db=db, accumulate=True)
        _within(dw.t, first[0].double() + held_w.double(), 2.0 ** -23 * (first[0].double().abs() + held_w.double().abs()), "dw added")
        assert torch.equal(db, held_b + first[1])
    alone = torch.empty(m, k, dtype=dtype, device=device)
    s.backward(dy, None, w, pre, dx=alone)
    assert torch.equal(alone, dx.t)


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("m, n, k", SHAPES + LARGE[:2])
def test_backward(cuda_device, m, n, k, layout, strided):
    _check_backward(cuda_device, m, n, k, torch.bfloat16, "silu", layout, torch.float32, strided)
    _check_backward(cuda_device, m, n, k, torch.float16, "gelu", layout, torch.float16, strided)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_backward_activations(cuda_device, act):
    _check_backward(cuda_device, 200, 130, 96, torch.bfloat16, act, "in_out", torch.bfloat16, False)
    _check_backward(cuda_device, 70, 64, 40, torch.float16, act, "out_in", torch.float32, False)


def test_gradient_against_differences(cuda_device):
    """The gradient of sum(dy * y) that the call gives against differences of the formula in 64 bits."""
    gen = _gen(cuda_device, 3)
    m, n, k = 4, 8, 16
    x, w = _rand(gen, m, k, dtype=torch.float16), _rand(gen, k, 2 * n, dtype=torch.float16, scale=0.25)
    dy = _rand(gen, m, n, dtype=torch.float16)
    s = L.GatedLinearSession(k, n, m, dtype=torch.float16, activation="gelu", device=cuda_device)
    pre = torch.empty(m, 2 * n, dtype=torch.float16, device=cuda_device)
    s.forward(x, w, pre=pre)
    dx, dw = torch.empty_like(x), torch.empty(k, 2 * n, device=cuda_device)
    s.backward(dy, x, w, pre, dx=dx, dw=dw)

    def loss(x, w):
        z = x @ w
        return (dy.double() * torch.nn.functional.gelu(z[:, :n]) * z[:, n:]).sum()

    step = 1e-5
    for grad, at, spots in ((dx, 0, [(0, 0), (3, 15), (1, 7)]), (dw, 1, [(0, 0), (15, 15), (5, 3), (5, 11)])):
        for r, c in spots:
            up, down = [x.double(), w.double()], [x.double(), w.double()]
            up[at][r, c] += step
            down[at][r, c] -= step
            slope = float(loss(*up) - loss(*down)) / (2 * step)
            # pre and dz are rounded to 16 bits: 2^-11 each of at most 16 terms below 10
            assert abs(slope - float(grad[r, c])) < 2 * 16 * 10 * 2.0 ** -11


def test_rows_of_nan_and_of_nothing(cuda_device):
    """A row that is not finite spoils its own results alone; no rows, no outputs, no inputs."""
    for m in (20, 600):
        gen = _gen(cuda_device, m)
        x, w = _rand(gen, m, 64, dtype=torch.bfloat16), _rand(gen, 64, 2 * 4096, dtype=torch.bfloat16, scale=0.1)
        s = L.GatedLinearSession(64, 4096, m, device=cuda_device)
        clean = s.forward(x, w)
        x[3, 5], x[7, 0] = float("nan"), float("inf")
        y = s.forward(x, w)
        assert torch.isnan(y[3]).all() and not torch.isfinite(y[7]).any()
        rest = [r for r in range(m) if r not in (3, 7)]
        assert torch.equal(y[rest], clean[rest])
    s = L.GatedLinearSession(8, 16, 4, device=cuda_device)
    w = torch.ones(8, 32, dtype=torch.bfloat16, device=cuda_device)
    none = torch.empty(0, 8, dtype=torch.bfloat16, device=cuda_device)
    assert s.forward(none, w).shape == (0, 16)
    dw, db = torch.full((8, 32), 3.0, device=cuda_device), torch.full((32,), 3.0, device=cuda_device)
    s.backward(torch.empty(0, 16, dtype=torch.bfloat16, device=cuda_device), none, w, torch.empty(0, 32, dtype=torch.bfloat16, device=cuda_device), dx=none, dw=dw, db=db)
    assert (dw == 0).all() and (db == 0).all()
