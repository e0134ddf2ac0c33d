"""The operators of include/gd_train.h on a GPU against plain implementations in 64 bits.

Tolerances are bounds on what the stated arithmetic can do, not observations:
  products   fp32 accumulation in steps of 16 products, each rounding (possibly truncating) once: at most
             (k / 16 + 8) 2^-22 of the sum of magnitudes; a 16-bit result adds half a unit in its last place
  slopes     dz of GELU and SiLU is rounded to 16 bits before the products: half a unit per entry, so that share of the sum of magnitudes
  softmax    exp of a difference d in fp32 is off by |d| 2^-23 for the argument and 2^-21 for the function
  AdamW      fp32 results are the stated sequence of roundings, bit for bit; 8-bit moments land on a neighbour of their value
"""
import math

import numpy as np
import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import training as T

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}     # 2^-p for p significant bits
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}


def _gen(device, seed):
    return torch.Generator(device=device).manual_seed(seed)


def _rand(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen, device=gen.device) * scale).to(dtype)


def _within(got, ref, tol, what):
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = ((got - ref).abs() - tol)
    assert bool((over <= 0).all()), f"{what}: {float(over.max())} past the bound at {int(over.argmax())}"


def _act64(z, name):
    return {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[name](z)


def _slope64(z, name):
    z = z.clone().requires_grad_()
    if name == "none":
        return torch.ones_like(z)
    return torch.autograd.grad(_act64(z, name).sum(), z)[0]


def _pitched(t, pitch, offset):
    """The same matrix with rows `pitch` elements apart, starting `offset` elements into its buffer."""
    r, c = t.shape
    buf = torch.full((r * pitch + offset + 8,), float("nan"), dtype=t.dtype, device=t.device)
    view = buf[offset:offset + r * pitch].view(r, pitch)[:, :c] if r else buf[:0].view(0, c)
    view.copy_(t)
    return view


SHAPES = [(1, 1, 1), (1, 8, 16), (2, 24, 40), (17, 33, 65), (3, 10, 784), (80, 10, 4096), (128, 128, 64), (129, 257, 191), (300, 1000, 500),
          (1, 4096, 4096), (16, 520, 8192), (1000, 7, 96), (513, 520, 1031), (64, 64, 12000)]
LARGE = [(1024, 2048, 1000), (2500, 1544, 520), (4096, 640, 72)]


def _check_forward(device, m, n, k, dtype, act, layout, out_dtype, bias, residual, pre, seed=0, strided=False):
    gen = _gen(device, seed)
    x, w = _rand(gen, m, k, dtype=dtype), _rand(gen, *((k, n) if layout == "in_out" else (n, k)), dtype=dtype, scale=max(k, 1) ** -0.5)
    b = _rand(gen, n, dtype=bias) if bias else None
    r = _rand(gen, m, n, dtype=dtype) if residual else None
    y = torch.full((m, n), float("nan"), dtype=out_dtype, device=device)
    z = torch.full((m, n), float("nan"), dtype=dtype, device=device) if pre else None
    if strided:
        x, w, y = _pitched(x, k + 3, 1), _pitched(w, w.shape[1] + 5, 3), _pitched(y, n + 7, 5)
        r, z = (t if t is None else _pitched(t, n + 9, 1) for t in (r, z))
    s = T.LinearSession(k, n, m, dtype=dtype, activation=act, w_layout=layout, device=device, any_layout=strided)
    got = s.forward(x, w, b, r, out=y, pre=z)
    assert got is y and s.status() == B.GD_OK
    w64 = w.double() if layout == "in_out" else w.double().T
    ref = x.double() @ w64 + (b.double() if bias else 0.0)
    room = (k / 16 + 8) * 2.0 ** -22 * (x.double().abs() @ w64.abs() + (b.double().abs() if bias else 0.0))
    if pre:
        _within(z, ref, room + ref.abs() * HALF_ULP[dtype] + TINY[dtype], "pre")
    ref_y = _act64(ref, act)
    room = 1.2 * room + 2.0 ** -20 * (ref.abs() + 1.0) * (act in ("gelu", "silu")) + (2.0 ** -23 * (ref_y.abs() + r.double().abs()) if residual else 0.0)
    ref_y = ref_y + (r.double() if residual else 0.0)
    _within(y, ref_y, room + ref_y.abs() * HALF_ULP[out_dtype] + TINY[out_dtype], "y")


@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("shape", SHAPES + LARGE, ids=str)
def test_linear_forward(cuda_device, shape, layout):
    _check_forward(cuda_device, *shape, torch.bfloat16, "relu", layout, torch.bfloat16, torch.float32, True, True, seed=sum(shape))


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("out", ["same", "fp32"])
def test_linear_forward_types(cuda_device, act, dtype, out):
    for seed, (m, n, k) in enumerate([(70, 90, 200), (1100, 1300, 264)]):
        out_dtype = dtype if out == "same" else torch.float32
        _check_forward(cuda_device, m, n, k, dtype, act, "in_out", out_dtype, dtype if seed else torch.float32, seed == 0, False, seed=seed)
        _check_forward(cuda_device, m, n, k, dtype, act, "out_in", out_dtype, None, seed == 1, True, seed=seed)


@pytest.mark.parametrize("shape", [(1, 40, 24), (33, 65, 129), (1029, 1031, 257)], ids=str)
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
def test_linear_forward_strided(cuda_device, shape, layout):
    _check_forward(cuda_device, *shape, torch.bfloat16, "silu", layout, torch.bfloat16, torch.float32, True, True, strided=True)


@pytest.mark.parametrize("shape", [(5, 40000, 128), (1, 16384, 8), (17, 20001, 250)], ids=str)
def test_linear_long_contractions(cuda_device, shape):
    """Few results over a long sum, in every direction: the output layer of a small batch backward, a long input, many rows."""
    m, n, k = shape
    _check_backward(cuda_device, m, n, k, torch.bfloat16, "relu", "in_out", torch.float32)
    _check_forward(cuda_device, m, k, n, torch.bfloat16, "gelu", "out_in", torch.bfloat16, torch.float32, True, True)
    _check_backward(cuda_device, n, m, k, torch.bfloat16, "none", "out_in", torch.float32, accumulate=True)


@pytest.mark.parametrize("act", ["none", "silu"])
def test_linear_wide_results(cuda_device, act):
    """fp32 results next to 16-bit pre-activations and residuals, whole tiles and cut ones."""
    for m, n, k in [(2048, 2048, 64), (1100, 1304, 640)]:
        _check_forward(cuda_device, m, n, k, torch.bfloat16, act, "out_in", torch.float32, torch.float32, True, True, seed=m)
        _check_forward(cuda_device, m, n, k, torch.float16, act, "in_out", torch.float32, None, True, False, seed=n)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("shape", [(1, 33, 40), (50, 70, 72), (77, 1001, 136), (1500, 1502, 200), (4100, 2051, 64)], ids=str)
def test_linear_rows_of_four_bytes(cuda_device, shape, dtype):
    """Results, z and residual in rows that start at multiples of 4 bytes only, with odd and even widths: right inside, untouched outside."""
    m, n, k = shape
    gen = _gen(cuda_device, n)
    pitch = (n + 1) // 2 * 2 + (2 if (n + 1) // 2 % 4 == 0 else 0)
    x, w, b = _rand(gen, m, k, dtype=dtype), _rand(gen, k, n, dtype=dtype, scale=k ** -0.5), _rand(gen, n)

    def wide():
        return torch.full((m * pitch + 2,), 77.0, dtype=dtype, device=cuda_device)

    bufs = [wide() for _ in range(3)]
    y, z, r = (t[2:].view(m, pitch)[:, :n] for t in bufs)
    r.copy_(_rand(gen, m, n, dtype=dtype))
    s = T.LinearSession(k, n, m, dtype=dtype, activation="relu", device=cuda_device, any_layout=True)
    s.forward(x, w, b, residual=r, pre=z, out=y)
    z64 = x.double() @ w.double() + b.double()
    room = (k / 16 + 8) * 2.0 ** -22 * (x.double().abs() @ w.double().abs() + b.double().abs())
    _within(z, z64, room + z64.abs() * HALF_ULP[dtype] + TINY[dtype], "z")
    ref = z64.clamp_min(0) + r.double()
    _within(y, ref, room + ref.abs() * HALF_ULP[dtype] + 2.0 ** -23 * r.double().abs() + TINY[dtype], "y")
    for t in bufs:
        assert bool((t[:2] == 77).all()) and bool((t[2:].view(m, pitch)[:, n:] == 77).all())
    kept = y.clone()
    s.forward(x, w, b, residual=r, pre=z, out=r)
    assert torch.equal(r, kept)


def test_linear_residual_in_place(cuda_device):
    gen = _gen(cuda_device, 5)
    x, w, r = _rand(gen, 50, 64, dtype=torch.bfloat16), _rand(gen, 64, 72, dtype=torch.bfloat16, scale=0.1), _rand(gen, 50, 72, dtype=torch.bfloat16)
    s = T.LinearSession(64, 72, 50, device=cuda_device)
    apart = s.forward(x, w, residual=r)
    s.forward(x, w, residual=r, out=r)
    assert torch.equal(apart, r)


def _check_backward(device, m, n, k, dtype, act, layout, dw_dtype, seed=0, strided=False, accumulate=False):
    gen = _gen(device, seed)
    x, w = _rand(gen, m, k, dtype=dtype), _rand(gen, *((k, n) if layout == "in_out" else (n, k)), dtype=dtype, scale=max(k, 1) ** -0.5)
    dy, pre = _rand(gen, m, n, dtype=dtype), _rand(gen, m, n, dtype=dtype)
    dx, dw = torch.full((m, k), float("nan"), dtype=dtype, device=device), torch.full(w.shape, float("nan"), dtype=dw_dtype, device=device)
    db = torch.full((n,), float("nan"), device=device)
    if strided:
        x, dx, dy, pre = _pitched(x, k + 3, 1), _pitched(dx, k + 1, 3), _pitched(dy, n + 5, 1), _pitched(pre, n + 3, 7)
        w, dw = _pitched(w, w.shape[1] + 5, 3), _pitched(dw, w.shape[1] + 3, 1)
    w0 = db0 = 0.0
    if accumulate:
        dw.copy_(_rand(gen, *w.shape)), db.copy_(_rand(gen, n))
        w0, db0 = dw.double().clone(), db.double().clone()
    s = T.LinearSession(k, n, m, dtype=dtype, activation=act, w_layout=layout, device=device, any_layout=strided)
    s.backward(dy, x, w, pre if act != "none" else None, dx=dx, dw=dw, db=db, accumulate=accumulate)
    assert s.status() == B.GD_OK
    dz = dy.double() * _slope64(pre.double(), act)
    soft = act in ("gelu", "silu")
    cut = (HALF_ULP[dtype] * 1.01 if soft else 0.0) + (2.0 ** -20 if soft else 0.0)
    x64, w64 = x.double(), w.double() if layout == "in_out" else w.double().T
    ref = dz @ w64.T
    room = ((n / 16 + 8) * 2.0 ** -22 + cut) * (dz.abs() @ w64.abs().T) + TINY[dtype] * n
    if soft:     # the slope itself is good to a few units of 2^-21 even where it is near 0
        room = room + 2.0 ** -19 * (dy.double().abs() @ w64.abs().T)
    _within(dx, ref, room + ref.abs() * HALF_ULP[dtype] + TINY[dtype], "dx")
    ref, size = x64.T @ dz, x64.abs().T @ dz.abs()
    room = ((m / 16 + 8) * 2.0 ** -22 + cut) * size + TINY[dtype] * x64.abs().sum(0)[:, None]
    if soft:
        room = room + 2.0 ** -19 * (x64.abs().T @ dy.double().abs())
    if layout == "out_in":
        ref, room = ref.T, room.T
    ref = ref + w0
    _within(dw, ref, room + ref.abs() * HALF_ULP[dw_dtype] + 2.0 ** -24 * (ref - w0).abs() + TINY[dw_dtype], "dw")
    ref = dz.sum(0)
    room = (m / 256 + 48) * 2.0 ** -23 * dz.abs().sum(0) + (2.0 ** -19 * dy.double().abs().sum(0) if soft else 0.0)
    _within(db, ref + db0, room + (ref + db0).abs() * 2.0 ** -23 + TINY[torch.float32], "db")


@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("shape", SHAPES + LARGE, ids=str)
def test_linear_backward(cuda_device, shape, layout):
    _check_backward(cuda_device, *shape, torch.bfloat16, "relu", layout, torch.float32, seed=sum(shape))


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
def test_linear_backward_types(cuda_device, act, dtype):
    for seed, (m, n, k) in enumerate([(70, 90, 200), (1100, 1304, 264)]):
        _check_backward(cuda_device, m, n, k, dtype, act, "in_out", dtype, seed=seed)
        _check_backward(cuda_device, m, n, k, dtype, act, "out_in", torch.float32, seed=seed)


@pytest.mark.parametrize("layout", ["in_out", "out_in"])
def test_linear_backward_strided_and_accumulated(cuda_device, layout):
    for shape in [(1, 40, 24), (33, 65, 129), (1029, 1031, 257)]:
        _check_backward(cuda_device, *shape, torch.bfloat16, "gelu", layout, torch.float32, strided=True)
        _check_backward(cuda_device, *shape, torch.bfloat16, "relu", layout, torch.float32, accumulate=True)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("n", [1024, 1025, 1031, 1540, 3347])
def test_linear_backward_wide_ragged_rows(cuda_device, n, act):
    """Rows of dy and pre that start at every 16-bit place of an aligned vector, their ends inside one."""
    _check_backward(cuda_device, 37, n, 24, torch.bfloat16, act, "in_out", torch.float32, seed=n, strided=True)
    _check_backward(cuda_device, 300, n, 40, torch.float16, act, "out_in", torch.float16, seed=n)


@pytest.mark.parametrize("shape", [(4000, 1000, 1500), (80, 10, 4096), (300, 200, 100), (20000, 24, 600), (500, 17000, 72)], ids=str)
def test_linear_backward_products_side_by_side(cuda_device, shape):
    """Both gradients from one call, time and again with changing inputs: the bits of a call for each alone, and of the first time."""
    m, n, k = shape
    gen = _gen(cuda_device, 13)
    w = _rand(gen, k, n, dtype=torch.bfloat16, scale=0.05)
    s = T.LinearSession(k, n, m, activation="relu", device=cuda_device, any_layout=True)
    sets = [(_rand(gen, m, n, dtype=torch.bfloat16), _rand(gen, m, k, dtype=torch.bfloat16), _rand(gen, m, n, dtype=torch.bfloat16)) for _ in range(2)]
    alone, first = [], [None, None]
    for dy, x, pre in sets:
        dw, db = torch.empty(k, n, device=cuda_device), torch.empty(n, device=cuda_device)
        s.backward(dy, x, w, pre, dw=dw, db=db)
        alone.append((dw, db))
    for i in range(20):
        dy, x, pre = sets[i & 1]
        dx = torch.full((m, k), float("nan"), dtype=torch.bfloat16, device=cuda_device)
        dw, db = torch.full((k, n), float("nan"), device=cuda_device), torch.full((n,), float("nan"), device=cuda_device)
        s.backward(dy, x, w, pre, dx=dx, dw=dw, db=db)
        kept = (dx + 0, dw + 0)                          # (read by the kernel behind the call: it must find both complete)
        assert torch.equal(dw, alone[i & 1][0]) and torch.equal(db, alone[i & 1][1])
        if first[i & 1] is None:
            first[i & 1] = dx
            plain = (dy.float() * (pre > 0)) @ w.float().T
            assert float((dx.float() - plain).abs().max()) <= 2.0 ** -7 * float(plain.abs().max())
        assert torch.equal(dx, first[i & 1]) and torch.equal(kept[0], dx) and torch.equal(kept[1], dw)
    assert s.status() == B.GD_OK


@pytest.mark.parametrize("shape", [(4000, 1000, 1500), (80, 10, 4096)], ids=str)
def test_linear_backward_in_a_graph(cuda_device, shape):
    """A captured backward call, replayed over new inputs, gives the bits of the call itself."""
    m, n, k = shape
    gen = _gen(cuda_device, 14)
    w = _rand(gen, k, n, dtype=torch.bfloat16, scale=0.05)
    s = T.LinearSession(k, n, m, activation="relu", device=cuda_device, any_layout=True)
    dy, x, pre = (_rand(gen, m, c, dtype=torch.bfloat16) for c in (n, k, n))
    dx, dw, db = torch.empty_like(x), torch.empty(k, n, device=cuda_device), torch.empty(n, device=cuda_device)
    s.backward(dy, x, w, pre, dx=dx, dw=dw, db=db)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.backward(dy, x, w, pre, dx=dx, dw=dw, db=db)
    for seed in range(4):
        for t in (dy, x, pre):
            t.copy_(_rand(gen, *t.shape, dtype=torch.bfloat16))
        graph.replay()
        replayed = [t + 0 for t in (dx, dw, db)]
        s.backward(dy, x, w, pre, dx=dx, dw=dw, db=db)
        assert all(torch.equal(a, b) for a, b in zip(replayed, (dx, dw, db)))
    assert s.status() == B.GD_OK


def test_linear_empty_sizes(cuda_device):
    """No rows, no inputs, no outputs: sums over nothing are 0, and nothing else is touched."""
    dev, dt = cuda_device, torch.bfloat16
    s = T.LinearSession(0, 24, 5, activation="relu", device=dev)
    bias = torch.linspace(-1, 1, 24, device=dev)
    y = s.forward(torch.empty(5, 0, dtype=dt, device=dev), torch.empty(0, 24, dtype=dt, device=dev), bias)
    assert torch.equal(y, torch.relu(bias).to(dt).expand(5, 24))
    s = T.LinearSession(16, 24, 5, device=dev)
    x, w, dy = torch.empty(0, 16, dtype=dt, device=dev), torch.ones(16, 24, dtype=dt, device=dev), torch.empty(0, 24, dtype=dt, device=dev)
    assert s.forward(x, w).shape == (0, 24)
    dw, db = torch.full((16, 24), 3.0, device=dev), torch.full((24,), 3.0, device=dev)
    s.backward(dy, x, w, dw=dw, db=db, accumulate=True)
    assert bool((dw == 3).all()) and bool((db == 3).all())
    s.backward(dy, x, w, dx=torch.empty_like(x), dw=dw, db=db)
    assert bool((dw == 0).all()) and bool((db == 0).all())
    s = T.LinearSession(16, 0, 5, device=dev)
    dx = torch.full((5, 16), 3.0, dtype=dt, device=dev)
    s.backward(torch.empty(5, 0, dtype=dt, device=dev), torch.ones(5, 16, dtype=dt, device=dev), torch.empty(16, 0, dtype=dt, device=dev), dx=dx)
    assert bool((dx == 0).all()) and s.status() == B.GD_OK


def test_linear_special_values(cuda_device):
    """Infinities and NaN reach the rows they belong to and no others; padding never leaks into a result."""
    dev, dt = cuda_device, torch.bfloat16
    x = torch.ones(40, 100, dtype=dt, device=dev)
    w = torch.ones(100, 30, dtype=dt, device=dev)
    x[3, 7], x[5, 99], x[39, 0] = float("inf"), float("nan"), -float("inf")
    s = T.LinearSession(100, 30, 40, device=dev)
    y = s.forward(x, w).double()
    plain = x.double() @ w.double()
    assert torch.equal(torch.isnan(y), torch.isnan(plain)) and torch.equal(y.nan_to_num(7.0), plain.nan_to_num(7.0))


def test_linear_gradient_against_differences(cuda_device):
    """The gradients of L = sum(y * c) against central differences of the 64-bit forward formula."""
    dev, dt, (m, n, k) = cuda_device, torch.float16, (6, 9, 11)
    gen = _gen(dev, 2)
    x, w, c = _rand(gen, m, k, dtype=dt), _rand(gen, k, n, dtype=dt, scale=0.4), _rand(gen, m, n, dtype=dt)
    for act in ("gelu", "silu"):
        s = T.LinearSession(k, n, m, dtype=dt, activation=act, device=dev, any_layout=True)
        b, pre = _rand(gen, n), torch.empty(m, n, dtype=dt, device=dev)
        s.forward(x, w, b, pre=pre)
        dx, dw, db = torch.empty_like(x), torch.empty(k, n, device=dev), torch.empty(n, device=dev)
        s.backward(c, x, w, pre, dx=dx, dw=dw, db=db)

        def loss(x, w, b):
            return float((_act64(x @ w + b, act) * c.double()).sum())

        base = [x.double(), w.double(), b.double()]
        for which, got in enumerate((dx, dw, db)):
            flat = got.double().reshape(-1)
            for at in range(0, flat.numel(), 5):
                sides = []
                for h in (1e-4, -1e-4):
                    moved = [t.clone() for t in base]
                    moved[which].view(-1)[at] += h
                    sides.append(loss(*moved))
                # pre is held in 16 bits (2^-11 of |z| <= 8, slope's slope <= 1.2), dz in 16 bits; sums of at most 11 terms of size <= 4
                assert abs((sides[0] - sides[1]) / 2e-4 - float(flat[at])) <= 11 * 4 * (2.0 ** -8 * 1.2 + 2.0 ** -11) * 0.25 + 1e-6


def test_linear_repeats_bit_for_bit(cuda_device):
    gen = _gen(cuda_device, 9)
    x, w = _rand(gen, 48, 6000, dtype=torch.bfloat16), _rand(gen, 6000, 200, dtype=torch.bfloat16)
    dy = _rand(gen, 48, 200, dtype=torch.bfloat16)
    s = T.LinearSession(6000, 200, 48, device=cuda_device)
    outs = []
    for _ in range(3):
        dx, dw, db = torch.empty_like(x), torch.empty(6000, 200, device=cuda_device), torch.empty(200, device=cuda_device)
        y = s.forward(x, w, out=torch.empty(48, 200, device=cuda_device))
        s.backward(dy, x, w, dx=dx, dw=dw, db=db)
        outs.append((y, dx, dw, db))
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))


@pytest.mark.parametrize("shape", [(4000, 1500, 1000), (8192, 1280, 128), (6000, 1000, 64)], ids=str)
def test_linear_many_tiles_repeat_bit_for_bit(cuda_device, shape):
    """Many tiles per pair of CTAs with little to sum: what leaves one tile must not meet what the next one writes."""
    m, n, k = shape
    gen = _gen(cuda_device, 12)
    for layout in ("in_out", "out_in"):
        x, w = _rand(gen, m, k, dtype=torch.bfloat16), _rand(gen, *((k, n) if layout == "in_out" else (n, k)), dtype=torch.bfloat16)
        r = _rand(gen, m, n, dtype=torch.bfloat16)
        s = T.LinearSession(k, n, m, w_layout=layout, device=cuda_device, any_layout=True)
        for residual in (None, r):
            first = s.forward(x, w, residual=residual)
            plain = x.float() @ (w if layout == "in_out" else w.t()).float() + (0 if residual is None else residual.float())
            assert float((first.float() - plain).abs().max()) <= 2.0 ** -7 * float(plain.abs().max())
            for _ in range(10):
                assert torch.equal(first, s.forward(x, w, residual=residual, out=torch.empty_like(first)))


def test_linear_on_another_stream(cuda_device):
    gen = _gen(cuda_device, 4)
    x, w = _rand(gen, 33, 72, dtype=torch.bfloat16), _rand(gen, 72, 40, dtype=torch.bfloat16)
    s = T.LinearSession(72, 40, 33, device=cuda_device)
    here = s.forward(x, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = s.forward(x, w, out=torch.empty_like(here), stream=side)
    side.synchronize()
    assert torch.equal(here, there)


def test_linear_refusals(cuda_device):
    dev, dt = cuda_device, torch.bfloat16
    with pytest.raises(ValueError):
        T.LinearSession(8, 8, 8, dtype=torch.float32, device=dev)
    with pytest.raises(ValueError):
        T.LinearSession(8, 8, 8, activation="tanh", device=dev)
    with pytest.raises(RuntimeError):
        T.LinearSession(8, 8, 8, device="cpu")
    s = T.LinearSession(16, 24, 4, activation="gelu", device=dev)
    x, w = torch.ones(4, 16, dtype=dt, device=dev), torch.ones(16, 24, dtype=dt, device=dev)
    with pytest.raises(ValueError):
        s.forward(torch.ones(5, 16, dtype=dt, device=dev), w)                     # more rows than planned
    with pytest.raises(ValueError):
        s.forward(x.half(), w)
    with pytest.raises(ValueError):
        s.forward(x, w.T.contiguous())
    with pytest.raises(ValueError):
        s.forward(x, torch.ones(24, 16, dtype=dt, device=dev).T)                  # rows not contiguous
    with pytest.raises(ValueError):
        s.forward(x, w, bias=torch.ones(23, device=dev))
    with pytest.raises(ValueError):
        s.backward(torch.ones(4, 24, dtype=dt, device=dev), x, w)                 # no pre-activation
    narrow = T.LinearSession(512, 8, 4, device=dev)
    with pytest.raises(B.GdError) as err:                                         # a ragged operand and no room to lay it out
        narrow.forward(_pitched(torch.ones(4, 512, dtype=dt, device=dev), 513, 0), torch.ones(512, 8, dtype=dt, device=dev))
    assert err.value.code == B.GD_ERR_WORKSPACE
    with pytest.raises(B.GdError):                                                # half-precision gradients cannot accumulate
        s.backward(torch.ones(4, 24, dtype=dt, device=dev), x, w, torch.ones(4, 24, dtype=dt, device=dev), dw=torch.ones(16, 24, dtype=dt, device=dev),
                   accumulate=True)


# ------------------------------------------------------------------------------------------------------------ cross-entropy

def _check_xent(device, logits, targets, scale=1.0, ignore=-100, in_place=False, scale_dev=None, grad=None):
    rows, classes = logits.shape
    z = logits.double()
    live = targets != ignore
    t = torch.where(live, targets, torch.zeros_like(targets)).long()
    lse = torch.logsumexp(z, 1)
    ref_loss = torch.where(live, lse - z.gather(1, t[:, None])[:, 0], torch.zeros_like(lse))
    p = torch.softmax(z, 1)
    hot = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    full = scale * (1.0 if scale_dev is None else float(scale_dev))
    ref = (p - hot) * full * live[:, None]
    loss, out_lse = torch.full((rows,), float("nan"), device=device), torch.full((rows,), float("nan"), device=device)
    grad = logits if in_place else torch.full_like(logits, float("nan")) if grad is None else grad
    dtype = logits.dtype
    T.cross_entropy(logits, targets, loss=loss, lse=out_lse, grad=grad, grad_scale=scale, grad_scale_dev=scale_dev, ignore_index=ignore)
    top = z.max(1).values
    room = 2.0 ** -22 * (top.abs() + (lse - top) + ref_loss.abs()) + 2.0 ** -20
    _within(out_lse, lse, room, "lse")
    _within(loss, ref_loss, room, "loss")
    dist = (top[:, None] - z).clamp(max=200.0)
    room = (p * (2.0 ** -19 + dist * 2.0 ** -22) + 2.0 ** -23 * hot) * abs(full) + 2.0 ** -126 * abs(full)
    _within(grad, ref, room + ref.abs() * HALF_ULP[dtype] + TINY[dtype], "grad")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", [(1, 1), (5, 2), (80, 10), (33, 17), (7, 65), (9, 300), (4, 1000), (3, 1025), (2, 4099), (300, 2048), (1, 85000), (20, 50257),
                                   (2, 200001), (310, 40001), (300, 85000), (170, 60003), (900, 33000)], ids=str)
def test_cross_entropy(cuda_device, shape, dtype):
    gen = _gen(cuda_device, sum(shape))
    logits = _rand(gen, *shape, dtype=dtype, scale=3.0)
    targets = torch.randint(shape[1], (shape[0],), generator=gen, device=cuda_device)
    targets[::3] = -100 if shape[0] > 1 else targets[::3]
    _check_xent(cuda_device, logits, targets)
    _check_xent(cuda_device, logits, targets.int(), scale=-0.25, scale_dev=torch.tensor([3.0], device=cuda_device))
    _check_xent(cuda_device, logits.clone(), targets, in_place=True)


def _masked_rows(dev, classes, dtype):
    low = torch.finfo(dtype).min
    x = _rand(_gen(dev, 1), 12, classes, dtype=dtype)
    t = torch.zeros(12, dtype=torch.int64, device=dev)
    x[0, 1:] = -float("inf")                       # one class left, the target: loss 0
    x[1, 1:] = low
    x[2] = low                                     # every class at the lowest value: uniform
    x[3, : classes // 2] = -float("inf")
    t[3] = classes - 1
    x[4] = -float("inf")                           # nothing left, and no target
    x[5] = float("nan")
    t[4] = t[5] = -100
    x[6] = -float("inf")                           # nothing left, but a target
    x[7, classes - 1] = float("nan")
    x[8, classes // 2] = float("inf")
    t[9], t[10] = classes, -1                      # targets out of range
    return x, t


def _check_masked_rows(classes, loss, lse, grad):
    dev = loss.device
    assert loss[0] == 0 and loss[1] == 0 and bool((grad[:2] == 0).all())
    assert abs(float(loss[2]) - math.log(classes)) < 1e-5
    want = torch.full((classes,), 1.0 / classes, dtype=torch.float64, device=dev)
    want[0] -= 1.0
    assert bool(((grad[2].double() - want).abs() <= 2.0 ** -8 * want.abs()).all())
    assert bool((grad[3, : classes // 2] == 0).all()) and torch.isfinite(lse[3])
    assert bool((loss[4:6] == 0).all()) and bool((grad[4:6] == 0).all()) and lse[4] == -float("inf")
    for row in (6, 7, 8, 9, 10):
        assert torch.isnan(loss[row]) and bool(torch.isnan(grad[row]).all()), row
    assert torch.isfinite(loss[11]) and bool(torch.isfinite(grad[11]).all())


@pytest.mark.parametrize("classes", [10, 700, 5000, 700003])
def test_cross_entropy_masks(cuda_device, classes):
    """Masked classes (-inf, the type's lowest value), rows that keep one class or none, infinities and NaN, bad targets."""
    for dtype in (torch.float32, torch.bfloat16):
        x, t = _masked_rows(cuda_device, classes, dtype)
        loss, lse, grad = torch.empty(12, device=cuda_device), torch.empty(12, device=cuda_device), torch.empty_like(x)
        T.cross_entropy(x, t, loss=loss, lse=lse, grad=grad)
        _check_masked_rows(classes, loss, lse, grad)
        assert abs(float(lse[3]) - float(torch.logsumexp(x[3].double(), 0))) < 1e-5


@pytest.mark.parametrize("classes", [33000, 36001, 60008])
def test_cross_entropy_masks_in_many_rows(cuda_device, classes):
    """The same rows thirty times over: what one row leaves behind must not reach the next."""
    for dtype in (torch.float32, torch.bfloat16):
        x, t = _masked_rows(cuda_device, classes, dtype)
        x, t = x.repeat(30, 1), t.repeat(30)
        loss, lse, grad = torch.empty(360, device=cuda_device), torch.empty(360, device=cuda_device), torch.empty_like(x)
        T.cross_entropy(x, t, loss=loss, lse=lse, grad=grad)
        for at in range(0, 360, 12):
            _check_masked_rows(classes, loss[at:at + 12], lse[at:at + 12], grad[at:at + 12])


def test_cross_entropy_strides(cuda_device):
    gen = _gen(cuda_device, 3)
    for classes, pitch, offset in [(10, 13, 1), (3000, 3001, 3), (9000, 9008, 8), (6001, 6008, 0)]:
        logits = _pitched(_rand(gen, 9, classes, dtype=torch.bfloat16, scale=2.0), pitch, offset)
        targets = torch.randint(classes, (9,), generator=gen, device=cuda_device)
        _check_xent(cuda_device, logits, targets)                                                            # ends of rows differ in alignment
        _check_xent(cuda_device, logits, targets, grad=_pitched(torch.zeros(9, classes, dtype=torch.bfloat16, device=cuda_device), pitch + 2, 5))


def test_cross_entropy_gradient_against_differences(cuda_device):
    z = torch.randn(3, 40, dtype=torch.float64, generator=torch.Generator().manual_seed(0)).float()
    t = torch.tensor([0, 7, 39])
    grad = torch.empty(3, 40, device=cuda_device)
    T.cross_entropy(z.to(cuda_device), t.to(cuda_device), grad=grad)
    loss = lambda a: float((torch.logsumexp(a, 1) - a.gather(1, t[:, None])[:, 0]).sum())  # noqa: E731
    for i in range(3):
        for j in range(0, 40, 3):
            sides = []
            for h in (1e-5, -1e-5):
                a = z.double().clone()
                a[i, j] += h
                sides.append(loss(a))
            assert abs((sides[0] - sides[1]) / 2e-5 - float(grad[i, j])) < 1e-6


def test_cross_entropy_refusals(cuda_device):
    x, t = torch.zeros(4, 8, device=cuda_device), torch.zeros(4, dtype=torch.int64, device=cuda_device)
    for bad in (dict(loss=torch.zeros(3, device=cuda_device)), dict(grad=torch.zeros(4, 8, dtype=torch.bfloat16, device=cuda_device)),
                dict(loss=torch.zeros(4, device=cuda_device), grad_scale_dev=torch.zeros(2, device=cuda_device))):
        with pytest.raises(ValueError):
            T.cross_entropy(x, t, **bad)
    with pytest.raises(ValueError):
        T.cross_entropy(x, t.short(), loss=torch.zeros(4, device=cuda_device))
    with pytest.raises(ValueError):
        T.cross_entropy(x.T, t, loss=torch.zeros(8, device=cuda_device))
    with pytest.raises(B.GdError):
        T.cross_entropy(x, t)                                                     # nothing to compute
    with pytest.raises(B.GdError):
        T.cross_entropy(x[:, :0], t, loss=torch.zeros(4, device=cuda_device))     # no classes
    T.cross_entropy(x[:0], t[:0], loss=torch.zeros(0, device=cuda_device))        # no rows: nothing to do


# ------------------------------------------------------------------------------------------------------------ AdamW

HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)


def _rounded_step(p, g, m, v, step, decay, scale, h):
    """The header's sequence, each operation one fp32 rounding (numpy on the host rounds every operation)."""
    f = np.float32
    g = g * f(scale)
    m = m * f(h["beta1"]) + g * f(1 - h["beta1"])
    v = v * f(h["beta2"]) + (g * f(1 - h["beta2"])) * g
    root = np.sqrt(v)
    with np.errstate(all="ignore"):
        d = root * f(1 / math.sqrt(1 - h["beta2"] ** step)) + f(h["eps"])
        p = p * f(1 - h["lr"] * decay) - (m / d) * f(h["lr"] / (1 - h["beta1"] ** step))
    return p, m, v, root


def _mix(x):
    x = x.astype(np.uint64) & 0xFFFFFFFF
    x ^= x >> 16
    x = x * 0x7FEB352D & 0xFFFFFFFF
    x ^= x >> 15
    x = x * 0x846CA68B & 0xFFFFFFFF
    return x ^ x >> 16


FP8 = np.array([0.0 if c == 0 else (c % 8) / 8 * 2.0 ** -6 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7) for c in range(127)])


def _hold(x, random16, positive):
    """Codes and scales of a moment by the header's definition, with real-number neighbours instead of bits."""
    n = x.size
    code, scales = np.zeros(n, np.uint8), np.zeros(-(-n // 128), np.float32)
    for b in range(scales.size):
        part = slice(b * 128, min(n, b * 128 + 128))
        size = np.abs(x[part]).astype(np.float64)
        top = size.max()
        unit = 2.0 ** max(math.floor(math.log2(top)) - 7, -126) if top > 0 else 2.0 ** -126
        scales[b] = unit
        y = size / unit
        low = np.searchsorted(FP8, y, side="right") - 1
        way = np.floor((y - FP8[low]) / (FP8[low + 1] - FP8[low]) * 2 ** 20)          # 2^-20 ths of the way, as fp32 holds it
        c = low + (way + random16[part] * 16.0 >= 2 ** 20)
        if positive:
            c = np.where(size > 0, np.maximum(c, 1), c)
        code[part] = c + 128 * np.signbit(x[part])
    return code, scales


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", [torch.float32, torch.bfloat16, torch.float16], ids=["p32", "pbf16", "pfp16"])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16, torch.float16], ids=["g32", "gbf16", "gfp16"])
def test_adamw_is_the_stated_sequence(cuda_device, bits, param, grad):
    """Three steps over tensors of all kinds of lengths, pieces of flat vectors, against the host, bit for bit."""
    dev = cuda_device
    sizes = [1, 3, 127, 128, 129, 0, 1000, 4096, 5001, 20000]
    total = sum(sizes)
    gen = _gen(dev, 7)
    params, grads = _rand(gen, total, dtype=param, scale=0.05), None
    copies = torch.empty(total, dtype=torch.bfloat16, device=dev)
    cut = lambda t: list(torch.split(t, sizes))  # noqa: E731
    grads = torch.empty(total, dtype=grad, device=dev)
    decay = [0.1 if i % 2 else 0.0 for i in range(len(sizes))]
    s = T.AdamWSession(cut(params), cut(grads), copies=cut(copies), weight_decay=decay, state_bits=bits)
    p_host = [t.float().cpu().numpy() for t in s.params]
    m_host = [np.zeros(n, np.float32) for n in sizes]
    v_host = [np.zeros(n, np.float32) for n in sizes]
    scale_dev = torch.tensor([0.5], device=dev)
    for step in (1, 2, 3):
        grads.copy_(_rand(gen, total, scale=1e-2))
        g_host = [t.float().cpu().numpy() for t in s.grads]
        s.step(step=step, grad_scale=2.0, grad_scale_dev=scale_dev, seed=1000 + step, **HYPER)
        for i, n in enumerate(sizes):
            p, m, v, root = _rounded_step(p_host[i], g_host[i], m_host[i], v_host[i], step, decay[i], 1.0, HYPER)
            got = s.params[i].cpu()
            want = torch.from_numpy(p).to(param)
            assert torch.equal(got, want), (step, i, "param")
            assert torch.equal(s.copies[i].cpu(), torch.from_numpy(p).bfloat16()), (step, i, "copy")
            p_host[i] = want.float().numpy()
            if bits == 32:
                assert torch.equal(s.m[i].cpu(), torch.from_numpy(m)) and torch.equal(s.v[i].cpu(), torch.from_numpy(v)), (step, i)
                m_host[i], v_host[i] = m, v
                continue
            if n == 0:
                continue
            h = _mix(np.arange(n, dtype=np.uint64) * 0x9E3779B9 + (1000 + step + i * 0x85EBCA77))
            for name, x, rnd, positive in (("m", m, h >> 16, False), ("v", root, h & 0xFFFF, True)):
                code, scales = _hold(x, rnd.astype(np.float64), positive)
                held, unit = getattr(s, name)[i].view(torch.uint8).cpu().numpy(), getattr(s, name + "_scale")[i].cpu().numpy()
                assert np.array_equal(unit, scales), (step, i, name, "scale")
                assert np.array_equal(held, code), (step, i, name, int((held != code).sum()))
                back = (s.__dict__[name][i].float().cpu().numpy() * np.repeat(unit, 128)[:n])
                if name == "m":
                    m_host[i] = back
                else:
                    v_host[i] = back * back


def test_adamw_against_64_bits(cuda_device):
    """One step against the textbook form in 64 bits: fp32 moments and parameters within a few roundings of it."""
    gen, n = _gen(cuda_device, 3), 100_003
    p, g, m = (_rand(gen, n, scale=s) for s in (0.1, 1e-3, 1e-3))
    v = torch.rand(n, generator=gen, device=cuda_device) * 1e-6
    p0, m0, v0 = p.double(), m.double(), v.double()
    s = T.AdamWSession([p], [g], [m], [v], weight_decay=0.01)
    s.step(step=10, **HYPER)
    m1 = 0.9 * m0 + 0.1 * g.double()
    v1 = 0.999 * v0 + 0.001 * g.double() ** 2
    q = p0 - 1e-3 * ((m1 / (1 - 0.9 ** 10)) / ((v1 / (1 - 0.999 ** 10)).sqrt() + 1e-8) + 0.01 * p0)
    _within(m, m1, 2.0 ** -22 * (m0.abs() + g.double().abs()), "m")
    _within(v, v1, 2.0 ** -21 * v1, "v")
    _within(p, q, 2.0 ** -22 * p0.abs() + 2.0 ** -20 * (q - p0).abs() + 2.0 ** -20 * 1e-3 * (m0.abs() + g.double().abs()) / v1.sqrt(), "p")


def test_adamw_unaligned_pieces_give_the_same_bits(cuda_device):
    for bits in (32, 8):
        gen = _gen(cuda_device, 1)
        n = 9000
        p, g = _rand(gen, n), _rand(gen, n)
        results = []
        for offset in (0, 1, 3):
            bp, bg = torch.zeros(n + 8, device=cuda_device), torch.zeros(n + 8, device=cuda_device)
            bp[offset:offset + n], bg[offset:offset + n] = p, g
            s = T.AdamWSession([bp[offset:offset + n]], [bg[offset:offset + n]], state_bits=bits)
            for step in (1, 2):
                s.step(step=step, seed=step, **HYPER)
            assert bool((bp[:offset] == 0).all()) and bool((bp[offset + n:] == 0).all())
            results.append((s.params[0].clone(), s.m[0].view(torch.uint8).clone(), s.v[0].view(torch.uint8).clone()))
        for other in results[1:]:
            assert all(torch.equal(a, b) for a, b in zip(results[0], other))


def test_adamw_more_tensors_than_one_table_holds(cuda_device):
    gen = _gen(cuda_device, 8)
    sizes = [int(x) for x in torch.randint(1, 600, (950,), generator=gen, device=cuda_device).tolist()]
    flat, grads = _rand(gen, sum(sizes)), _rand(gen, sum(sizes))
    one = flat.clone()
    s = T.AdamWSession(list(torch.split(flat, sizes)), list(torch.split(grads, sizes)), weight_decay=0.1)
    s.step(step=1, **HYPER)
    T.AdamWSession([one], [grads], weight_decay=0.1).step(step=1, **HYPER)
    assert torch.equal(flat, one)


def test_adamw_8_bit_moments_follow_on_average(cuda_device):
    """With a constant gradient the root of the second moment approaches |g| although each step moves it by far less than a code."""
    n = 1 << 16
    p, g = torch.zeros(n, device=cuda_device), torch.full((n,), 0.01, device=cuda_device)
    s = T.AdamWSession([p], [g], state_bits=8)
    for step in range(1, 1001):
        s.step(step=step, seed=step, **HYPER)
    root = s.v[0].float() * s.v_scale[0].repeat_interleave(128)
    want = 0.01 * math.sqrt(1 - 0.999 ** 1000)
    # rounding up or down at random is right on average for the root; its spread adds at most a step's worth (1/8) to the mean square
    assert abs(float(root.mean()) / want - 1) < 0.06


def test_adamw_not_finite_moments_are_held_as_nan(cuda_device):
    g = torch.ones(300, device=cuda_device)
    g[5], g[200] = float("inf"), float("nan")
    s = T.AdamWSession([torch.zeros(300, device=cuda_device)], [g], state_bits=8)
    s.step(step=1, seed=3, **HYPER)
    for held in (s.m[0].float(), s.v[0].float()):
        assert torch.isnan(held[5]) and torch.isnan(held[200]) and int(torch.isnan(held).sum()) == 2


def test_adamw_refusals(cuda_device):
    p = torch.zeros(300, device=cuda_device)
    with pytest.raises(ValueError):
        T.AdamWSession([p], [torch.zeros(299, device=cuda_device)])
    with pytest.raises(ValueError):
        T.AdamWSession([p], [p.double()])
    with pytest.raises(ValueError):
        T.AdamWSession([p], [p], state_bits=4)
    with pytest.raises(ValueError):
        T.AdamWSession([p], [p], m=[p])
    with pytest.raises(RuntimeError):
        T.AdamWSession([torch.zeros(3)], [torch.zeros(3)])
    s = T.AdamWSession([p], [p.clone()])
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(lr=float("nan"))):
        with pytest.raises(B.GdError) as err:
            s.step(**{**dict(step=1), **HYPER, **bad})
        assert err.value.code == B.GD_ERR_INVALID_ARG
