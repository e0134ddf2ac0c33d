"""Embedding, layer norm and recurrence of include/gd_layers.h on a GPU against plain implementations in 64 bits.

Tolerances are bounds on what the stated arithmetic can do, not observations; u = 2^-24 is half a step of fp32:
  embedding   one product (u) and the rounding of the result; a sum of c rows takes c additions at most
  norm        a sum over a row passes through at most DEPTH additions; the mean is off by that, the squares about it by as much again
  recurrence  f and 1 - f are off by ETA = 2^-21 + |gate| 2^-23 of themselves (two approximations of 2^-22 and the exponent's argument); a
              state carries the error of the one before, times f, and adds (ETA + 6 u) of the magnitudes that meet in it
"""
import numpy as np
import pytest
import torch

from paper_1704_05021_b200 import layers as L

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


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
    """A matrix with rows `pitch` elements apart that starts `offset` elements into a buffer of a number nobody computes."""

    def __init__(self, rows, cols, dtype, device, strided, fill=-77.0):
        pitch, self.offset = (cols + 5, 3) if strided else (cols, 0)
        self.buf = torch.full((rows * pitch + 16,), fill, dtype=dtype, device=device)
        self.t = self.buf[self.offset:self.offset + rows * pitch].view(rows, pitch)[:, :cols]
        self.inside = torch.zeros_like(self.buf, dtype=torch.bool)
        self.inside[self.offset:self.offset + rows * pitch].view(rows, pitch)[:, :cols] = True
        self.fill = fill

    def set(self, x):
        self.t.copy_(x)
        return self.t

    def check_around(self):
        assert bool((self.buf[~self.inside] == self.fill).all()), "written outside the matrix"


def _inset(x, strided):
    return Inset(*x.shape, x.dtype, x.device, strided).set(x)


# ------------------------------------------------------------------------------------------------------------- embedding

@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("table_dtype, out_dtype", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.float32, torch.float16),
                                                    (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
                                                    (torch.float16, torch.float32)])
@pytest.mark.parametrize("tokens, vocab, width", [(1, 1, 1), (7, 5, 3), (33, 100, 500), (1000, 37, 64), (5, 3, 4097), (4000, 850, 500)])
def test_embedding_lookup(cuda_device, tokens, vocab, width, table_dtype, out_dtype, strided):
    gen = _gen(cuda_device, tokens + width)
    table = _inset(_rand(gen, vocab, width, dtype=table_dtype), strided)
    ids = torch.randint(vocab, (tokens,), generator=gen, device=cuda_device)
    if tokens > 6:
        ids[2], ids[4] = -100, vocab - 1
    out = Inset(tokens, width, out_dtype, cuda_device, strided)
    scale = float(np.float32(width ** 0.5))
    got = L.EmbeddingSession(vocab, width, tokens, device=cuda_device).forward(table, ids, out=out.t, scale=scale)
    assert got is out.t
    live = ids >= 0
    ref = torch.where(live[:, None], table.double()[ids.clamp(min=0)] * scale, torch.zeros((), dtype=torch.float64, device=cuda_device))
    _within(out.t, ref, ref.abs() * (U + HALF_ULP[out_dtype]) + TINY[out_dtype], "y")
    out.check_around()


def test_embedding_ids_outside_the_table(cuda_device):
    """NaN rows, no gradient and no access outside; ignore_index comes first, wherever it lies; 32-bit ids."""
    table = torch.ones(4, 8, device=cuda_device)
    s = L.EmbeddingSession(4, 8, 8, device=cuda_device)
    ids = torch.tensor([0, 3, 4, -1, 2 ** 31 - 1, -2 ** 31, 1, -100], dtype=torch.int32, device=cuda_device)
    y = s.forward(table, ids, ignore_index=1)
    assert torch.isnan(y[2:6]).all() and torch.isnan(y[7]).all() and (y[:2] == 1).all() and (y[6] == 0).all()
    dtable = torch.full((4, 8), 7.0, device=cuda_device)
    s.backward(torch.ones(8, 8, device=cuda_device), ids, dtable, ignore_index=1)
    assert dtable.sum(1).tolist() == [8.0, 0.0, 0.0, 8.0]
    big = torch.tensor([2 ** 40, -2 ** 40, 2 ** 32, 0], dtype=torch.int64, device=cuda_device)
    y = s.forward(table, big)
    assert torch.isnan(y[:3]).all() and (y[3] == 1).all()
    s.backward(torch.ones(4, 8, device=cuda_device), big, dtable)
    assert dtable.sum(1).tolist() == [8.0, 0.0, 0.0, 0.0]


def _ids(gen, kind, tokens, vocab):
    if kind == "uniform":
        return torch.randint(vocab, (tokens,), generator=gen, device=gen.device)
    if kind == "one":
        return torch.full((tokens,), vocab - 1, device=gen.device)
    if kind == "padding":
        return torch.full((tokens,), -100, device=gen.device)
    # frequent and rare words, runs that begin and end everywhere within the chunks, a tenth of padding
    u = torch.rand(tokens, generator=gen, device=gen.device, dtype=torch.float64)
    ids = ((vocab + 1.0) ** u - 1.0).long().clamp(max=vocab - 1)
    ids[torch.rand(tokens, generator=gen, device=gen.device) < 0.1] = -100
    return ids


@pytest.mark.parametrize("kind", ["uniform", "one", "frequent", "padding"])
@pytest.mark.parametrize("tokens, vocab, width", [(1, 1, 1), (2, 9, 8), (31, 4, 3), (64, 2, 40), (65, 2, 40), (97, 600, 500), (1000, 13, 129), (8192, 85000, 16),
                                                  (8193, 700, 12), (20000, 1 << 20, 4), (70000, 300, 9)])
def test_embedding_gradient(cuda_device, kind, tokens, vocab, width):
    gen = _gen(cuda_device, tokens)
    for dtype, grads, strided in [(torch.bfloat16, torch.float32, False), (torch.float32, torch.float32, True), (torch.float16, torch.float16, False),
                                  (torch.bfloat16, torch.bfloat16, True)]:
        ids = _ids(gen, kind, tokens, vocab)
        dy = _inset(_rand(gen, tokens, width, dtype=dtype), strided)
        out = Inset(vocab, width, grads, cuda_device, strided)
        scale = 1.5
        s = L.EmbeddingSession(vocab, width, tokens, device=cuda_device)
        s.backward(dy, ids, out.t, scale=scale)
        live = ids >= 0
        add = lambda x: torch.zeros(vocab, x.shape[1], dtype=torch.float64, device=cuda_device).index_add_(0, ids[live], x[live])  # noqa: E731
        ref, size = add(dy.double()) * scale, add(dy.double().abs()) * scale
        count = add(torch.ones(tokens, 1, dtype=torch.float64, device=cuda_device))
        _within(out.t, ref, (count + 2) * U * size + HALF_ULP[grads] * ref.abs() + TINY[grads], f"{dtype} {grads}")
        out.check_around()
        again = torch.empty_like(out.t)
        s.backward(dy, ids, again, scale=scale)
        assert torch.equal(again, out.t)                       # the same bits, rows one behind the other or not
        if grads is torch.float32:
            held = _rand(gen, vocab, width)
            total = Inset(vocab, width, grads, cuda_device, strided)
            total.set(held)
            s.backward(dy, ids, total.t, scale=scale, accumulate=True)
            _within(total.t, ref + held.double(), (count + 3) * U * size + 2 * U * held.double().abs(), "accumulated")
            assert torch.equal(total.t[count[:, 0] == 0], held[count[:, 0] == 0])
            total.check_around()


def test_embedding_gradient_of_nothing(cuda_device):
    s = L.EmbeddingSession(5, 8, 4, device=cuda_device)
    dtable = torch.full((5, 8), 3.0, device=cuda_device)
    none, no_ids = torch.empty(0, 8, device=cuda_device), torch.empty(0, dtype=torch.int64, device=cuda_device)
    s.backward(none, no_ids, dtable, accumulate=True)
    assert (dtable == 3).all()
    s.backward(none, no_ids, dtable)
    assert (dtable == 0).all()
    assert s.forward(dtable, no_ids).shape == (0, 8)


# ------------------------------------------------------------------------------------------------------------- layer norm

NORM_SHAPES = [(1, 1), (3, 2), (5, 16), (1, 4096), (300, 33), (257, 500), (64, 512), (40, 513), (33, 1000), (70, 1001), (21, 2049), (700, 4096), (9, 6001),
               (5, 8192), (4, 8193), (3, 16384), (2, 20000), (1500, 24)]


def _norm_ref(x, weight, bias, eps):
    """y in 64 bits and a bound on its error before its last rounding."""
    x = x.double()
    width = x.shape[1]
    depth = 16 + 5 + 32 + width / 1024
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    off = (depth + 2) * U * x.abs().mean(1, keepdim=True)                      # of the mean
    rel = 0.5 * ((depth + 6) * U * var + off * off) * rstd * rstd + 3 * U      # of rstd
    n = (x - mean) * rstd
    w = torch.ones(width, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    b = torch.zeros_like(w) if bias is None else bias.double()
    return n * w + b, w.abs() * (n.abs() * (rel + 4 * U) + off * rstd) + 2 * U * (n * w).abs() + 2 * U * b.abs(), mean[:, 0], off[:, 0], rstd[:, 0], rel[:, 0]


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, width", NORM_SHAPES)
def test_layer_norm(cuda_device, rows, width, dtype, strided):
    gen = _gen(cuda_device, rows * width)
    eps = 1e-5
    x = _inset((_rand(gen, rows, 1) * 2 + _rand(gen, rows, width) * (0.1 + _rand(gen, rows, 1).abs())).to(dtype), strided)
    s = L.LayerNormSession(width, rows, dtype=dtype, eps=eps, device=cuda_device)
    for params in {torch.float32, dtype}:
        weight, bias = _rand(gen, width, dtype=params), _rand(gen, width, dtype=params)
        out = Inset(rows, width, dtype, cuda_device, strided)
        mean, rstd = (torch.empty(rows, device=cuda_device) for _ in range(2))
        s.forward(x, weight, bias, out=out.t, mean=mean, rstd=rstd)
        y, tol, mean64, off, rstd64, rel = _norm_ref(x, weight, bias, eps)
        _within(out.t, y, tol + HALF_ULP[dtype] * (y.abs() + tol) + TINY[dtype], "y")
        _within(mean, mean64, off + U * mean64.abs(), "mean")
        _within(rstd, rstd64, rstd64 * (rel + U), "rstd")
        out.check_around()
    y, tol, *_ = _norm_ref(x, None, None, eps)
    _within(s.forward(x), y, tol + HALF_ULP[dtype] * (y.abs() + tol) + TINY[dtype], "without parameters")
    place = x.clone()
    s.forward(place, None, None, out=place)
    assert torch.equal(place, s.forward(x.clone()))


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, width", NORM_SHAPES)
def test_layer_norm_gradient(cuda_device, rows, width, dtype, strided):
    gen = _gen(cuda_device, rows * width + 1)
    x = _inset(_rand(gen, rows, width, dtype=dtype), strided)
    dy, add = (_inset(_rand(gen, rows, width, dtype=dtype), strided) for _ in range(2))
    weight = _rand(gen, width)
    x64, dy64 = x.double(), dy.double()
    mean64 = x64.mean(1, keepdim=True)
    mean, rstd = mean64[:, 0].float(), ((x64 - mean64).square().mean(1) + 1e-5).rsqrt().float()
    n = (x64 - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy64 * weight.double()
    r = rstd.double()[:, None]
    p, q = g.mean(1, keepdim=True), (g * n).mean(1, keepdim=True)
    dx = (g - p - n * q) * r
    depth = 16 + 5 + 32 + width / 1024
    off_p, off_q = (depth + 3) * U * g.abs().mean(1, keepdim=True), (depth + 6) * U * (g * n).abs().mean(1, keepdim=True)
    tol = r * (off_p + n.abs() * off_q + 4 * U * (g.abs() + p.abs() + 3 * (n * q).abs()))
    s = L.LayerNormSession(width, rows, dtype=dtype, device=cuda_device)
    out = Inset(rows, width, dtype, cuda_device, strided)
    dweight, dbias = (torch.full((width,), 9.0, device=cuda_device) for _ in range(2))
    s.backward(dy, x, weight, mean, rstd, dx=out.t, dweight=dweight, dbias=dbias)
    _within(out.t, dx, tol + HALF_ULP[dtype] * (dx.abs() + tol) + TINY[dtype], "dx")
    out.check_around()
    # a column passes through the rows of a CTA (at most one in 32 of all, or all of few), the CTAs' shares and the warps that join them
    steps = rows / 32 + 64
    dw64, db64 = (dy64 * n).sum(0), dy64.sum(0)
    _within(dweight, dw64, (steps + 4) * U * (dy64 * n).abs().sum(0) + TINY[torch.float32], "dweight")
    _within(dbias, db64, steps * U * dy64.abs().sum(0) + TINY[torch.float32], "dbias")
    first = dweight.clone(), dbias.clone()
    held = _rand(gen, width)
    dweight.copy_(held), dbias.copy_(held)
    # with the gradient that comes past the norm, in dy's own place, sums added to what is there
    place = _inset(dy, strided)
    s.backward(place, x, weight, mean, rstd, dx=place, add=add, dweight=dweight, dbias=dbias, accumulate=True)
    with_add = dx + add.double()
    _within(place, with_add, tol + 2 * U * add.double().abs() + HALF_ULP[dtype] * (with_add.abs() + tol) + TINY[dtype], "dx + add")
    assert torch.equal(dweight, held + first[0]) and torch.equal(dbias, held + first[1])
    # each alone, and no weight
    alone = torch.empty(width, device=cuda_device)
    s.backward(dy, x, weight, mean, rstd, dbias=alone)
    assert torch.equal(alone, first[1])
    s.backward(dy, x, weight, mean, rstd, dweight=alone)
    assert torch.equal(alone, first[0])
    only = torch.empty_like(dy)
    s.backward(dy, x, torch.ones(width, device=cuda_device), mean, rstd, dx=only)
    bare = torch.empty_like(dy)
    s.backward(dy, x, None, mean, rstd, dx=bare)
    assert torch.equal(only, bare)


def test_layer_norm_rows_that_are_not_ordinary(cuda_device):
    """Constant rows, rows far from zero, rows with an infinity or a NaN (theirs alone); no rows at all."""
    s = L.LayerNormSession(1000, 8, dtype=torch.float32, device=cuda_device)
    x = _rand(_gen(cuda_device, 5), 8, 1000)
    x[1] = 3.0
    x[2] += 1e4
    x[3, 7], x[4, 999], x[5] = float("nan"), float("inf"), 0.0
    y = s.forward(x)
    assert (y[1] == 0).all() and (y[5] == 0).all() and torch.isnan(y[3]).all() and torch.isnan(y[4]).all()
    ref, tol, *_ = _norm_ref(x[[0, 2, 6, 7]], None, None, 1e-5)
    _within(y[[0, 2, 6, 7]], ref, tol + 2 * U * ref.abs(), "the others")
    dweight = torch.full((1000,), 5.0, device=cuda_device)
    none, few = torch.empty(0, 1000, device=cuda_device), torch.empty(0, device=cuda_device)
    assert s.forward(none).shape == (0, 1000)
    s.backward(none, none, None, few, few, dx=none, dweight=dweight, accumulate=True)
    assert (dweight == 5).all()
    s.backward(none, none, None, few, few, dx=none, dweight=dweight)
    assert (dweight == 0).all()


# ------------------------------------------------------------------------------------------------------------- recurrence

def _recurrence64(gate, value, ends, h0, dy=None, dh_last=None):
    """States and gradients in 64 bits, row by row, with bounds on the errors before the last rounding."""
    g, v = gate.double(), value.double()
    f, s, eta = torch.sigmoid(g), torch.sigmoid(-g), 2.0 ** -21 + g.abs().nan_to_num(0, 100, 100) * 2.0 ** -23 + 6 * U
    y, before, tol_y, tol_before = (torch.zeros_like(g) for _ in range(4))
    h_last, tol_last = h0.double().clone(), torch.zeros_like(h0, dtype=torch.float64)
    dgate, dvalue, tol_dg, tol_dv = (torch.zeros_like(g) for _ in range(4))
    dh0 = None if dy is None else dh_last.double().clone()
    tol_dh0 = torch.zeros_like(h_last)
    for q, (b, e) in enumerate(zip(ends, ends[1:])):
        h, size, off = h0[q].double(), h0[q].double().abs(), torch.zeros_like(h_last[q])
        for t in range(b, e):
            before[t], tol_before[t] = h, off
            meet = f[t] * size + s[t] * v[t].abs()
            h, size, off = f[t] * h + s[t] * v[t], meet, f[t] * off + eta[t] * meet
            y[t], tol_y[t] = h, off
        h_last[q], tol_last[q] = h, off
        if dy is None:
            continue
        c, size, off = dh_last[q].double(), dh_last[q].double().abs(), torch.zeros_like(h)
        for t in range(e - 1, b - 1, -1):
            dh, size, off = dy[t].double() + c, dy[t].double().abs() + size, off + 4 * U * (dy[t].double().abs() + size)
            dvalue[t], tol_dv[t] = s[t] * dh, s[t] * (off + eta[t] * size)
            apart = (before[t] - v[t]).abs()
            dgate[t] = dh * (before[t] - v[t]) * f[t] * s[t]
            tol_dg[t] = f[t] * s[t] * (off * apart + size * (tol_before[t] + 4 * U * (before[t].abs() + v[t].abs())) + 3 * eta[t] * size * apart)
            c, size, off = f[t] * dh, f[t] * size, f[t] * off + eta[t] * f[t] * size
        dh0[q], tol_dh0[q] = c, off
    return dict(y=(y, tol_y), h_last=(h_last, tol_last), dgate=(dgate, tol_dg), dvalue=(dvalue, tol_dv), dh0=(dh0, tol_dh0))


def _check_recurrence(device, lengths, width, dtype, strided, lead=0, tail=0, packed=True, bits=64, seed=0, zero_start=False):
    gen = _gen(device, seed + width)
    ends = np.cumsum([lead] + list(lengths)).tolist()
    rows, count = ends[-1] + tail, len(lengths)
    gate, value, dy = (_inset(_rand(gen, rows, width, scale=k).to(dtype), strided) for k in (2.0, 1.0, 1.0))
    gate += 1.0
    h0, dh_last = _rand(gen, count, width), _rand(gen, count, width)
    offsets = torch.tensor(ends, dtype=torch.int64 if bits == 64 else torch.int32, device=device) if packed else None
    ref = _recurrence64(gate, value, ends, torch.zeros_like(h0) if zero_start else h0, dy, torch.zeros_like(dh_last) if zero_start else dh_last)
    out, dgate, dvalue = (Inset(rows, width, dtype, device, strided) for _ in range(3))
    h_last, dh0, marks = torch.empty_like(h0), torch.empty_like(h0), L.recurrence_marks(rows, count, width, device=device)
    marks.fill_(float("nan"))
    start, end = (None, None) if zero_start else (h0, dh_last)
    L.recurrence_forward(gate, value, out=out.t, offsets=offsets, sequences=count, h0=start, h_last=h_last, marks=marks)
    L.recurrence_backward(dy, gate, value, marks, dgate.t, dvalue.t, offsets=offsets, sequences=count, dh_last=end, dh0=dh0)
    inside = slice(lead, rows - tail)
    for got, name in ((out, "y"), (dgate, "dgate"), (dvalue, "dvalue")):
        want, tol = (x[inside] for x in ref[name])
        _within(got.t[inside], want, tol + HALF_ULP[dtype] * (want.abs() + tol) + TINY[dtype], name)
        assert (got.t[:lead] == got.fill).all() and (got.t[rows - tail:] == got.fill).all(), f"{name}: rows of no sequence were written"
        got.check_around()
    for got, name in ((h_last, "h_last"), (dh0, "dh0")):
        want, tol = ref[name]
        _within(got, want, tol + 2 * U * want.abs() + TINY[torch.float32], name)
    # the states and gradients in the places of what they are made from, no marks, no y's: the same bits
    state, again = (torch.zeros_like(h0) if zero_start else h0.clone()), Inset(rows, width, dtype, device, strided)
    L.recurrence_forward(gate, value, out=again.t, offsets=offsets, sequences=count, h0=state, h_last=state)
    assert torch.equal(state, h_last) and torch.equal(again.t, out.t)
    back = torch.zeros_like(h0) if zero_start else dh_last.clone()
    L.recurrence_backward(dy, gate, value, marks, gate, value, offsets=offsets, sequences=count, dh_last=back, dh0=back)
    assert torch.equal(gate[inside], dgate.t[inside]) and torch.equal(value[inside], dvalue.t[inside]) and torch.equal(back, dh0)


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths, width, lead, tail", [
    ([1], 1, 0, 0), ([1, 1, 1], 64, 0, 0), ([0, 3, 0, 1, 0], 7, 2, 3), ([5, 17, 23], 130, 0, 1), ([63], 65, 0, 0), ([64, 65, 1], 66, 0, 0), ([200], 2, 1, 1),
    ([129, 0, 70, 640], 96, 3, 0), ([700], 70, 0, 0), ([1500, 3], 32, 0, 2)])
def test_recurrence(cuda_device, lengths, width, lead, tail, dtype, strided):
    _check_recurrence(cuda_device, lengths, width, dtype, strided, lead, tail)


@pytest.mark.parametrize("lengths, width", [([40] * 3, 34), ([2] * 9, 16), ([1] * 64, 1024), ([600] * 2, 64), ([4100], 64)])
def test_recurrence_of_equal_parts(cuda_device, lengths, width):
    _check_recurrence(cuda_device, lengths, width, torch.bfloat16, False, packed=False)
    _check_recurrence(cuda_device, lengths, width, torch.float32, False, packed=True, bits=32, zero_start=True)


@pytest.mark.parametrize("rows", [3, 50, 400])
def test_recurrence_gates_without_bound(cuda_device, rows):
    """A gate of -inf begins anew, one of +inf and the type's largest keep the state; a NaN stays in its column."""
    gen = _gen(cuda_device, rows)
    gate, value = _rand(gen, rows, 6, dtype=torch.bfloat16), _rand(gen, rows, 6, dtype=torch.bfloat16)
    gate[:, 1], gate[:, 2], gate[:, 3] = float("inf"), torch.finfo(torch.bfloat16).max, float("-inf")
    gate[rows // 2, 4] = float("nan")
    gate[rows // 2, 5] = float("-inf")
    h0 = _rand(gen, 1, 6)
    y = L.recurrence_forward(gate, value, h0=h0)
    assert torch.equal(y[:, 1:3], h0[:, 1:3].bfloat16().expand(rows, 2)) and torch.equal(y[:, 3], value[:, 3])
    assert torch.isnan(y[rows // 2:, 4]).all() and torch.isfinite(y[:rows // 2, 4]).all()
    fresh = L.recurrence_forward(gate[rows // 2:].contiguous(), value[rows // 2:].contiguous(), h0=torch.full((1, 6), 1e30, device=cuda_device))
    _within(y[rows // 2:, 5], fresh[:, 5].double(), fresh[:, 5].double().abs() * 2.0 ** -7 + 1e-6, "after a reset")


def test_recurrence_offsets_that_make_no_sense_are_cut(cuda_device):
    """Ends behind the rows, before the first one or before their beginning: nothing outside is touched, empty sequences keep their state."""
    gate, value = (torch.zeros(100, 8, device=cuda_device) for _ in range(2))
    h0 = torch.ones(3, 8, device=cuda_device)
    out = Inset(100, 8, torch.float32, cuda_device, False)
    h_last = torch.empty_like(h0)
    for offsets in ([-5, 2, 2, 1 << 40], [90, 200, 150, 400], [0, 50, 20, -1]):
        marks = L.recurrence_marks(100, 3, 8, device=cuda_device)
        L.recurrence_forward(gate, value, out=out.t, offsets=torch.tensor(offsets, device=cuda_device), sequences=3, h0=h0, h_last=h_last, marks=marks)
        out.check_around()
    assert (h_last[1:] == 1).all() and (h_last[0] == 0.5 ** 50).all()


def test_recurrence_of_nothing(cuda_device):
    none, h0 = torch.empty(0, 7, device=cuda_device), torch.ones(2, 7, device=cuda_device)
    h_last, dh0 = torch.zeros_like(h0), torch.zeros_like(h0)
    marks = L.recurrence_marks(0, 2, 7, device=cuda_device)
    L.recurrence_forward(none, none, sequences=2, h0=h0, h_last=h_last, marks=marks)
    L.recurrence_backward(none, none, none, marks, none, none, sequences=2, dh_last=h0, dh0=dh0)
    assert torch.equal(h_last, h0) and torch.equal(dh0, h0)


def test_recurrence_gradient_against_differences(cuda_device):
    gen = _gen(cuda_device, 9)
    rows, width = 90, 3
    gate, value, dy = (_rand(gen, rows, width) for _ in range(3))
    h0, dh_last = _rand(gen, 1, width), _rand(gen, 1, width)
    marks = L.recurrence_marks(rows, 1, width, device=cuda_device)
    L.recurrence_forward(gate, value, h0=h0, marks=marks)
    dgate, dvalue, dh0 = torch.empty_like(gate), torch.empty_like(gate), torch.empty_like(h0)
    L.recurrence_backward(dy, gate, value, marks, dgate, dvalue, dh_last=dh_last, dh0=dh0)

    def loss(g, v, h):
        g, v, h, total = g.double(), v.double(), h[0].double(), 0.0
        for t in range(rows):
            f = torch.sigmoid(g[t])
            h = f * h + (1 - f) * v[t]
            total = total + (dy[t].double() * h).sum()
        return total + (dh_last[0].double() * h).sum()

    step = 1e-4
    for grad, at in ((dgate, 0), (dvalue, 1), (dh0, 2)):
        for row in {0, grad.shape[0] // 2, grad.shape[0] - 1}:
            inputs = [t.double() for t in (gate, value, h0)]
            up, down = [t.clone() for t in inputs], [t.clone() for t in inputs]
            up[at][row, 1] += step
            down[at][row, 1] -= step
            slope = float(loss(*up) - loss(*down)) / (2 * step)
            # differences in 64 bits: off by step^2 times a third derivative (below 10 here); the gradient by 2^-18 of magnitudes below 30
            assert abs(slope - float(grad[row, 1])) < 1e-7 * 10 + 30 * 2.0 ** -18
