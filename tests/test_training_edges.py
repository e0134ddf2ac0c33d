"""The training operators where a result or a row ends inside what a kernel works on at a time: cut tiles of the large products, lengths at
the limits of shared memory, rows worked on in place, values that are not finite.

Tolerances are bounds on the stated arithmetic: a product accumulates in fp32 in steps of 16 products, each rounding (possibly truncating)
once, at most (depth / 16 + 8) 2^-22 of the sum of magnitudes; a result rounds once to its type; a residual is one more fp32 sum.
"""
import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import training as T

pytestmark = pytest.mark.gpu

ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def _rand(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen, device=gen.device) * scale).to(dtype)


def _gen(device, seed):
    return torch.Generator(device=device).manual_seed(seed)


def _kernels(call):
    """The kernels a call launches, by their tags."""
    B.gd_profile_enable(0)
    B.gd_profile_collect()
    B.gd_profile_enable(2)
    try:
        call()
        return [name for name, _ in B.gd_profile_collect(with_tags=True)]
    finally:
        B.gd_profile_enable(0)


def _within(got, ref, room, what):
    over = (got.double() - ref).abs() - room
    assert bool((over <= 0).all()), f"{what}: {float(over.max())} past the bound at {int(over.argmax())}"


def _repeats(call, result, times=20):
    """The call once more and again: the same bits every time.  `call` puts back whatever it adds to."""
    first = result.clone()
    for _ in range(times):
        call()
        assert torch.equal(result, first)


# ------------------------------------------------------------------------------------------ products whose last tiles are cut

CUTS = [8, 32, 40, 64, 72, 96]


@pytest.mark.parametrize("more_rows", [8, 136])
@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("width, kernel", [(4096, "linear_pair"), (2048, "linear_pair_narrow")])
def test_cut_tiles_of_the_forward_product(cuda_device, width, kernel, cut, more_rows):
    """Two to three tiles per pair of CTAs, the last column of them ending after any number of 32-column pieces, the last row of them after
    part of one CTA's half: what is stored of one piece must have left before the next takes its place, stored or not."""
    m, n, k, dt = 2560 + more_rows, width + cut, 200, torch.bfloat16
    gen = _gen(cuda_device, cut)
    x, w, r = _rand(gen, m, k, dtype=dt), _rand(gen, k, n, dtype=dt, scale=k ** -0.5), _rand(gen, m, n, dtype=dt)
    s = T.LinearSession(k, n, m, device=cuda_device)
    ref, size = x.double() @ w.double(), x.double().abs() @ w.double().abs()
    for out_dt in (torch.float32, dt):
        for residual in (None, r):
            for with_pre in (False, True):
                y = torch.full((m, n), float("nan"), dtype=out_dt, device=cuda_device)
                z = torch.full((m, n), float("nan"), dtype=dt, device=cuda_device) if with_pre else None
                call = lambda: s.forward(x, w, residual=residual, out=y, pre=z)  # noqa: B023, E731
                assert _kernels(call) == [kernel]
                want = ref if residual is None else ref + residual.double()
                room = (k / 16 + 8) * 2.0 ** -22 * size + 2.0 ** -23 * (ref.abs() + want.abs())
                _within(y, want, room + ROUND[out_dt] * want.abs(), (out_dt, residual is None, with_pre))
                if with_pre:
                    _within(z, ref, room + ROUND[dt] * ref.abs(), "pre")
                _repeats(call, y)
    assert s.status() == B.GD_OK


def _check_weights(device, m, n, k, layout, accumulate, dtype=torch.bfloat16, kernel="linear_pair"):
    gen = _gen(device, m + n)
    x, dy = _rand(gen, m, k, dtype=dtype), _rand(gen, m, n, dtype=dtype, scale=1e-2)
    shape = (k, n) if layout == "in_out" else (n, k)
    start = _rand(gen, *shape) if accumulate else torch.full(shape, float("nan"), device=device)
    dw = torch.empty_like(start)
    s = T.LinearSession(k, n, m, dtype=dtype, w_layout=layout, device=device)

    def call():
        dw.copy_(start)
        s.backward(dy, x, None, dw=dw, accumulate=accumulate)

    launched = _kernels(call)
    assert launched[-1] == kernel, launched
    ref, size = x.double().T @ dy.double(), x.double().abs().T @ dy.double().abs()
    if layout == "out_in":
        ref, size = ref.T, size.T
    want = ref + start.double() if accumulate else ref
    _within(dw, want, (m / 16 + 8) * 2.0 ** -22 * size + 2.0 ** -23 * (ref.abs() + want.abs()), "dw")
    _repeats(call, dw)
    assert s.status() == B.GD_OK


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("cut", CUTS)
def test_cut_tiles_of_the_weight_gradient(cuda_device, cut, layout, accumulate):
    """The same for fp32 gradients of the weights, written and added to: chains of one and of two."""
    k, n = (2568, 4096 + cut) if layout == "in_out" else (4096 + cut, 2696)
    for m in (200, 648):
        _check_weights(cuda_device, m, n, k, layout, accumulate)
    k, n = (2568, 2048 + cut) if layout == "in_out" else (2048 + cut, 2696)
    _check_weights(cuda_device, 200, n, k, layout, accumulate, kernel="linear_pair_narrow")


def test_weight_gradient_of_the_vocabulary(cuda_device):
    """The output projection of the translation model, 500 x 85000 over 4000 rows: the last column tile has eight columns."""
    _check_weights(cuda_device, 4000, 85000, 500, "in_out", False)
    _check_weights(cuda_device, 4000, 85000, 500, "in_out", True)


def test_weight_gradient_added_to_a_large_matrix(cuda_device):
    _check_weights(cuda_device, 8192, 4104, 4096, "in_out", True)


def _slice_of_a_wider_matrix(rows, cols, dtype, device):
    """[rows, cols] in rows at multiples of 16 bytes, everything around it 77, and a check that it still is."""
    item = 4 if dtype is torch.float32 else 2
    pitch = (cols * item // 16 + 2) * 16 // item
    buf = torch.full(((rows + 1) * pitch,), 77.0, dtype=dtype, device=device)
    view = buf[:rows * pitch].view(rows, pitch)[:, :cols]

    def untouched():
        return bool((buf[:rows * pitch].view(rows, pitch)[:, cols:] == 77).all()) and bool((buf[rows * pitch:] == 77).all())
    return view, untouched


@pytest.mark.parametrize("width, kernel", [(4096, "linear_pair"), (2048, "linear_pair_narrow"), (2400, None)])
@pytest.mark.parametrize("more", [1, 2, 3, 5, 7, 39, 126])
def test_results_in_a_slice_of_a_wider_matrix(cuda_device, width, kernel, more):
    """Widths that are no multiple of 16 bytes in rows that are: nothing behind a row is written, whatever the type, with and without z
    and residual, written and added to.  (The last width comes in 100 rows: the kernel for few tiles.)"""
    m, n, k, dt = (2560 if kernel else 100), width + more, 136, torch.bfloat16
    gen = _gen(cuda_device, more)
    x, w, r = _rand(gen, m, k, dtype=dt), _rand(gen, k, n, dtype=dt, scale=k ** -0.5), _rand(gen, m, n, dtype=dt)
    ref, size = x.double() @ w.double(), x.double().abs() @ w.double().abs()
    s = T.LinearSession(k, n, m, device=cuda_device, any_layout=True)
    for out_dt in (torch.float32, dt):
        for with_residual in (False, True):
            for with_pre in (False, True):
                y, y_kept = _slice_of_a_wider_matrix(m, n, out_dt, cuda_device)
                z, z_kept = _slice_of_a_wider_matrix(m, n, dt, cuda_device)
                res, res_kept = _slice_of_a_wider_matrix(m, n, dt, cuda_device)
                res.copy_(r)
                call = lambda: s.forward(x, w, residual=res if with_residual else None, out=y, pre=z if with_pre else None)  # noqa: B023, E731
                assert kernel is None or _kernels(call)[-1] == kernel
                call()
                assert y_kept() and z_kept() and res_kept(), (out_dt, with_residual, with_pre)
                want = ref + r.double() if with_residual else ref
                room = (k / 16 + 8) * 2.0 ** -22 * size + 2.0 ** -23 * (ref.abs() + want.abs())
                _within(y, want, room + ROUND[out_dt] * want.abs(), "y")
                if with_pre:
                    _within(z, ref, room + ROUND[dt] * ref.abs(), "z")
    # the weights' gradient of a layer with m inputs and n outputs over k rows
    xs, dy = _rand(gen, k, m, dtype=dt), _rand(gen, k, n, dtype=dt)
    ref, size = xs.double().T @ dy.double(), xs.double().abs().T @ dy.double().abs()
    s = T.LinearSession(m, n, k, device=cuda_device, any_layout=True)
    start = _rand(gen, m, n)
    for dw_dt, accumulate in ((torch.float32, False), (torch.float32, True), (dt, False)):
        dw, kept = _slice_of_a_wider_matrix(m, n, dw_dt, cuda_device)
        if accumulate:
            dw.copy_(start)
        s.backward(dy, xs, None, dw=dw, accumulate=accumulate)
        assert kept(), (dw_dt, accumulate)
        want = ref + start.double() if accumulate else ref
        _within(dw, want, (k / 16 + 8) * 2.0 ** -22 * size + 2.0 ** -23 * (ref.abs() + want.abs()) + ROUND[dw_dt] * want.abs(), "dw")


# ------------------------------------------------------------------------------------------ waits that run out

def test_a_wait_that_runs_out_reaches_the_status(cuda_device):
    """The sum of a bias gradient by two CTAs, one waiting (a millisecond) for more than the other sends: the status says so, the sums are NaN,
    and the next call works once the word is zeroed."""
    s = T.LinearSession(32, 32, 512, device=cuda_device)
    ws, lib = s.workspace, T.load_library()
    assert ws.numel() >= 16896
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.gd_selftest_linear_wait(ws.data_ptr(), 16895, 1_000_000, stream) == B.GD_ERR_WORKSPACE
    assert lib.gd_selftest_linear_wait(ws.data_ptr(), ws.numel(), 1_000_000, stream) == B.GD_OK
    assert s.status() == B.GD_ERR_DEVICE_TIMEOUT
    assert bool(torch.isnan(ws[256:384].view(torch.float32)).all())
    ws[:256].zero_()
    dy, db = torch.ones(512, 32, dtype=torch.bfloat16, device=cuda_device), torch.empty(32, device=cuda_device)
    s.backward(dy, None, None, db=db)
    assert bool((db == 512).all()) and s.status() == B.GD_OK


# ------------------------------------------------------------------------------------------ results made by the call

def test_result_made_on_another_stream(cuda_device):
    """Without `out`, on a stream other than the current one, given as an object and as a handle."""
    gen = _gen(cuda_device, 3)
    x, w = _rand(gen, 33, 72, dtype=torch.bfloat16), _rand(gen, 72, 40, dtype=torch.bfloat16)
    s = T.LinearSession(72, 40, 33, device=cuda_device)
    here = s.forward(x, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream, torch.cuda.default_stream()):
        there = s.forward(x, w, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(here, there)


# ------------------------------------------------------------------------------------------ values that are not finite

@pytest.mark.parametrize("offset", [0, 1])
def test_a_moment_that_is_not_finite_leaves_its_block_alone(cuda_device, offset):
    """8-bit moments: the 127 elements that share a scale with an infinite or NaN gradient go on as they would next to a gradient of 0, with the
    same scales, bit for bit; the element itself is NaN from then on."""
    n, bad = 1000, [5, 200, 201, 999]
    gen = _gen(cuda_device, 21)
    grad, start = _rand(gen, n, scale=1e-2), _rand(gen, n, scale=0.1)
    runs = []
    for values in ([0.0] * 4, [float("inf"), float("nan"), -float("inf"), float("inf")]):
        flat = [torch.zeros(n + 4, device=cuda_device) for _ in range(2)]
        p, g = (t[offset:offset + n] for t in flat)
        p.copy_(start), g.copy_(grad)
        s = T.AdamWSession([p], [g], weight_decay=0.01, state_bits=8)
        for step in range(1, 6):
            g[bad] = torch.tensor(values if step == 2 else [0.0] * 4, device=cuda_device)
            s.step(step=step, lr=1e-3, seed=step)
        runs.append([p, s.m[0].float(), s.v[0].float(), s.m_scale[0], s.v_scale[0]])
    others = torch.ones(n, dtype=torch.bool, device=cuda_device)
    others[bad] = False
    for plain, hit in zip(runs[0][:3], runs[1][:3]):
        assert torch.equal(plain[others], hit[others])
        assert bool(torch.isfinite(hit[others]).all())
    for held in runs[1][1:3]:
        assert bool(torch.isnan(held[bad]).all())
    for plain, hit in zip(runs[0][3:], runs[1][3:]):
        assert torch.equal(plain, hit)


# ------------------------------------------------------------------------------------------ memory the session was given

def test_adamw_keeps_the_memory_it_was_given(cuda_device):
    """The session holds addresses: after a tensor has been pointed at other memory, a step must not write what the allocator has made of the old."""
    n = 1 << 20
    p, g, copy = (torch.nn.Parameter(torch.ones(n, device=cuda_device), requires_grad=False) for _ in range(3))
    s = T.AdamWSession([p], [g], copies=[copy])
    for t in (p, g, copy):
        t.data = torch.zeros(4, device=cuda_device)
    others = [torch.full((n,), 7.0, device=cuda_device) for _ in range(6)]
    s.step(step=1, lr=0.1)
    assert all(bool((t == 7).all()) for t in others)
    assert bool((p == 0).all())
