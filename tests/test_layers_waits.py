"""Device-side waits of the layers that run out: a wait for more than anybody sends, for a few milliseconds, by the library's own self-tests."""
import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import layers as L

BF16 = torch.bfloat16
SPACE, RESULTS, MATRIX = 663552, 401408, 131072


def test_the_recurrences_self_test_refuses_what_does_not_fit():
    """Fake addresses: the checks come before anything is enqueued."""
    lib = L.load_library()
    for space, size, which, code in ((0x10000, SPACE - 1, 0, B.GD_ERR_WORKSPACE), (None, SPACE, 0, B.GD_ERR_WORKSPACE), (0x10010, SPACE, 3, B.GD_ERR_WORKSPACE),
                                     (0x10000, SPACE, 4, B.GD_ERR_INVALID_ARG), (0x10000, SPACE, -1, B.GD_ERR_INVALID_ARG)):
        assert lib.gd_selftest_recurrence_wait(space, size, which, 1, None) == code


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_a_wait_of_the_recurrence_that_runs_out_leaves_nan(cuda_device, which):
    """Copies or maps that never come whole, forward and backward: every result is NaN - those of the rows that the wait was for among them - and the
    call ends after a few waits, not one for each of its 64 tiles; the next call works."""
    lib, budget_ns = L.load_library(), 20_000_000
    ws = torch.empty(SPACE + 256, dtype=torch.uint8, device=cuda_device)
    ws[SPACE:] = 7
    stream = torch.cuda.current_stream().cuda_stream
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for _ in range(2):                                   # (the first call may load the kernel)
        begin.record()
        assert lib.gd_selftest_recurrence_wait(ws.data_ptr(), SPACE, which, budget_ns, stream) == B.GD_OK
        end.record()
        end.synchronize()
        results = ws[RESULTS:RESULTS + (2 if which > 1 else 1) * MATRIX].view(BF16)
        assert bool(torch.isnan(results).all())
    assert begin.elapsed_time(end) < 16 * budget_ns * 1e-6
    assert bool((ws[SPACE:] == 7).all())
    gate, value = torch.zeros(8192, 8, dtype=BF16, device=cuda_device), torch.ones(8192, 8, dtype=BF16, device=cuda_device)
    marks = L.recurrence_marks(8192, 1, 8, device=cuda_device)
    y = L.recurrence_forward(gate, value, marks=marks)
    assert bool((y[20:] == 1).all()) and bool((y[0] == 0.5).all())
    dgate, dvalue = torch.empty_like(gate), torch.empty_like(gate)
    L.recurrence_backward(value, gate, value, marks, dgate, dvalue)
    assert bool((dvalue[:-20] == 1).all()) and bool((dvalue[-1] == 0.5).all()) and bool(torch.isfinite(dgate).all())


@pytest.mark.gpu
def test_a_wait_of_the_gated_blocks_bias_gradient_that_runs_out_reaches_the_status(cuda_device):
    """The status says so, the sums are NaN, and the next call works once the word is zeroed."""
    s = L.GatedLinearSession(32, 32, 512, device=cuda_device)
    ws, lib = s.workspace, L.load_library()
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.gd_selftest_gated_wait(ws.data_ptr(), 25087, 1_000_000, stream) == B.GD_ERR_WORKSPACE
    assert lib.gd_selftest_gated_wait(ws.data_ptr(), ws.numel(), 1_000_000, stream) == B.GD_OK
    assert s.status() == B.GD_ERR_DEVICE_TIMEOUT
    assert bool(torch.isnan(ws[256:512].view(torch.float32)).all())
    ws[:256].zero_()
    dy, pre, db = torch.ones(512, 32, dtype=BF16, device=cuda_device), torch.ones(512, 64, dtype=BF16, device=cuda_device), torch.empty(64, device=cuda_device)
    s.backward(dy, None, None, pre, db=db)
    silu = 1 / (1 + 2.718281828459045 ** -1)             # of 1, and its slope there s (1 + 1 - s)
    # (sums of 512 equal terms up to 0.93: 20 additions in a row of 2^-24 and a sigmoid good to 2^-20 are below 1e-3 of them)
    assert bool(((db[32:] - 512 * silu).abs() < 1e-3).all()) and bool(((db[:32] - 512 * silu * (2 - silu)).abs() < 1e-3).all()) and s.status() == B.GD_OK
