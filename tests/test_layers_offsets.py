"""Offsets of the recurrence that descend: sequences then overlap.  What the rows they share hold is not defined; that nothing else is touched is."""
import pytest
import torch

from paper_1704_05021_b200 import layers as L
from test_layers_ops import Inset, _gen, _rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, offsets, width, dtype", [
    (100, [0, 50, 20, 100], 8, torch.float32), (100, [0, 50, 20, 100], 7, torch.float16),                        # rows a thread, or tiles
    (900, [10, 800, 3, 890], 64, torch.bfloat16), (900, [10, 800, 3, 890], 33, torch.bfloat16),                  # in clusters
    (20, [5, 12, 5, 12, 5, 12], 130, torch.bfloat16),                                                          # single rows on the mean
    (5000, [100, 3000, 90] + [200 + 60 * i for i in range(37)] + [4990], 1024, torch.bfloat16)])                # in the order of lengths
@pytest.mark.parametrize("strided", [False, True])
def test_overlapping_sequences_touch_nothing_outside(cuda_device, rows, offsets, width, dtype, strided):
    sequences, gen = len(offsets) - 1, _gen(cuda_device, rows)
    place = lambda: Inset(rows, width, dtype, cuda_device, strided)  # noqa: E731
    gate, value, dy = (place().set(_rand(gen, rows, width, dtype=dtype)) for _ in range(3))
    at = torch.tensor(offsets, device=cuda_device)
    h0 = _rand(gen, sequences, width)
    h_last, dh0 = (torch.full((sequences + 1, width), 9.0, device=cuda_device) for _ in range(2))
    count = rows // 64 + sequences
    marks = torch.full((count + 1, width), 9.0, device=cuda_device)
    out, dgate, dvalue = place(), place(), place()
    L.recurrence_forward(gate, value, out=out.t, offsets=at, sequences=sequences, h0=h0, h_last=h_last[:sequences], marks=marks)
    L.recurrence_backward(dy, gate, value, marks, dgate.t, dvalue.t, offsets=at, sequences=sequences, dh_last=h0, dh0=dh0[:sequences])
    covered = torch.zeros(rows, dtype=torch.bool, device=cuda_device)
    for first, last in zip(offsets, offsets[1:]):
        covered[first:max(first, last)] = True
    for t in (out, dgate, dvalue):
        t.check_around()
        assert bool((t.t[~covered] == t.fill).all())
    for t in (marks, h_last, dh0):
        assert bool((t[-1] == 9.0).all())
    # empty ones pass their states on
    for s, (first, last) in enumerate(zip(offsets, offsets[1:])):
        if last <= first:
            assert torch.equal(h_last[s], h0[s]) and torch.equal(dh0[s], h0[s])
