"""The measurement hooks over the layers' calls: how many kernels a call launches, and one tagged pair of events for each."""
import os
import re

import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import layers as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16 = torch.bfloat16


def test_every_tag_has_a_name_and_a_line():
    """The library's tags, the binding's names for them and the header's list are of one length."""
    source = open(os.path.join(ROOT, "paper_1704_05021_b200", "csrc", "gd_internal.cuh")).read()
    tags = sorted(int(n) for n in re.findall(r"\bPT_[A-Z_]+ = (\d+)", source))
    assert tags == list(range(len(B.PROFILE_TAGS))) and len(set(B.PROFILE_TAGS)) == len(tags)
    header = open(os.path.join(ROOT, "include", "gd.h")).read()
    text = header[header.index("kernel each belongs to"):header.index("then forgets them")]
    assert {int(n) for n in re.findall(r"\b\d+\b", text) if int(n) != 256 and int(n) != 128} == set(tags)


@pytest.mark.gpu
def test_a_pair_of_events_for_every_kernel_of_the_layers(cuda_device):
    """Every call by the names of its kernels in the order of their launches."""
    half = lambda *s: torch.ones(*s, dtype=BF16, device=cuda_device)  # noqa: E731
    wide = lambda *s: torch.ones(*s, device=cuda_device)  # noqa: E731
    words, norm = L.EmbeddingSession(600, 64, 9000, device=cuda_device), L.LayerNormSession(9000, 400, device=cuda_device)
    short, gated, marks = L.LayerNormSession(64, 400, device=cuda_device), L.GatedLinearSession(64, 128, 400, device=cuda_device), L.recurrence_marks(400, 4, 64, device=cuda_device)
    ids, x, long, stat, table = torch.zeros(9000, dtype=torch.int64, device=cuda_device), half(400, 64), half(400, 9000), wide(400), wide(600, 64)
    calls = [(lambda: words.forward(table, ids), ["embedding"]),
             (lambda: words.backward(half(9000, 64), ids, table), ["embedding_sort"] * 3 + ["embedding_sum", "embedding_join"]),
             (lambda: words.backward(half(400, 64), ids[:400], table), ["embedding_sort", "embedding_sum", "embedding_join"]),
             (lambda: words.backward(half(0, 64), ids[:0], table), ["embedding_zeros"]),
             (lambda: short.forward(x), ["norm"]), (lambda: norm.forward(long), ["norm"]),
             (lambda: short.backward(x, x, None, stat, stat, dx=torch.empty_like(x), dweight=wide(64)), ["norm_backward"]),
             (lambda: norm.backward(long, long, None, stat, stat, dx=torch.empty_like(long), dweight=wide(9000)), ["norm_backward", "norm_backward", "norm_join"]),
             (lambda: L.recurrence_forward(x, x, sequences=4, marks=marks), ["recurrence"]),
             (lambda: L.recurrence_backward(x, x, x, marks, torch.empty_like(x), torch.empty_like(x), sequences=4), ["recurrence_backward"]),
             (lambda: gated.forward(x, half(64, 256)), ["gated"]),
             (lambda: gated.backward(half(400, 128), x, None, half(400, 256), db=wide(256)), ["gated_slope"])]
    B.gd_profile_enable(2)
    try:
        B.gd_profile_collect()
        for call, names in calls:
            before = B.gd_launch_count()
            call()
            pairs = B.gd_profile_collect(with_tags=True)
            assert [name for name, _ in pairs] == names and all(ms >= 0 for _, ms in pairs)
            assert B.gd_launch_count() - before == len(names)
    finally:
        B.gd_profile_enable(0)
        B.gd_profile_collect()


@pytest.mark.gpu
@pytest.mark.parametrize("rows, width, dx, sums, launches", [(4, 9000, True, True, 3), (4, 9000, True, False, 1), (4, 9000, False, True, 2), (400, 9000, False, True, 2),
                                                            (0, 9000, True, True, 1), (4, 64, True, True, 1), (40000, 64, False, True, 2), (40000, 64, True, False, 1)])
def test_launches_of_the_norms_backward_pass_are_counted(cuda_device, rows, width, dx, sums, launches):
    """Rows too long to hold: the sums of columns, dx, and the join of the sums are a launch each, where they are wanted."""
    norm = L.LayerNormSession(width, max(rows, 1), dtype=BF16, device=cuda_device)
    x = torch.ones(rows, width, dtype=BF16, device=cuda_device)
    stat = torch.ones(rows, device=cuda_device)
    dw = torch.empty(width, device=cuda_device) if sums else None
    before = B.gd_launch_count()
    norm.backward(x, x, None, stat, stat, dx=torch.empty_like(x) if dx else None, dweight=dw)
    assert B.gd_launch_count() - before == launches
