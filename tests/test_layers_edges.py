"""Embedding, layer norm, recurrence and gated block where calls meet: other streams, captured graphs, sessions side by side, clusters of every size,
matrices that 32 bits do not count.  Equal bits are asked for wherever the same call is made twice."""
import pytest
import torch

from paper_1704_05021_b200 import layers as L
from test_layers_ops import Inset, _check_recurrence, _gen, _rand

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


class Calls:
    """Every call of layers.py on inputs of its own; run() gives all their results."""

    def __init__(self, device, seed, rows=700, width=264):
        self.device, self.rows, self.width = device, rows, width
        half = lambda *s: torch.empty(*s, dtype=BF16, device=device)  # noqa: E731
        wide = lambda *s: torch.empty(*s, device=device)  # noqa: E731
        self.ids = torch.empty(9000, dtype=torch.int64, device=device)
        self.offsets = torch.empty(5, dtype=torch.int64, device=device)
        self.table, self.x, self.dy, self.gate, self.w = half(300, width), half(rows, width), half(rows, width), half(rows, width), half(width, 512)
        self.e_dy, self.gamma, self.beta, self.h0 = half(9000, width), wide(width), wide(width), wide(4, width)
        self.embedding, self.norm = L.EmbeddingSession(300, width, 9000, device=device), L.LayerNormSession(width, rows, device=device)
        self.gated = L.GatedLinearSession(width, 256, rows, device=device)
        self.marks = L.recurrence_marks(rows, 4, width, device=device)
        self.out = dict(e=half(9000, width), de=wide(300, width), few=wide(300, width), n=half(rows, width), mean=wide(rows), rstd=wide(rows), dn=half(rows, width),
                        dgamma=wide(width), dbeta=wide(width), h=half(rows, width), last=wide(4, width), dgate=half(rows, width), dvalue=half(rows, width),
                        dh0=wide(4, width), g=half(rows, 256), pre=half(rows, 512), dx=half(rows, width), dw=wide(width, 512), db=wide(512))
        self.fill(seed)

    def fill(self, seed):
        gen = _gen(self.device, seed)
        for t in (self.table, self.x, self.dy, self.gate, self.e_dy, self.gamma, self.beta, self.h0):
            t.copy_(torch.randn(t.shape, generator=gen, device=self.device))
        self.w.copy_(torch.randn(self.w.shape, generator=gen, device=self.device) * 0.05)
        self.ids.copy_((torch.rand(9000, generator=gen, device=self.device) ** 3 * 300).long())
        cuts = torch.randint(self.rows + 1, (3,), generator=gen, device=self.device).sort().values
        self.offsets.copy_(torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), self.rows)]))

    def run(self, stream=None):
        o, k = self.out, dict(stream=stream)
        self.embedding.forward(self.table, self.ids, out=o["e"], scale=2.0, **k)
        self.embedding.backward(self.e_dy, self.ids, o["de"], **k)                       # sorted by many CTAs
        self.embedding.backward(self.e_dy[:500], self.ids[:500], o["few"], **k)          # and by one, in the same workspace
        self.norm.forward(self.x, self.gamma, self.beta, out=o["n"], mean=o["mean"], rstd=o["rstd"], **k)
        self.norm.backward(self.dy, self.x, self.gamma, o["mean"], o["rstd"], dx=o["dn"], add=self.gate, dweight=o["dgamma"], dbias=o["dbeta"], **k)
        spans = dict(offsets=self.offsets, sequences=4)
        L.recurrence_forward(self.gate, self.x, out=o["h"], h0=self.h0, h_last=o["last"], marks=self.marks, **spans, **k)
        L.recurrence_backward(self.dy, self.gate, self.x, self.marks, o["dgate"], o["dvalue"], dh_last=self.h0, dh0=o["dh0"], **spans, **k)
        self.gated.forward(self.x, self.w, out=o["g"], pre=o["pre"], **k)
        self.gated.backward(o["g"], self.x, self.w, o["pre"], dx=o["dx"], dw=o["dw"], db=o["db"], **k)

    def results(self):
        return {name: t.clone() for name, t in self.out.items()}


def _same(a, b):
    assert a.keys() == b.keys()
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_captured_calls_replay_to_the_same_bits(cuda_device):
    c = Calls(cuda_device, 1)
    want = []
    for seed in (1, 2):
        c.fill(seed)
        c.run()
        want.append(c.results())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for seed in (2, 1, 1):
        c.fill(seed)
        for t in c.out.values():
            t.zero_()
        graph.replay()
        _same(c.results(), want[seed - 1])


def test_two_sessions_on_two_streams_at_once(cuda_device):
    both = [Calls(cuda_device, seed) for seed in (3, 4)]
    want = []
    for c in both:
        c.run()
        want.append(c.results())
    streams = [torch.cuda.Stream(cuda_device) for _ in both]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(both, streams):
            c.run(stream=s)
    torch.cuda.synchronize()
    for c, w in zip(both, want):
        _same(c.results(), w)


def test_results_made_by_a_call_come_from_its_stream(cuda_device):
    """Without `out` on another stream than the current one: the result is that of the call, whatever the current stream does with freed memory."""
    s = torch.cuda.Stream(cuda_device)
    norm = L.LayerNormSession(512, 4000, dtype=torch.float32, device=cuda_device)
    x = _rand(_gen(cuda_device, 0), 4000, 512)
    want = norm.forward(x)
    torch.cuda.synchronize()
    for _ in range(20):
        y = norm.forward(x, stream=s)
        junk = torch.full((4000, 512), 7.0, device=cuda_device)
        del junk
        s.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("sequences, rows, width, dtype", [(2, 1100, 1024, BF16), (4, 700, 1024, BF16), (9, 300, 1024, torch.float16), (1, 2300, 72, BF16),
                                                          (1, 4200, 40, BF16), (1, 1100, 48, BF16), (2, 1100, 544, torch.float32), (1, 2200, 36, torch.float32),
                                                          (3, 500, 328, BF16), (40, 100, 520, BF16)])
def test_recurrence_in_clusters_of_every_size(cuda_device, sequences, rows, width, dtype):
    """Tiles that end a set, sets that end inside a cluster, sequences of other lengths than the mean that the cluster was chosen by."""
    lengths = [rows + 13 * (i % 3) - 9 * (i % 2) for i in range(sequences)]
    if sequences > 2:
        lengths[1], lengths[2] = 0, 2 * rows - lengths[2]
    _check_recurrence(cuda_device, lengths, width, dtype, False, seed=rows)


@pytest.mark.parametrize("sequences, width, dtype, bits", [(3, 6400, BF16, 64), (40, 520, BF16, 64), (41, 1000, torch.float16, 32), (40, 300, torch.float32, 64),
                                                           (70, 321, BF16, 32)])
def test_recurrence_in_the_order_of_lengths(cuda_device, sequences, width, dtype, bits):
    """More items than run at once: empty sequences, many of one length, the longest last."""
    lengths = [(0, 40, 40, 97, 1)[i % 5] for i in range(sequences - 1)]
    _check_recurrence(cuda_device, lengths + [sequences * sequences - sum(lengths) + 300], width, dtype, width % 2 == 0, 2, 1, bits=bits)


@pytest.mark.parametrize("tokens, vocab, width, ld", [(9000, 4500, 1204, 1204), (9001, 4499, 1203, 1210), (8200, 33, 2100, 2100), (20000, 9999, 4, 5)])
def test_embedding_gradient_of_many_positions(cuda_device, tokens, vocab, width, ld):
    """Positions enough for most rows: every row that no id has is zero, wherever it lies, and nothing between the rows is touched."""
    gen = _gen(cuda_device, tokens)
    ids = torch.randint(vocab // 3, vocab - vocab // 4, (tokens,), generator=gen, device=cuda_device)      # none of the first and of the last rows
    ids[::7] = -100
    dy = _rand(gen, tokens, width, dtype=BF16)
    room = torch.full((vocab, ld), float("nan"), device=cuda_device)
    room[:, width:] = 5.0
    L.EmbeddingSession(vocab, width, tokens, device=cuda_device).backward(dy, ids, room[:, :width])
    live = ids >= 0
    ref = torch.zeros(vocab, width, dtype=torch.float64, device=cuda_device).index_add_(0, ids[live], dy[live].double())
    size = torch.zeros_like(ref).index_add_(0, ids[live], dy[live].double().abs())
    assert ((room[:, :width].double() - ref).abs() <= (tokens + 2) * 2.0 ** -24 * size).all() and bool((room[:, width:] == 5.0).all())


def test_matrices_past_32_bits(cuda_device):
    """More than 2^31 elements: the last rows are those of a call on them alone."""
    rows, width = (1 << 20) + 37, 2056
    x = torch.empty(rows, width, dtype=BF16, device=cuda_device)
    for at in range(0, rows, 1 << 17):
        x[at:at + (1 << 17)].normal_()
    dy = torch.empty_like(x).copy_(x.flip(0))
    y, tail = torch.empty_like(x), slice(rows - 500, rows)
    norm, few = L.LayerNormSession(width, rows, device=cuda_device), L.LayerNormSession(width, 500, device=cuda_device)
    mean, rstd = torch.empty(rows, device=cuda_device), torch.empty(rows, device=cuda_device)
    norm.forward(x, out=y, mean=mean, rstd=rstd)
    assert torch.equal(y[tail], few.forward(x[tail]))
    norm.backward(dy, x, None, mean, rstd, dx=y)
    dx = torch.empty(500, width, dtype=BF16, device=cuda_device)
    few.backward(dy[tail], x[tail], None, mean[tail], rstd[tail], dx=dx)
    assert torch.equal(y[tail], dx)
    # a table of so many elements, its last rows looked up and summed; 500 rows out of a long list
    table_rows = rows
    ids = torch.randint(table_rows - 300, table_rows, (500,), device=cuda_device)
    s = L.EmbeddingSession(table_rows, width, 500, device=cuda_device)
    assert torch.equal(s.forward(x, ids), x[ids])
    s.backward(dy[tail], ids, y, scale=1.0)
    small = torch.empty(300, width, dtype=BF16, device=cuda_device)
    L.EmbeddingSession(300, width, 500, device=cuda_device).backward(dy[tail], ids - (table_rows - 300), small)
    assert torch.equal(y[table_rows - 300:], small) and not bool(y[:1000].any())
    # the last sequence of many rows
    offsets = torch.tensor([0, rows - 400, rows], device=cuda_device)
    marks = L.recurrence_marks(rows, 2, width, device=cuda_device)
    L.recurrence_forward(dy, x, out=y, offsets=offsets, sequences=2, marks=marks)
    alone, own = torch.empty(400, width, dtype=BF16, device=cuda_device), L.recurrence_marks(400, 1, width, device=cuda_device)
    L.recurrence_forward(dy[rows - 400:], x[rows - 400:], out=alone, marks=own)
    close = lambda a, b: float((a.float() - b.float()).abs().max()) <= 2.0 ** -7 * float(b.float().abs().max())  # noqa: E731  (two roundings: other tiles)
    assert close(y[rows - 400:], alone)
    dv, dv_alone = torch.empty_like(x), torch.empty_like(alone)
    L.recurrence_backward(dy, dy, x, marks, y, dv, offsets=offsets, sequences=2)
    L.recurrence_backward(dy[rows - 400:], dy[rows - 400:], x[rows - 400:], own, alone, dv_alone)
    assert close(y[rows - 400:], alone) and close(dv[rows - 400:], dv_alone)


def test_gated_block_past_32_bits(cuda_device):
    m, n, k = 262144 + 100, 4104, 64
    x, w = torch.empty(m, k, dtype=BF16, device=cuda_device).normal_(), torch.randn(2 * n, k, device=cuda_device).bfloat16() * 0.1
    s, few = (L.GatedLinearSession(k, n, rows, w_layout="out_in", device=cuda_device) for rows in (m, 100))
    pre, y = torch.empty(m, 2 * n, dtype=BF16, device=cuda_device), torch.empty(m, n, dtype=BF16, device=cuda_device)
    s.forward(x, w, out=y, pre=pre)
    z = torch.empty(100, 2 * n, dtype=BF16, device=cuda_device)
    want = few.forward(x[-100:], w, pre=z)
    # (other tiles sum in another order: a rounding of 16 bits may fall the other way)
    assert float((y[-100:].float() - want.float()).abs().max()) <= 2.0 ** -7 * float(want.float().abs().max())
    assert float((pre[-100:].float() - z.float()).abs().max()) <= 2.0 ** -7 * float(z.float().abs().max())
    dx = torch.empty(m, k, dtype=BF16, device=cuda_device)
    s.backward(y, x, w, pre, dx=dx)
    few_dx = torch.empty(100, k, dtype=BF16, device=cuda_device)
    few.backward(y[-100:], x[-100:], w, pre[-100:], dx=few_dx)
    assert float((dx[-100:].float() - few_dx.float()).abs().max()) <= 2.0 ** -7 * float(few_dx.float().abs().max())
