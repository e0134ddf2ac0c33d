"""The layers together, as they are used: a language model's gradient against 64 bits, its training with dropped gradients, its answers word by
word against the pass over whole sentences."""
import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import train_lm as M
from paper_1704_05021_b200.train_mlp import Trainer

pytestmark = pytest.mark.gpu


def _logits64(model, tokens, offsets, tensors):
    """The model's formula in 64 bits on the given tensors."""
    d, it = model.width, iter(tensors)
    norm = lambda x, g, b: torch.nn.functional.layer_norm(x, (d,), g, b, 1e-5)  # noqa: E731
    x = next(it)[tokens] * model.scale
    for _ in range(model.blocks):
        g1, b1, wz, bz, wo, bo, g2, b2, wu, bu, wd, bd = (next(it) for _ in range(12))
        gate, value = (norm(x, g1, b1) @ wz + bz).split(d, 1)
        f, rows = torch.sigmoid(gate), []
        begins = set(offsets.tolist())
        for t in range(len(tokens)):
            h = torch.zeros_like(value[0]) if t in begins else h  # noqa: F821
            h = f[t] * h + (1 - f[t]) * value[t]
            rows.append(h)
        x = x + torch.stack(rows) @ wo + bo
        a, u = (norm(x, g2, b2) @ wu + bu).chunk(2, 1)
        x = x + (torch.nn.functional.silu(a) * u) @ wd + bd
    g, b, w, bias = (next(it) for _ in range(4))
    return norm(x, g, b) @ w + bias


def _tensors64(model):
    """What the model computes with: 16-bit matrices, fp32 vectors."""
    pairs = zip(model.views(model.params), model.views(model.copies), model.shapes)
    return [(c if len(s) == 2 else p).double().requires_grad_() for p, c, s in pairs]


def test_gradient_is_that_of_the_formula(cuda_device):
    """Against autograd in 64 bits on the same weights.  The path rounds its activations and the gradients between its calls to bf16, about ten of
    each in a row over two blocks, so tensors agree to a few times ten roundings (2^-8 each) in norm."""
    model = M.Lm(vocab=96, width=64, hidden=96, blocks=2, rows=150, sentences=5, device=cuda_device, seed=3)
    (tokens, offsets), targets = M.synthetic_batches(96, 150, 5, 1, 0, cuda_device)[0]
    grad = torch.full((model.layer_off[-1],), float("nan"), device=cuda_device)
    loss = model.gradient((tokens, offsets), targets, grad).clone()
    tensors = _tensors64(model)
    with torch.enable_grad():
        rows = torch.nn.functional.cross_entropy(_logits64(model, tokens, offsets, tensors), targets, reduction="none")
        want = torch.autograd.grad(rows.sum() / len(tokens), tensors)
    assert all(s.status() == B.GD_OK for s in model.layers)
    assert float((loss.double() - rows.detach()).norm()) <= 20 * 2.0 ** -8 * float(rows.detach().norm())
    for got, ref, shape in zip(model.views(grad), want, model.shapes):
        assert float((got.double() - ref).norm()) <= 20 * 2.0 ** -8 * float(ref.norm()), shape


def test_answers_word_by_word_are_those_of_the_whole_sentence(cuda_device):
    """One token a call with the state carried on, and a sentence cut in two: the logits of one pass, but for bf16 roundings on the way."""
    model = M.Lm(vocab=64, width=64, hidden=64, blocks=2, rows=60, sentences=3, device=cuda_device)
    gen = torch.Generator(device=cuda_device).manual_seed(1)
    tokens = torch.randint(64, (3, 20), generator=gen, device=cuda_device)
    whole = model.forward(tokens.flatten(), None, 3).clone().view(3, 20, -1)
    room = 10 * 2.0 ** -8 * float(whole.float().abs().max())
    state = model.new_state(3)
    for t in range(20):
        assert float((model.answer(tokens[:, t].contiguous(), state).float() - whole[:, t].float()).abs().max()) <= room
    state = model.new_state(3)
    first = model.forward(tokens[:, :7].flatten(), None, 3, state).clone().view(3, 7, -1)
    second = model.forward(tokens[:, 7:].flatten(), None, 3, state).view(3, 13, -1)
    assert float((torch.cat([first, second], 1).float() - whole.float()).abs().max()) <= room


@pytest.mark.parametrize("state_bits", [32, 8])
def test_training_runs_and_repeats(cuda_device, state_bits):
    """Steps end without a refused call or a wait that ran out, parameters and copies move together, and the same seed gives the same bits."""
    def run():
        model = M.Lm(vocab=200, width=64, hidden=128, blocks=2, rows=300, sentences=9, device=cuda_device)
        trainer = Trainer(workers=2, drop_ppm=900_000, state_bits=state_bits, model=model)
        losses = [trainer.step(M.synthetic_batches(200, 300, 9, 2, step, cuda_device)) for step in range(4)]
        assert all(w.status() == B.GD_OK for w in trainer.workers) and all(s.status() == B.GD_OK for s in model.layers)
        assert torch.isfinite(torch.stack(losses)).all() and torch.equal(model.copies, model.params.bfloat16())
        return model.params

    assert torch.equal(run(), run())


def test_step_captured_and_replayed(cuda_device):
    """A whole gradient captured once gives the same bits as the calls, also on other tokens."""
    model = M.Lm(vocab=96, width=64, hidden=96, blocks=1, rows=200, sentences=4, device=cuda_device)
    batches = [M.synthetic_batches(96, 200, 4, 1, step, cuda_device)[0] for step in range(3)]
    want = []
    for batch, targets in batches:
        grad = torch.empty(model.layer_off[-1], device=cuda_device)
        model.gradient(batch, targets, grad)
        want.append(grad)
    (tokens, offsets), targets = ([t.clone() for t in batches[0][0]], batches[0][1].clone())
    grad = torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        model.gradient((tokens, offsets), targets, grad)
    for n in (1, 2, 0, 0):
        tokens.copy_(batches[n][0][0]), offsets.copy_(batches[n][0][1]), targets.copy_(batches[n][1])
        grad.zero_()
        graph.replay()
        assert torch.equal(grad, want[n])
