"""The operators and the gradient exchange together: the MNIST-shaped model trained with dropped gradients."""
import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import train_mlp as M

pytestmark = pytest.mark.gpu


def test_flat_gradient_is_that_of_the_formulas(cuda_device):
    """Loss and gradient of one batch against 64 bits on the same 16-bit activations' weights; the path rounds activations and the
    gradients between layers to bf16 (2^-8 each, two hidden layers and back), so tensors agree to a few of those in norm."""
    model = M.Mlp(48, cuda_device, hidden=512)
    x, t = M.synthetic_batches(48, 1, 0, cuda_device)[0]
    grad = torch.full((model.layer_off[-1],), float("nan"), device=cuda_device)
    loss = model.gradient(x, t, grad)
    w = [p.double().requires_grad_() for p in (v if len(s) == 2 else model.views(model.params)[i] for i, (v, s) in enumerate(zip(model.views(model.copies), model.shapes)))]
    with torch.enable_grad():
        h = torch.relu(x.double() @ w[0] + w[1])
        h = torch.relu(h @ w[2] + w[3])
        rows = torch.nn.functional.cross_entropy(h @ w[4] + w[5], t, reduction="none")
        want = torch.autograd.grad(rows.mean(), w)
    assert float((loss.double() - rows.detach()).abs().max()) < 0.05 * float(rows.detach().max()) + 0.05
    for got, ref in zip(model.views(grad), want):
        assert float((got.double() - ref).norm()) <= 8 * 2.0 ** -8 * float(ref.norm())


@pytest.mark.parametrize("state_bits", [32, 8])
def test_training_with_dropped_gradients_learns(cuda_device, state_bits):
    trainer = M.Trainer(batch=64, workers=2, drop_ppm=990_000, state_bits=state_bits, hidden=512, device=cuda_device)
    losses = [float(trainer.step(M.synthetic_batches(64, 2, step, cuda_device))) for step in range(60)]
    assert all(w.status() == B.GD_OK for w in trainer.workers) and all(s.status() == B.GD_OK for s in trainer.model.layers)
    assert sum(losses[-10:]) < 0.35 * sum(losses[:10]), losses
    assert torch.equal(trainer.model.copies, trainer.model.params.bfloat16())


def test_two_runs_are_the_same(cuda_device):
    """Pushes are applied in order and nothing else depends on timing: the same seed trains the same parameters, bit for bit."""
    def run():
        trainer = M.Trainer(batch=32, workers=2, state_bits=8, hidden=256, device=cuda_device)
        for step in range(5):
            trainer.step(M.synthetic_batches(32, 2, step, cuda_device))
        return trainer.model.params
    assert torch.equal(run(), run())
