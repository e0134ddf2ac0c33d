"""Training the MNIST-shaped model of the benchmark with dropped gradients: every operator of the library in one loop.

    python -m paper_1704_05021_b200.train_mlp [--steps 60] [--workers 2] [--drop-ppm 990000] [--state-bits 8]

Each worker draws a batch, runs three linear layers forward, the cross-entropy and the layers backward; its gradient lands in one
flat fp32 vector, which GradDrop thins out to a push.  The server adds the pushes into a dense vector of zeros and takes one
AdamW step over the six tensors, which also writes the bf16 weights the next forward pass reads.  The workers
share the GPU and take turns; their residuals are their own.  The data are synthetic: ten random prototypes of 784 pixels and noise.
"""
from __future__ import annotations

import argparse
from typing import List

import torch

from . import binding as B
from . import workloads as W
from .session import GradDropSession
from .training import AdamWSession, LinearSession, cross_entropy


class Mlp:
    """784 - 4096 - 4096 - 10 with ReLU: fp32 parameters in one flat vector (W1, b1, W2, b2, W3, b3; matrices are [in, out]) and
    their bf16 copies, and what one worker needs for a pass over `batch` rows."""

    def __init__(self, batch: int, device, hidden: int = 4096, seed: int = 0):
        self.batch, self.device = batch, torch.device(device)
        widths = [784, hidden, hidden, 10]
        self.shapes = [s for i, o in zip(widths, widths[1:]) for s in ((i, o), (o,))]
        self.sizes = [s[0] * (s[1] if len(s) > 1 else 1) for s in self.shapes]
        self.layer_off = [sum(self.sizes[:i]) for i in range(len(self.sizes) + 1)]
        n, dev = self.layer_off[-1], self.device
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.params, self.copies = torch.zeros(n, device=dev), torch.empty(n, dtype=torch.bfloat16, device=dev)
        for t, shape in zip(self.views(self.params), self.shapes):
            if len(shape) == 2:
                t.copy_(torch.randn(shape, generator=gen, device=dev) * (2.0 / shape[0]) ** 0.5)
        self.copies.copy_(self.params)
        bf16 = dict(dtype=torch.bfloat16, device=dev)
        self.layers = [LinearSession(i, o, batch, activation="relu" if o != 10 else "none", device=dev) for i, o in zip(widths, widths[1:])]
        self.hidden = [torch.empty(batch, hidden, **bf16) for _ in range(2)]
        self.pre = [torch.empty(batch, hidden, **bf16) for _ in range(2)]
        self.back = [torch.empty(batch, hidden, **bf16) for _ in range(2)]
        self.logits, self.d_logits = torch.empty(batch, 10, device=dev), torch.empty(batch, 10, device=dev)
        self.d_out, self.loss = torch.empty(batch, 10, **bf16), torch.empty(batch, device=dev)

    def views(self, flat: torch.Tensor) -> List[torch.Tensor]:
        """The six tensors of a flat vector."""
        return [t.view(s) for t, s in zip(torch.split(flat, self.sizes), self.shapes)]

    def gradient(self, x: torch.Tensor, targets: torch.Tensor, flat_grad: torch.Tensor) -> torch.Tensor:
        """Forward and backward of the mean loss: fills flat_grad (fp32, laid out like the parameters); returns the rows' losses."""
        w1, _, w2, _, w3, _ = self.views(self.copies)
        _, b1, _, b2, _, b3 = self.views(self.params)
        g = self.views(flat_grad)
        l1, l2, l3 = self.layers
        l1.forward(x, w1, b1, out=self.hidden[0], pre=self.pre[0])
        l2.forward(self.hidden[0], w2, b2, out=self.hidden[1], pre=self.pre[1])
        l3.forward(self.hidden[1], w3, b3, out=self.logits)
        cross_entropy(self.logits, targets, loss=self.loss, grad=self.d_logits, grad_scale=1.0 / self.batch)
        self.d_out.copy_(self.d_logits)
        l3.backward(self.d_out, self.hidden[1], w3, dx=self.back[1], dw=g[4], db=g[5])
        l2.backward(self.back[1], self.hidden[0], w2, self.pre[1], dx=self.back[0], dw=g[2], db=g[3])
        l1.backward(self.back[0], x, w1, self.pre[0], dw=g[0], db=g[1])
        return self.loss


class Trainer:
    """`workers` workers and one server with `shards` shards on one GPU, that of `model` where one is given."""

    def __init__(self, batch: int = 80, workers: int = 2, drop_ppm: int = 990_000, state_bits: int = 32, shards: int = 4, hidden: int = 4096,
                 device="cuda:0", seed: int = 0, lr: float = 1e-3, model=None):
        self.model = m = Mlp(batch, device, hidden, seed) if model is None else model     # (another model: see train_lm.py)
        n, device = m.layer_off[-1], m.device
        chunk = -(-n // shards)
        shard_off = [min(j * chunk, n) for j in range(shards + 1)]
        self.lr, self.seed, self.taken = lr, seed, 0
        self.workers = [GradDropSession(m.layer_off, shard_off, drop_ppm, B.GD_SCOPE_PER_LAYER, device=device) for _ in range(workers)]
        self.grad = torch.empty(n, device=device)
        self.dense = torch.empty(n, device=device)
        self.apply = self.workers[0].apply_call(self.workers[0].shard_views(self.dense), 1.0 / workers, [w.push() for w in self.workers])
        decay = [0.01 if len(s) == 2 else 0.0 for s in m.shapes]
        split = lambda t: list(torch.split(t, m.sizes))  # noqa: E731
        self.optimiser = AdamWSession(split(m.params), split(self.dense), copies=split(m.copies), weight_decay=decay, state_bits=state_bits)

    def step(self, batches) -> torch.Tensor:
        """One update from one (x, targets) per worker; returns the mean loss (on the GPU)."""
        losses = []
        for worker, (x, targets) in zip(self.workers, batches):
            losses.append(self.model.gradient(x, targets, self.grad).mean())
            worker.compress(self.grad)
        self.dense.zero_()
        B.gd_decompress_apply(self.apply)
        self.taken += 1
        self.optimiser.step(step=self.taken, lr=self.lr, seed=self.seed + self.taken)
        return torch.stack(losses).mean()


def synthetic_batches(batch: int, workers: int, step: int, device):
    """One (x, targets) per worker: prototypes of ten classes, the same every step, with noise."""
    prototypes = torch.randn(10, 784, generator=W._generator(device, 1), device=device)
    gen = W._generator(device, 1000 + step)
    out = []
    for _ in range(workers):
        targets = torch.randint(10, (batch,), generator=gen, device=device)
        noise = torch.randn(batch, 784, generator=gen, device=device)
        out.append(((prototypes[targets] + 2.0 * noise).to(torch.bfloat16), targets))
    return out


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--batch", type=int, default=80)
    ap.add_argument("--drop-ppm", type=int, default=990_000)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    trainer = Trainer(a.batch, a.workers, a.drop_ppm, a.state_bits)
    for step in range(a.steps):
        loss = trainer.step(synthetic_batches(a.batch, a.workers, step, trainer.model.device))
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step}: loss {loss.item():.4f}")


if __name__ == "__main__":
    main()
