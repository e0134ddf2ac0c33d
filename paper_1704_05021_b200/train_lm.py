"""Training a small language model with dropped gradients, and answering with it token by token.

    python -m paper_1704_05021_b200.train_lm [--steps 60] [--workers 2] [--drop-ppm 990000] [--state-bits 8]

The model is an embedding, some blocks of two skip connections each - layer norm, projection to gate and value, gated linear recurrence,
projection; layer norm, gated feed-forward, projection - a last norm and the projection onto the vocabulary.  Everything runs in the
library: embedding, norms, recurrences and gated blocks through layers.py, the other products and the loss through training.py.  Workers,
exchange and optimiser are train_mlp's.  The data are synthetic: each sentence repeats a random phrase.
"""
from __future__ import annotations

import argparse
from typing import List, Optional

import torch

from . import workloads as W
from .layers import EmbeddingSession, GatedLinearSession, LayerNormSession, recurrence_backward, recurrence_forward, recurrence_marks
from .train_mlp import Trainer
from .training import LinearSession, cross_entropy


class Lm:
    """`blocks` blocks of `width` columns and `hidden` hidden ones over `vocab` words: fp32 parameters in one flat vector, their bf16 copies,
    and what a pass over up to `rows` positions in `sentences` sentences keeps.  All sizes are multiples of 8."""

    def __init__(self, vocab: int, width: int, hidden: int, blocks: int, rows: int, sentences: int, device="cuda:0", seed: int = 0):
        if any(n % 8 for n in (vocab, width, hidden)):
            raise ValueError("vocab, width and hidden are multiples of 8")
        self.vocab, self.width, self.hidden, self.blocks, self.rows, self.sentences = vocab, width, hidden, blocks, rows, sentences
        self.device = dev = torch.device(device)
        d, n = width, hidden
        block = [(d,), (d,), (d, 2 * d), (2 * d,), (d, d), (d,), (d,), (d,), (d, 2 * n), (2 * n,), (n, d), (d,)]
        self.shapes = [(vocab, d)] + block * blocks + [(d,), (d,), (d, vocab), (vocab,)]
        self.sizes = [s[0] * (s[1] if len(s) > 1 else 1) for s in self.shapes]
        self.layer_off = [sum(self.sizes[:i]) for i in range(len(self.sizes) + 1)]
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.params = torch.zeros(self.layer_off[-1], device=dev)
        self.copies = torch.empty_like(self.params, dtype=torch.bfloat16)
        views = self.views(self.params)
        for t, shape in zip(views[1:], self.shapes[1:]):
            if len(shape) == 2:
                t.copy_(torch.randn(shape, generator=gen, device=dev) * shape[0] ** -0.5)
        views[0].copy_(torch.randn(vocab, d, generator=gen, device=dev) * d ** -0.5)
        for b in range(blocks):
            p = self._block(views, b)
            p[0].fill_(1.0), p[6].fill_(1.0)
            p[3][:d].fill_(1.0)                                      # gates that remember a little
        views[-4].fill_(1.0)
        self.copies.copy_(self.params)

        self.scale = d ** 0.5
        self.embedding = EmbeddingSession(vocab, d, rows, device=dev)
        self.norm = LayerNormSession(d, rows, device=dev)
        make = lambda i, o: LinearSession(i, o, rows, device=dev)  # noqa: E731
        self.project, self.join, self.down, self.words = make(d, 2 * d), make(d, d), make(n, d), make(d, vocab)
        self.gated = GatedLinearSession(d, n, rows, device=dev)
        half = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device=dev)  # noqa: E731
        stat = lambda: torch.empty(rows, device=dev)  # noqa: E731
        self.x = [half(rows, d) for _ in range(2 * blocks + 1)]       # the skip connections' rows, before, between and behind the halves of blocks
        self.kept = [dict(a=half(rows, d), z=half(rows, 2 * d), h=half(rows, d), marks=recurrence_marks(rows, sentences, d, dev), c=half(rows, d),
                          pre=half(rows, 2 * n), u=half(rows, n), m1=stat(), r1=stat(), m2=stat(), r2=stat()) for _ in range(blocks)]
        self.f, self.mf, self.rf, self.logits, self.loss = half(rows, d), stat(), stat(), half(rows, vocab), stat()
        self.back = [half(rows, d) for _ in range(3)]
        self.d_z, self.d_u = half(rows, 2 * d), half(rows, n)

    @property
    def layers(self) -> List:
        """The sessions with a status."""
        return [self.project, self.join, self.down, self.words, self.gated]

    def views(self, flat: torch.Tensor) -> List[torch.Tensor]:
        """The tensors of a flat vector."""
        return [t.view(s) for t, s in zip(torch.split(flat, self.sizes), self.shapes)]

    def _block(self, views: List[torch.Tensor], b: int) -> List[torch.Tensor]:
        return views[1 + 12 * b:13 + 12 * b]

    def forward(self, tokens: torch.Tensor, offsets: Optional[torch.Tensor], sentences: int, state: Optional[List[torch.Tensor]] = None,
                marks: bool = False) -> torch.Tensor:
        """The logits of every position.  tokens: the sentences one behind the other, which begin at offsets (None: equal parts); state: one
        [sentences, width] per block, the recurrences' states before the first position, replaced by those behind the last; marks: keep what the
        recurrences' backward pass takes, of up to the model's number of sentences."""
        r, d = len(tokens), self.width
        w, p = self.views(self.copies), self.views(self.params)
        x = [t[:r] for t in self.x]
        self.embedding.forward(w[0], tokens, out=x[0], scale=self.scale)
        for b, k in enumerate(self.kept):
            k = {name: t if name == "marks" else t[:r] for name, t in k.items()}
            (g1, b1, _, bz, _, bo, g2, b2, _, bu, _, bd), (_, _, wz, _, wo, _, _, _, wu, _, wd, _) = self._block(p, b), self._block(w, b)
            self.norm.forward(x[2 * b], g1, b1, out=k["a"], mean=k["m1"], rstd=k["r1"])
            self.project.forward(k["a"], wz, bz, out=k["z"])
            h = None if state is None else state[b]
            recurrence_forward(k["z"][:, :d], k["z"][:, d:], out=k["h"], offsets=offsets, sequences=sentences, h0=h, h_last=h, marks=k["marks"] if marks else None)
            self.join.forward(k["h"], wo, bo, residual=x[2 * b], out=x[2 * b + 1])
            self.norm.forward(x[2 * b + 1], g2, b2, out=k["c"], mean=k["m2"], rstd=k["r2"])
            self.gated.forward(k["c"], wu, bu, out=k["u"], pre=k["pre"])
            self.down.forward(k["u"], wd, bd, residual=x[2 * b + 1], out=x[2 * b + 2])
        self.norm.forward(x[-1], p[-4], p[-3], out=self.f[:r], mean=self.mf[:r], rstd=self.rf[:r])
        return self.words.forward(self.f[:r], w[-2], p[-1], out=self.logits[:r])

    def answer(self, tokens: torch.Tensor, state: List[torch.Tensor]) -> torch.Tensor:
        """The logits behind one more token of each of up to `rows` sentences; `state` (new_state()) moves on."""
        return self.forward(tokens, None, len(tokens), state)

    def new_state(self, sentences: int) -> List[torch.Tensor]:
        return [torch.zeros(sentences, self.width, device=self.device) for _ in range(self.blocks)]

    def gradient(self, batch, targets: torch.Tensor, flat_grad: torch.Tensor) -> torch.Tensor:
        """Forward and backward of the mean loss over the positions of batch = (tokens, offsets): fills flat_grad (fp32, laid out like the
        parameters); returns the positions' losses.  Positions with the target -100 count for nothing."""
        tokens, offsets = batch
        r, d, sentences = len(tokens), self.width, len(offsets) - 1
        logits = self.forward(tokens, offsets, sentences, marks=True)
        cross_entropy(logits, targets, loss=self.loss[:r], grad=logits, grad_scale=1.0 / r)
        w, p, g = self.views(self.copies), self.views(self.params), self.views(flat_grad)
        x = [t[:r] for t in self.x]
        dx, between, inner = (t[:r] for t in self.back)
        dz, du = self.d_z[:r], self.d_u[:r]
        self.words.backward(logits, self.f[:r], w[-2], dx=inner, dw=g[-2], db=g[-1])
        self.norm.backward(inner, x[-1], p[-4], self.mf[:r], self.rf[:r], dx=dx, dweight=g[-4], dbias=g[-3])
        for b in reversed(range(self.blocks)):
            k = {name: t if name == "marks" else t[:r] for name, t in self.kept[b].items()}
            (g1, _, _, _, _, _, g2, _, _, _, _, _), (_, _, wz, _, wo, _, _, _, wu, _, wd, _) = self._block(p, b), self._block(w, b)
            dg1, db1, dwz, dbz, dwo, dbo, dg2, db2, dwu, dbu, dwd, dbd = self._block(g, b)
            self.down.backward(dx, k["u"], wd, dx=du, dw=dwd, db=dbd)
            self.gated.backward(du, k["c"], wu, k["pre"], dx=inner, dw=dwu, db=dbu)
            self.norm.backward(inner, x[2 * b + 1], g2, k["m2"], k["r2"], dx=between, add=dx, dweight=dg2, dbias=db2)
            self.join.backward(between, k["h"], wo, dx=inner, dw=dwo, db=dbo)
            recurrence_backward(inner, k["z"][:, :d], k["z"][:, d:], k["marks"], dz[:, :d], dz[:, d:], offsets=offsets, sequences=sentences)
            self.project.backward(dz, k["a"], wz, dx=inner, dw=dwz, db=dbz)
            self.norm.backward(inner, x[2 * b], g1, k["m1"], k["r1"], dx=dx, add=between, dweight=dg1, dbias=db1)
        self.embedding.backward(dx, tokens, g[0], scale=self.scale)
        return self.loss[:r]


def synthetic_batches(vocab: int, rows: int, sentences: int, workers: int, step: int, device):
    """One ((tokens, offsets), targets) per worker: sentences of many lengths, each a random phrase of up to eight words over and over; the target
    is the next word, the last position has none."""
    gen = W._generator(device, 2000 + step)
    out = []
    for _ in range(workers):
        cuts = torch.rand(sentences - 1, generator=gen, device=device).sort().values
        offsets = torch.cat([torch.zeros(1, device=device), (cuts * rows).floor(), torch.full((1,), float(rows), device=device)]).long()
        at = torch.arange(rows, device=device)
        whose = torch.searchsorted(offsets[1:].contiguous(), at, right=True)
        period = torch.randint(2, 9, (sentences,), generator=gen, device=device)
        phrases = torch.randint(vocab, (sentences, 8), generator=gen, device=device)
        tokens = phrases[whose, (at - offsets[whose]) % period[whose]]
        targets = torch.cat([tokens[1:], tokens[:1]])
        targets[at + 1 == offsets[whose + 1]] = -100
        out.append(((tokens, offsets), targets))
    return out


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--rows", type=int, default=4000)
    ap.add_argument("--sentences", type=int, default=80)
    ap.add_argument("--vocab", type=int, default=8000)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--drop-ppm", type=int, default=990_000)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    model = Lm(a.vocab, a.width, a.hidden, a.blocks, a.rows, a.sentences)
    trainer = Trainer(workers=a.workers, drop_ppm=a.drop_ppm, state_bits=a.state_bits, model=model)
    for step in range(a.steps):
        loss = trainer.step(synthetic_batches(a.vocab, a.rows, a.sentences, a.workers, step, model.device))
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step}: loss {loss.item():.4f}")
    # the last step's first sentence once more, word by word
    (tokens, _), _ = synthetic_batches(a.vocab, a.rows, a.sentences, 1, a.steps - 1, model.device)[0]
    state, said = model.new_state(1), []
    word = tokens[:1]
    for _ in range(16):
        word = model.answer(word, state).argmax(1)
        said.append(word)
    print("answers", torch.cat(said).tolist())


if __name__ == "__main__":
    main()
