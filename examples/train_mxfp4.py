"""Trains a small next-token model whose layers multiply in MXFP4, and then serves it token by token.

    python examples/train_mxfp4.py [--steps 200] [--width 256]

The data are sequences of a random Markov chain, so that the loss has a floor (the chain's entropy)
to fall to.  Every product of the layers, forward and backward, runs on 4-bit operands
(``mx.linear``); the weights are fp32 masters that AdamW updates (``optim.AdamWStep``), with the
gradients clipped by their global norm and a step left out whose norm is not finite.  The table of
the embedding is read from the bf16 copy that the step writes.  For serving, the trained weights are
quantised once, and one token at a time goes through products of a single row.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_18112_gb300 import mx, optim  # noqa: E402


class Model:
    """An embedding, `layers` residual blocks of two MXFP4 layers with a ReLU, an output layer."""

    def __init__(self, vocab: int, width: int, layers: int, seed: int):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std):
            return torch.randn(*shape, generator=gen, device="cuda").mul_(std).requires_grad_()

        self.embed = normal(vocab, width, std=1.0)
        self.blocks = [(normal(4 * width, width, std=width ** -0.5),
                        normal(width, 4 * width, std=(8 * width) ** -0.5)) for _ in range(layers)]
        self.out = normal(vocab, width, std=width ** -0.5)

    def params(self):
        return [self.embed, *(w for block in self.blocks for w in block), self.out]

    def forward(self, tokens, table):
        x = torch.nn.functional.embedding(tokens, table)
        for up, down in self.blocks:
            x = x + mx.linear(torch.relu(mx.linear(x, up)), down)
        return mx.linear(x, self.out)


def serve(model: Model, table, tokens):
    """Logits of each token by itself, from weights that were quantised once."""
    with torch.no_grad():
        blocks = [(mx.quantize(up), mx.quantize(down)) for up, down in model.blocks]
        out = mx.quantize(model.out)
        logits = []
        for t in tokens:
            x = table[t:t + 1]
            for up, down in blocks:
                h = torch.relu(mx.matmul(mx.quantize(x), up))
                x = x + mx.matmul(mx.quantize(h), down)
            logits.append(mx.matmul(mx.quantize(x), out))
        return torch.cat(logits)


def train(steps=200, width=256, layers=2, vocab=512, batch=4096, seed=0, lr=2e-3, log=print):
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    chain = torch.softmax(3.0 * torch.randn(vocab, vocab, generator=gen, device="cuda"), 1)
    floor = float(-(chain * chain.log()).sum(1).mean())
    model = Model(vocab, width, layers, seed)
    params = model.params()
    for p in params:
        p.grad = torch.zeros_like(p)
    copies = [p.detach().to(torch.bfloat16) for p in params]
    step = optim.AdamWStep([p.detach() for p in params], [p.grad for p in params],
                           [torch.zeros_like(p) for p in params], [torch.zeros_like(p) for p in params],
                           copies=copies, max_norm=1.0, skip_nonfinite=True)
    losses = []
    for i in range(steps):
        tokens = torch.randint(vocab, (batch,), generator=gen, device="cuda")
        target = torch.multinomial(chain[tokens], 1, generator=gen)[:, 0]
        table = copies[0].detach().requires_grad_()
        logits = model.forward(tokens, table)
        loss = torch.nn.functional.cross_entropy(logits.float(), target)
        for p in params:
            p.grad.zero_()
        loss.backward()
        params[0].grad.copy_(table.grad)
        step(lr * min(1.0, (i + 1) / 20) * 0.5 * (1 + math.cos(math.pi * i / steps)), (0.9, 0.95), 1e-8, 0.01)
        losses.append(loss.detach())
        if log and (i % 50 == 0 or i == steps - 1):
            log(f"step {i:4d}  loss {float(loss.detach()):.4f}  |G| {float(step.record[0]):.3f}  (entropy {floor:.4f})")
    return model, copies, [float(x) for x in losses], floor, step


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--width", type=int, default=256)
    a = ap.parse_args()
    model, copies, losses, floor, step = train(a.steps, a.width)
    tokens = torch.arange(16, device="cuda")
    batch = model.forward(tokens, copies[0]).detach()
    one = serve(model, copies[0], tokens.tolist())
    print(f"steps taken, left out: {step.steps.tolist()}; loss {losses[0]:.3f} -> {losses[-1]:.3f}, entropy {floor:.3f}")
    print("served token by token, the logits differ from the batch's by at most "
          f"{float((batch.float() - one.float()).abs().max()):.3g}")


if __name__ == "__main__":
    main()
