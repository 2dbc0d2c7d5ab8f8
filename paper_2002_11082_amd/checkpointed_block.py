"""A gated block, trained with everything the package has and then served: python -m paper_2002_11082_amd.checkpointed_block

  y = (silu(x Wg^T) * (x Wu^T)) Wd^T

Every worker runs its share of the tokens, in two parts whose gradients are added up.  What the backward pass needs of a part waits in 8 bits: x and the
activation's result (ogq_group_quantize), and the activation's inputs (ogq_activation_forward).  The weight gradients come from there (ogq_weight_gradient)
straight into the worker's flat fp32 gradient, which is quantized for sending (ogq_quantize); the average of all workers' streams (ogq_dequantize_average)
moves the weights.  In the end the weights are laid out in 4 bits and answer tokens (ogq_group_matvec).

The workers are simulated one after the other on one GPU, the targets come from a block of random weights, of which the trained one starts as a disturbed
copy, and the products with the weights themselves are torch's.  Needs a GPU; everything is seeded."""
from __future__ import annotations

import argparse
import math

import torch

import paper_2002_11082_amd as ogq

GROUP = ogq.make_group_params(32, 8)
SERVED = ogq.make_group_params(32, 4)


class Block:
    """Weights in fp32 as views of one flat tensor, and in bf16 for the products."""

    def __init__(self, width: int, hidden: int, seed: int):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.shapes = {"gate": (hidden, width), "up": (hidden, width), "down": (width, hidden)}
        self.flat = torch.empty(3 * width * hidden, device="cuda")
        for name, w in self.views(self.flat).items():
            w.normal_(0.0, 1.0 / math.sqrt(self.shapes[name][1]), generator=gen)
        self.refresh()

    def views(self, flat):
        parts = flat.split([rows * cols for rows, cols in self.shapes.values()])
        return {name: part.view(shape) for (name, shape), part in zip(self.shapes.items(), parts)}

    def refresh(self):
        self.half = {name: w.bfloat16() for name, w in self.views(self.flat).items()}

    def plain(self, x):
        """The block's answer in fp32 from the fp32 weights."""
        w = self.views(self.flat)
        g = x.float() @ w["gate"].t()
        return (g * torch.sigmoid(g) * (x.float() @ w["up"].t())) @ w["down"].t()

    def forward(self, x):
        """The answer to x [tokens, width] in bf16 and what the backward pass needs, in 8 bits."""
        y, *inner = ogq.ogq_activation_forward(x @ self.half["gate"].t(), ogq.SILU, GROUP, x @ self.half["up"].t())
        kept = (ogq.ogq_group_quantize(x, GROUP), inner, ogq.ogq_group_quantize(y, GROUP))
        return y @ self.half["down"].t(), kept

    def backward(self, dz, kept, gradient):
        """Adds the weights' gradients to the flat `gradient`."""
        x, (codes, exponents, up_codes, up_exponents), y = kept
        width, hidden = self.shapes["down"]
        into = self.views(gradient)
        ogq.ogq_weight_gradient(dz, *y, hidden, GROUP, into["down"], accumulate=True)
        dgate, dup = ogq.ogq_activation_backward(dz @ self.half["down"], ogq.SILU, codes, exponents, GROUP, up_codes, up_exponents)
        ogq.ogq_weight_gradient(dgate, *x, width, GROUP, into["gate"], accumulate=True)
        ogq.ogq_weight_gradient(dup, *x, width, GROUP, into["up"], accumulate=True)


class Served:
    """A block's weights in 4 bits."""

    def __init__(self, block: Block):
        self.shapes = block.shapes
        self.held = {name: ogq.ogq_group_quantize(w, SERVED) for name, w in block.views(block.flat).items()}

    def __call__(self, x):
        width, hidden = self.shapes["down"]
        gate = ogq.ogq_group_matvec(*self.held["gate"], width, SERVED, x)
        up = ogq.ogq_group_matvec(*self.held["up"], width, SERVED, x)
        return ogq.ogq_group_matvec(*self.held["down"], hidden, SERVED, gate * torch.sigmoid(gate) * up)


def held_bytes(kept):
    """(bytes of what waits for the backward pass, what it would be in bf16)"""
    x, inner, y = kept
    codes = [x[0], inner[0], inner[2], y[0]]
    exponents = [x[1], inner[1], inner[3], y[1]]
    return sum(t.numel() for t in codes + exponents), sum(2 * t.numel() for t in codes)


def train(width=512, hidden=1024, tokens=256, workers=2, steps=60, rate=20.0, seed=0, tell=print):
    """Returns the loss before every step and the trained block."""
    teacher, block = Block(width, hidden, seed + 1), Block(width, hidden, seed + 2)
    block.flat.mul_(0.5).add_(teacher.flat)
    block.refresh()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    gradient = torch.empty_like(block.flat)
    losses = []
    for step in range(steps):
        streams, total = [], torch.zeros((), device="cuda")
        for worker in range(workers):
            gradient.zero_()
            for _ in range(2):
                x = torch.randn(tokens // 2, width, generator=gen, device="cuda").bfloat16()
                z, kept = block.forward(x)
                error = z.float() - teacher.plain(x)
                total += error.square().mean() / (2 * workers)
                block.backward((error * (2.0 / tokens)).bfloat16(), kept, gradient)
            params = ogq.make_params(2048, 3, ogq.ORQ, level_iters=2, seed=seed + 1000 * step + worker)
            streams.append(ogq.ogq_quantize(gradient, params))
        average = ogq.ogq_dequantize_average([codes for _, codes in streams], [levels for levels, _ in streams], gradient.numel(), params)
        block.flat.sub_(average, alpha=rate / width)
        block.refresh()
        losses.append(float(total))
        if step % 10 == 0 or step == steps - 1:
            held, plain = held_bytes(kept)
            tell(f"step {step}: loss {losses[-1]:.4f}, held for the backward pass {held / 1e6:.2f} MB ({plain / 1e6:.2f} in bf16)")
    return losses, block


def main():
    parser = argparse.ArgumentParser(description="Trains a gated block with 8-bit checkpoints and quantized gradients, then serves it from 4-bit weights.")
    parser.add_argument("--width", type=int, default=512)
    parser.add_argument("--hidden", type=int, default=1024)
    parser.add_argument("--tokens", type=int, default=256, help="of a worker and step")
    parser.add_argument("--workers", type=int, default=2)
    parser.add_argument("--steps", type=int, default=60)
    a = parser.parse_args()
    _, block = train(a.width, a.hidden, a.tokens, a.workers, a.steps)
    served = Served(block)
    for tokens in (1, 16):
        x = torch.randn(tokens, a.width, generator=torch.Generator(device="cuda").manual_seed(tokens), device="cuda").bfloat16()
        exact = block.plain(x)
        print(f"{tokens} token(s) from 4-bit weights: off by {float((served(x).float() - exact).norm() / exact.norm()):.3f} of the answer's norm")


if __name__ == "__main__":
    main()
