"""Training a class-conditional generator on the library, one step as it is used:

  labels -> embedding, added to the noise -> transposed convolutions, each but the last
  followed by group norm with ReLU -> tanh -> images; then the gradients back through
  all of them (data and weight gradients of the convolutions, the norms', the table's)
  and one AdamW step, which also writes the bf16 working weights.

Activations and gradients are bf16 NCHW (the layout of the weight gradients), parameters
and their moments fp32, or the moments in 8 bits with --states 8.  The task is synthetic:
each class has an image of its own to reproduce whatever the noise.

    python examples/conditional_generator.py --steps 200
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1907_11210_amd import huge2 as h2  # noqa: E402
from paper_1907_11210_amd import train  # noqa: E402


class Generator:
    """Parameters and kept objects of a generator of `batch` images of 4 * 2^stages pixels a
    side: noise and label of `dim` values -> channels[0] x 4 x 4 -> ... -> 3 channels."""

    def __init__(self, batch, classes=10, dim=64, channels=(256, 128, 64), groups=16, states=32,
                 seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.batch, self.dim, self.channels = batch, dim, tuple(channels)
        widths = (dim,) + self.channels + (3,)
        # the first layer takes 1 x 1 to 4 x 4, the others double the size
        self.conv = [dict(stride=1, padding=0)] + [dict(stride=2, padding=1)] * len(channels)
        shapes = [(a, b, 4, 4) for a, b in zip(widths, widths[1:])]
        self.embedding = train.Embedding(classes, dim, torch.bfloat16, scale=math.sqrt(dim),
                                         max_tokens=batch)
        self.norms = [train.GroupNorm((batch, c, 4 << i, 4 << i), groups, torch.bfloat16, "NCHW",
                                      "relu") for i, c in enumerate(self.channels)]
        self.stats = [n.new_stats() for n in self.norms]
        # parameters: the table, the convolutions' weights, the norms' gammas and betas
        table = torch.randn(classes, dim, generator=g) / math.sqrt(dim)
        weights = [torch.randn(s, generator=g) * math.sqrt(2 / s[0] / (16 if i == 0 else 4)) *
                   (4 if i == 0 else 1) for i, s in enumerate(shapes)]
        gammas = [torch.ones(c) for c in self.channels]
        betas = [torch.zeros(c) for c in self.channels]
        self.params = [p.to(device) for p in [table] + weights + gammas + betas]
        k = 1 + len(weights)
        self.work = [p.bfloat16() for p in self.params[:k]]  # what the layers read
        norms = len(gammas)
        self.table, self.weights = self.work[0], self.work[1:]
        self.gammas, self.betas = self.params[k:k + norms], self.params[k + norms:]
        self.optimizer = train.AdamW(
            self.params, states, weight_decay=[0.01] * k + [0.0] * (2 * norms),
            copies=self.work + [None] * (2 * norms))
        self.steps = 0

    def forward(self, noise, labels):
        """Images, and what the backward pass reads."""
        e = self.embedding(labels, self.table)
        x = (e + noise).reshape(self.batch, self.dim, 1, 1)
        kept = []
        for i, (w, conv) in enumerate(zip(self.weights, self.conv)):
            y = h2.conv2d_transpose(x, w, **conv)
            kept.append((x, y))
            if i < len(self.norms):
                x = self.norms[i](y, self.gammas[i], self.betas[i], stats=self.stats[i])
        return torch.tanh(y), kept

    def backward(self, dimages, images, kept, labels):
        """Gradients of all parameters, in their order, for the images' error."""
        dy = (dimages * (1 - images * images)).bfloat16()
        dws, dgammas, dbetas = [], [], []
        for i in reversed(range(len(self.weights))):
            x, _ = kept[i]
            w, conv = self.weights[i], self.conv[i]
            dws.append(h2.conv2d_transpose_wgrad(x, dy, w.shape, **conv))
            dx = h2.conv2d_transpose_dgrad(dy, w, **conv)
            if i:
                dy, dgamma, dbeta = self.norms[i - 1].grad(
                    kept[i - 1][1], dx, self.stats[i - 1], self.gammas[i - 1], self.betas[i - 1])
                dgammas.append(dgamma)
                dbetas.append(dbeta)
        dtable = self.embedding.grad(labels, dx.reshape(self.batch, self.dim))
        return [dtable] + dws[::-1] + dgammas[::-1] + dbetas[::-1]

    def step(self, noise, labels, target, lr=2e-3):
        """One training step on the mean square error; its loss (a device tensor)."""
        images, kept = self.forward(noise, labels)
        diff = images.float() - target
        grads = self.backward(diff * (2 / diff.numel()), images, kept, labels)
        self.steps += 1
        self.optimizer.step(grads, lr=lr, step=self.steps, betas=(0.5, 0.99))
        return (diff * diff).mean()


def class_images(classes, size, device="cuda"):
    """A smooth pattern of its own for each class, in [-0.8, 0.8]."""
    at = torch.arange(size, device=device) * (2 * math.pi / size)
    c = torch.arange(classes, device=device)
    rows = torch.sin(at[None] * (1 + c[:, None] % 3) + c[:, None])
    cols = torch.cos(at[None] * (1 + c[:, None] // 3 % 3))
    image = rows[:, None, :, None] * cols[:, None, None, :]
    return 0.8 * torch.cat([image, -image, image.roll(size // 4, 3)], 1)


def train_generator(steps, batch=64, classes=10, states=32, seed=0, report=None):
    gen = Generator(batch, classes, states=states, seed=seed)
    patterns = class_images(classes, 4 << len(gen.channels))
    rng = torch.Generator("cuda").manual_seed(seed)
    losses = []
    for i in range(steps):
        labels = torch.randint(classes, (batch,), generator=rng, device="cuda")
        noise = (0.1 * torch.randn(batch, gen.dim, generator=rng, device="cuda")).bfloat16()
        losses.append(gen.step(noise, labels, patterns[labels]))
        if report and (i + 1) % report == 0:
            print("step %d: loss %.4f" % (i + 1, float(losses[-1])), flush=True)
    return gen, [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawTextHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--classes", type=int, default=10)
    ap.add_argument("--states", type=int, default=32, choices=(32, 8))
    a = ap.parse_args()
    train_generator(a.steps, a.batch, a.classes, a.states, report=20)


if __name__ == "__main__":
    main()
