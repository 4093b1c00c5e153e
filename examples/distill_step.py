"""Quantisation-aware distillation of a small block, every step of it on the
library's kernels:

    teacher   logits -> top_logits              (k logits a token, and the rest's mass)
    student   linear with r, r, r -> logits     (r: the INT3 reconstruction)
    loss      distill_top                       (and the gradient, in the logits' place)
    backward  linear_backward                   (dr is the g of the reconstruction)
    update    adamw_recon_int_batch             (w', m', v' and the next r)

    python examples/distill_step.py [--steps N]

The block is an MLP with a residual and a head: h = silu(x Up^T + b), y = x +
h Down^T, logits = y Head^T.  The teacher is the same block in full precision;
the student starts from the teacher's weights, disturbed, and reconstructed in 3
bits.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_13966_gb300 import api  # noqa: E402

CLIP = [1.0, 0.95, 0.9, 0.85, 0.8, 0.75, 0.7, 0.65]
GROUP = 128
NAMES = ("up", "down", "head")


def make_block(width=512, hidden=1408, vocab=8003, seed=0):
    """The teacher's fp32 weights and bias."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    draw = lambda rows, cols: torch.randn(rows, cols, generator=g, device="cuda") / cols ** 0.5  # noqa: E731
    return {"up": draw(hidden, width), "down": draw(width, hidden), "head": 4.0 * draw(vocab, width),
            "bias": 0.1 * torch.randn(hidden, generator=g, device="cuda")}


def forward(x, r, bias):
    """Logits of the block and what its backward pass needs."""
    up = api.linear(x, r["up"], bias=bias, activation="silu", save_pre=True)
    y = api.linear(up["y"], r["down"], residual=x)["y"]
    return api.linear(y, r["head"])["y"], {"x": x, "pre": up["pre"], "h": up["y"], "y": y}


def backward(dlogits, kept, r):
    """The weights' and the bias's gradients from the logits'."""
    head = api.linear_backward(dlogits, kept["y"], r["head"])
    down = api.linear_backward(head["dx"], kept["h"], r["down"], pre_in=kept["pre"],
                               activation_in="silu")
    up = api.linear_backward(down["dx"], kept["x"], r["up"], dx=False, bias=True)
    return {"head": head["dr"], "down": down["dr"], "up": up["dr"], "bias": up["dbias"]}


class Student:
    """Latent weights with their moments, and the reconstruction r that the
    forward pass reads."""

    def __init__(self, block, disturbed=0.0, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.bias = block["bias"].clone()
        self.w = {n: block[n] + disturbed * block[n].std() *
                  torch.randn(block[n].shape, generator=g, device="cuda") for n in NAMES}
        self.m = {n: torch.zeros_like(w) for n, w in self.w.items()}
        self.v = {n: torch.full_like(w, 1e-12) for n, w in self.w.items()}
        made = api.recon_int_batch([(self.w[n], None, self.v[n]) for n in NAMES], bits=3,
                                   group_size=GROUP, clip=CLIP)
        self.r = {n: o["r"] for n, o in zip(NAMES, made)}
        self.steps = 0

    def update(self, g, lr):
        """One AdamW step and the reconstruction of the updated weights."""
        self.steps += 1
        items = [(self.w[n], g[n], self.m[n], self.v[n]) for n in NAMES]
        made = api.adamw_recon_int_batch(items, lr=lr, step=self.steps, bits=3, group_size=GROUP,
                                         clip=CLIP)
        self.r = {n: o["r"] for n, o in zip(NAMES, made)}
        self.bias -= lr * g["bias"]


def distill_step(student, x, targets, row_weight, temperature):
    """Loss a token and the gradients of sum(row_weight * loss)."""
    logits, kept = forward(x, student.r, student.bias)
    wide = -(-logits.shape[1] // 8) * 8  # rows the products can read
    dlogits = torch.empty(logits.shape[0], wide, dtype=logits.dtype,
                          device=logits.device)[:, :logits.shape[1]]
    made = api.distill_top(logits, targets["indices"], targets["values"], teacher_lse=targets["lse"],
                           row_weight=row_weight, temperature=temperature, out=dlogits)
    return made["loss"], backward(dlogits, kept, student.r)


def train(steps=60, tokens=512, k=64, temperature=2.0, lr=1e-3, seed=0, say=print):
    """Losses (mean over the tokens that count), step by step."""
    block = make_block(seed=seed)
    teacher = {n: block[n].to(torch.bfloat16) for n in NAMES}
    student = Student(block, disturbed=0.7, seed=seed + 2)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    losses = []
    for step in range(steps):
        x = torch.randn(tokens, block["up"].shape[1], generator=g, device="cuda").to(torch.bfloat16)
        live = (torch.arange(tokens, device="cuda") < tokens - 7).float()  # the last few are padding
        row_weight = live / live.sum()
        targets = api.top_logits(forward(x, teacher, block["bias"])[0], k, temperature=temperature)
        loss, grads = distill_step(student, x, targets, row_weight, temperature)
        student.update(grads, lr)
        losses.append(float((loss * row_weight).sum()))
        say(f"step {step:3d}  loss {losses[-1]:.5f}")
    api.check_device()
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=60)
    train(parser.parse_args().steps)
