"""Quantisation-aware distillation of a small transformer, every step of it on the
library's kernels:

    tokens    embedding (and positions)            -> the stream h
    block     layer_norm -> linear qkv -> attention -> linear + h
              layer_norm -> linear up, silu -> linear down + h
    head      layer_norm -> linear                 -> logits
    loss      distill_top from a teacher's top_logits
    backward  the same calls' gradients, back to the tables of the embedding
    update    adamw_recon_int_batch for the quantised projections

    python examples/transformer_step.py [--steps N]

Sequences of different lengths are packed into one batch; the rows behind the
last are padding (no token, no sequence, weight 0).  As in the paper's setting the
projections of the blocks are quantised, embedding, head and norms are not.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_13966_gb300 import api  # noqa: E402

CLIP = [1.0, 0.95, 0.9, 0.85, 0.8, 0.75, 0.7, 0.65]
QUANTISED = ("qkv", "out", "up", "down")


class Shape:
    def __init__(self, vocab=5003, width=512, heads=8, kv_heads=2, head_dim=64, hidden=1408, layers=2,
                 longest=256):
        self.vocab, self.width, self.heads, self.kv_heads = vocab, width, heads, kv_heads
        self.head_dim, self.hidden, self.layers, self.longest = head_dim, hidden, layers, longest
        self.widths = [heads * head_dim, kv_heads * head_dim, kv_heads * head_dim]


def make_weights(s, seed=0):
    """fp32 weights: the tables, the head, the norms and each layer's projections."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    draw = lambda rows, cols, gain=1.0: gain * torch.randn(rows, cols, generator=g, device="cuda") / cols ** 0.5  # noqa: E731
    w = {"tokens": draw(s.vocab, s.width) * s.width ** 0.5 * 0.3, "places": draw(s.longest, s.width) * 0.1,
         "head": draw(s.vocab, s.width, 4.0), "norm": torch.ones(s.width, device="cuda")}
    for i in range(s.layers):
        w[f"qkv{i}"] = draw(sum(s.widths), s.width)
        w[f"out{i}"] = draw(s.width, s.widths[0])
        w[f"up{i}"], w[f"down{i}"] = draw(s.hidden, s.width), draw(s.width, s.hidden)
        w[f"norm1{i}"], w[f"norm2{i}"] = (torch.ones(s.width, device="cuda") for _ in range(2))
    return w


def quantised(s):
    return [f"{n}{i}" for i in range(s.layers) for n in QUANTISED]


def forward(s, r, ids, places, starts):
    """Logits of the packed tokens, and what the backward pass needs.  r: the bf16 matrices
    (reconstructions, tables, head) and the fp32 weights of the norms."""
    kept = {}
    h = api.embedding(places, r["places"])
    h = api.embedding(ids, r["tokens"], residual=h)
    for i in range(s.layers):
        n1 = api.layer_norm(h, r[f"norm1{i}"], center=False, stats=True)
        qkv = api.linear(n1["y"], r[f"qkv{i}"])["y"]
        a = api.attention(*qkv.split(s.widths, 1), s.head_dim, starts=starts, lse=True)
        h1 = api.linear(a["y"], r[f"out{i}"], residual=h)["y"]
        n2 = api.layer_norm(h1, r[f"norm2{i}"], center=False, stats=True)
        up = api.linear(n2["y"], r[f"up{i}"], activation="silu", save_pre=True)
        kept[i] = {"h": h, "n1": n1, "qkv": qkv, "a": a, "h1": h1, "n2": n2, "up": up}
        h = api.linear(up["y"], r[f"down{i}"], residual=h1)["y"]
    n = api.layer_norm(h, r["norm"], center=False, stats=True)
    kept["h"], kept["n"] = h, n
    return api.linear(n["y"], r["head"])["y"], kept


def backward(s, dlogits, kept, r, ids, places, starts):
    """The gradients of every matrix and norm from the logits'."""
    g = {}
    made = api.linear_backward(dlogits, kept["n"]["y"], r["head"])
    g["head"] = made["dr"]
    made = api.layer_norm_backward(made["dx"], kept["h"], r["norm"], kept["n"]["stats"], center=False)
    dh, g["norm"] = made["dx"], made["dweight"]
    for i in reversed(range(s.layers)):
        k = kept[i]
        made = api.linear_backward(dh, k["up"]["y"], r[f"down{i}"], pre_in=k["up"]["pre"],
                                   activation_in="silu")
        g[f"down{i}"] = made["dr"]
        made = api.linear_backward(made["dx"], k["n2"]["y"], r[f"up{i}"])
        g[f"up{i}"] = made["dr"]
        made = api.layer_norm_backward(made["dx"], k["h1"], r[f"norm2{i}"], k["n2"]["stats"],
                                       center=False, residual=dh)
        dh1, g[f"norm2{i}"] = made["dx"], made["dweight"]
        made = api.linear_backward(dh1, k["a"]["y"], r[f"out{i}"])
        g[f"out{i}"] = made["dr"]
        dqkv = torch.empty_like(k["qkv"])
        api.attention_backward(made["dx"], *k["qkv"].split(s.widths, 1), k["a"]["y"], k["a"]["lse"],
                               s.head_dim, starts=starts, out=dqkv.split(s.widths, 1))
        made = api.linear_backward(dqkv, k["n1"]["y"], r[f"qkv{i}"])
        g[f"qkv{i}"] = made["dr"]
        made = api.layer_norm_backward(made["dx"], k["h"], r[f"norm1{i}"], k["n1"]["stats"],
                                       center=False, residual=dh1)
        dh, g[f"norm1{i}"] = made["dx"], made["dweight"]
    g["tokens"] = api.embedding_backward(dh, ids, s.vocab)
    g["places"] = api.embedding_backward(dh, places, s.longest)
    return g


def pack(s, lengths, tokens, seed=0):
    """A batch of sequences: ids, places (-1: padding) and where each starts."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = torch.full((tokens,), -1, dtype=torch.int32, device="cuda")
    places, starts, at = ids.clone(), [0], 0
    for n in lengths:
        ids[at:at + n] = torch.randint(0, s.vocab, (n,), generator=g, device="cuda").to(torch.int32)
        places[at:at + n] = torch.arange(n, device="cuda", dtype=torch.int32)
        at += n
        starts.append(at)
    return ids, places, torch.tensor(starts, dtype=torch.int32, device="cuda")


class Student:
    """Latent weights with their moments, and what the forward pass reads: the
    reconstructions, and the others in bf16."""

    def __init__(self, s, weights, disturbed=0.0, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.s, self.steps = s, 0
        self.w = {n: w.clone() for n, w in weights.items()}
        for n in quantised(s):
            self.w[n] += disturbed * self.w[n].std() * torch.randn(self.w[n].shape, generator=g, device="cuda")
        names = quantised(s)
        self.m = {n: torch.zeros_like(self.w[n]) for n in names}
        self.v = {n: torch.full_like(self.w[n], 1e-12) for n in names}
        made = api.recon_int_batch([(self.w[n], None, self.v[n]) for n in names], bits=4, group_size=64,
                                   clip=CLIP)
        self.r = self._others() | {n: o["r"] for n, o in zip(names, made)}

    def _others(self):
        return {n: w.to(torch.bfloat16) if w.dim() == 2 else w for n, w in self.w.items() if n not in self.m}

    def update(self, g, lr):
        self.steps += 1
        names = quantised(self.s)
        made = api.adamw_recon_int_batch([(self.w[n], g[n], self.m[n], self.v[n]) for n in names], lr=lr,
                                         step=self.steps, bits=4, group_size=64, clip=CLIP)
        for n in self.w:
            if n not in self.m:
                self.w[n] -= lr * g[n].float()
        self.r = self._others() | {n: o["r"] for n, o in zip(names, made)}


def distill_step(s, r, batch, targets, row_weight, temperature):
    """Loss a token and the gradients of sum(row_weight * loss)."""
    ids, places, starts = batch
    logits, kept = forward(s, r, ids, places, starts)
    wide = -(-logits.shape[1] // 8) * 8  # rows the products can read
    dlogits = torch.empty(logits.shape[0], wide, dtype=logits.dtype,
                          device=logits.device)[:, :logits.shape[1]]
    made = api.distill_top(logits, targets["indices"], targets["values"], teacher_lse=targets["lse"],
                           row_weight=row_weight, temperature=temperature, out=dlogits)
    return made["loss"], dlogits, kept, backward(s, dlogits, kept, r, ids, places, starts)


def train(steps=30, k=64, temperature=2.0, lr=1e-3, seed=0, shape=None, say=print):
    """Losses (mean over the tokens that count), step by step."""
    s = shape or Shape()
    weights = make_weights(s, seed)
    teacher = {n: w.to(torch.bfloat16) if w.dim() == 2 else w for n, w in weights.items()}
    student = Student(s, weights, disturbed=0.5, seed=seed + 1)
    losses = []
    for step in range(steps):
        lengths = [(37 * (step + 1) * i) % (s.longest - 1) + 1 for i in range(1, 5)]
        tokens = 4 * s.longest
        batch = pack(s, lengths, tokens, seed=seed + step)
        live = (torch.arange(tokens, device="cuda") < sum(lengths)).float()
        row_weight = live / live.sum()
        targets = api.top_logits(forward(s, teacher, *batch)[0], k, temperature=temperature)
        loss, _, _, grads = distill_step(s, student.r, batch, targets, row_weight, temperature)
        student.update(grads, lr)
        losses.append(float((loss * row_weight).sum()))
        say(f"step {step:3d}  loss {losses[-1]:.5f}")
    api.check_device()
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=30)
    train(parser.parse_args().steps)
