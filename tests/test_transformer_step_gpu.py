"""The operators run together: a packed, padded batch through the transformer of the
example and back, its gradients against fp64's at the activations that it kept (GPU)."""
import math

import pytest
import torch

from examples import transformer_step as T
from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu


def at(value, kept):
    """`value` in fp64, held to the activation that was kept: its gradient passes."""
    return value + (kept.double() - value).detach()


def forward64(s, w, batch, kept):
    ids, places, starts = batch
    live = (ids >= 0)[:, None]
    h = torch.where(live, w["tokens"][ids.long().clamp(min=0)] + w["places"][places.long().clamp(min=0)], 0.0)
    norm = lambda x, g: x * (x.square().mean(1, keepdim=True) + 1e-5).rsqrt() * g  # noqa: E731
    for i in range(s.layers):
        k = kept[i]
        h = at(h, k["h"])
        n1 = at(norm(h, w[f"norm1{i}"]), k["n1"]["y"])
        qkv = at(n1 @ w[f"qkv{i}"].t(), k["qkv"])
        a = torch.zeros(ids.shape[0], s.widths[0], dtype=torch.float64, device="cuda")
        for from_, to in zip(starts.tolist(), starts.tolist()[1:]):
            q, kk, v = (t.view(to - from_, -1, s.head_dim).transpose(0, 1)
                        for t in qkv[from_:to].split(s.widths, 1))
            kk, v = (t.repeat_interleave(s.heads // s.kv_heads, 0) for t in (kk, v))
            score = (q @ kk.transpose(1, 2) * s.head_dim ** -0.5).masked_fill(
                ~torch.ones(to - from_, to - from_, dtype=torch.bool, device="cuda").tril(), -math.inf)
            y = (torch.softmax(score, 2) @ v).transpose(0, 1).reshape(to - from_, -1)
            a = torch.cat([a[:from_], y, a[to:]])
        a = at(a, k["a"]["y"])
        h1 = at(h + a @ w[f"out{i}"].t(), k["h1"])
        n2 = at(norm(h1, w[f"norm2{i}"]), k["n2"]["y"])
        pre = at(n2 @ w[f"up{i}"].t(), k["up"]["pre"])
        up = at(torch.nn.functional.silu(pre), k["up"]["y"])
        h = h1 + up @ w[f"down{i}"].t()
    h = at(h, kept["h"])
    return at(norm(h, w["norm"]), kept["n"]["y"]) @ w["head"].t()


def test_gradients_along_the_chain():
    """On the way from the logits to the embedding a gradient is rounded to bf16 at most 11
    times (at the logits, an input or a norm's output each time, at the matrix) and passes three
    more roundings in attention (probabilities, ds, y): 2^-8 of its value each, so 14 x 2^-8 in
    the norm, where a later product spreads an earlier rounding as it spreads the gradient."""
    s = T.Shape(vocab=1003, width=256, heads=6, kv_heads=2, head_dim=64, hidden=384, layers=1, longest=160)
    student = T.Student(s, T.make_weights(s, seed=3))
    batch = T.pack(s, [150, 1, 70, 129], 400, seed=4)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    weight = torch.rand(400, generator=g, device="cuda")
    weight[350:] = 0.0
    other = T.make_weights(s, seed=5)
    teacher = {n: w.to(torch.bfloat16) if w.dim() == 2 else w for n, w in other.items()}
    targets = api.top_logits(T.forward(s, teacher, *batch)[0], 32, temperature=2.0)
    loss, dlogits, kept, grads = T.distill_step(s, student.r, batch, targets, weight, 2.0)
    api.check_device()
    assert (loss[350:] == 0).all() and loss.isfinite().all()
    assert all(v.isfinite().all() for v in grads.values())
    w = {n: r.double().requires_grad_(True) for n, r in student.r.items()}
    logits = forward64(s, w, batch, kept)
    logits.backward(dlogits.double())
    for name, t in w.items():
        off = (grads[name].double() - t.grad).norm() / t.grad.norm()
        assert off < 14 * 2.0 ** -8, (name, float(off))
    # rows of tables that no token has
    unused = torch.ones(s.vocab, dtype=torch.bool, device="cuda")
    unused[batch[0][:350].long()] = False
    assert (grads["tokens"][unused] == 0).all()


def test_captured_step():
    """Forward and backward pass of a step in one graph, replayed with other sequences."""
    s = T.Shape(vocab=1003, width=256, heads=4, kv_heads=4, head_dim=64, hidden=384, layers=2, longest=160)
    student = T.Student(s, T.make_weights(s, seed=3))
    batch = T.pack(s, [150, 1, 70, 129], 400, seed=4)
    weight = torch.ones(400, device="cuda")
    targets = api.top_logits(T.forward(s, student.r, *batch)[0], 32, temperature=2.0)
    run = lambda: T.distill_step(s, student.r, batch, targets, weight, 2.0)  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, _, _, grads = run()
    for to, now in zip(batch, T.pack(s, [3, 140, 160, 90], 400, seed=9)):
        to.copy_(now)
    graph.replay()
    torch.cuda.synchronize()
    want_loss, _, _, want = run()
    assert torch.equal(loss, want_loss)
    assert all(torch.equal(grads[n], want[n]) for n in want)


def test_it_runs():
    losses = T.train(steps=3, shape=T.Shape(vocab=1003, width=256, heads=4, kv_heads=2, head_dim=64, hidden=384,
                                            layers=2, longest=96), say=lambda line: None)
    assert len(losses) == 3 and all(math.isfinite(v) and v >= 0 for v in losses)
