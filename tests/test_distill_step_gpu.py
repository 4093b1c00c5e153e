"""The distillation example: its gradients against fp64's from the activations
that it kept, and its loss over a few steps (GPU)."""
import math

import pytest
import torch

from examples import distill_step as D
from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu


def test_gradients_along_the_chain():
    """Loss and gradients in fp64 from the logits and activations that the
    student's forward pass left.  On the way to a weight the gradient is
    rounded to bf16 four times at most (at the logits, twice at an input, at
    the weight): 2^-8 of its value each, so 2^-6 in the norm."""
    block = D.make_block(width=256, hidden=384, vocab=1003, seed=3)
    student = D.Student(block)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.randn(70, 256, generator=g, device="cuda").to(torch.bfloat16)
    teacher = {n: block[n].to(torch.bfloat16) for n in D.NAMES}
    weight = torch.rand(70, generator=g, device="cuda")
    weight[60:] = 0.0
    targets = api.top_logits(D.forward(x, teacher, block["bias"])[0], 32, temperature=2.0)
    loss, grads = D.distill_step(student, x, targets, weight, 2.0)
    out, kept = D.forward(x, student.r, student.bias)
    api.check_device()

    logits = out.double().requires_grad_(True)
    log_q = torch.log_softmax(logits / 2.0, 1)
    listed = targets["indices"].long()
    p = (targets["values"].double() / 2.0 - targets["lse"].double()[:, None]).exp()
    rest_p = 1.0 - p.sum(1)
    rest = torch.ones_like(log_q, dtype=torch.bool).scatter_(1, listed, False)
    rest_q = torch.logsumexp(log_q.masked_fill(~rest, -math.inf), 1)
    want = (p * (p.log() - log_q.gather(1, listed))).sum(1) + rest_p * (rest_p.log() - rest_q)
    (want * weight.double()).sum().backward()
    live = weight != 0
    assert torch.allclose(loss.double()[live], want[live].detach(), rtol=1e-4, atol=1e-6)
    assert (loss[~live] == 0).all()
    r = {n: student.r[n].double() for n in D.NAMES}
    pre = kept["pre"].double().requires_grad_(True)
    dy = logits.grad @ r["head"]
    torch.nn.functional.silu(pre).backward(dy @ r["down"])
    expected = {"head": logits.grad.t() @ kept["y"].double(), "down": dy.t() @ kept["h"].double(),
                "up": pre.grad.t() @ x.double(), "bias": pre.grad.sum(0)}
    for name, g64 in expected.items():
        off = (grads[name].double() - g64).norm() / g64.norm()
        assert off < 2.0 ** -6, (name, float(off))


def test_the_loss_falls():
    losses = D.train(say=lambda line: None)
    assert all(math.isfinite(v) and v >= 0 for v in losses)
    assert sum(losses[-4:]) < 0.85 * sum(losses[:4]), losses
