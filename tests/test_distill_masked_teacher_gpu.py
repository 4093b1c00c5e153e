"""A teacher row of nothing but -inf, as the top lists hand it on: values and
log-sum-exp -inf.  It has no mass, so loss and gradient are 0 (GPU)."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu
INF = math.inf


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("rows,vocab,k", [(4, 3, 3), (4, 1000, 1), (6, 5003, 64), (3, 80001, 200)])
def test_masked_teacher_row(rows, vocab, k, tail, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(vocab + k)
    teacher = (torch.randn(rows, vocab, generator=g, device="cuda") * 3.0).to(dtype)
    z = (torch.randn(rows, vocab, generator=g, device="cuda") * 3.0).to(dtype)
    weight = torch.rand(rows, generator=g, device="cuda") + 0.1

    def run(t):
        lse = t["lse"] if tail else None
        made = api.distill_top(z, t["indices"], t["values"], teacher_lse=lse, row_weight=weight,
                               stats=True)
        back = api.distill_top_backward(z, t["indices"], t["values"], made["stats"], weight,
                                        teacher_lse=lse)
        api.check_device()
        return made["loss"], made["grad"], back

    clean = run(api.top_logits(teacher, k))
    teacher[1] = -INF
    t = api.top_logits(teacher, k)
    assert float(t["lse"][1]) == -INF and (t["values"][1] == -INF).all()
    rest = [r for r in range(rows) if r != 1]
    for got, was in zip(run(t), clean):
        assert (got[1] == 0).all()
        assert torch.equal(got[rest], was[rest])
    # absent entries of such a row change nothing
    t["indices"][1, 0] = -1
    for got in run(t):
        assert (got[1] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_student_row_masked_as_well(dtype):
    z = torch.full((2, 2001), -INF, dtype=dtype, device="cuda")
    z[1] = torch.randn(2001, device="cuda").to(dtype)
    t = api.top_logits(z, 8)
    made = api.distill_top(z, t["indices"], t["values"], teacher_lse=t["lse"])
    api.check_device()
    assert float(made["loss"][0]) == 0.0 and not made["grad"][0].any()
    assert torch.isfinite(made["grad"]).all() and torch.isfinite(made["loss"]).all()
