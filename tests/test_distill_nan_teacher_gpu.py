"""A teacher that is not a number must not train a student on nothing: the
row's loss and gradient are NaN, and no other row changes (GPU)."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan
BF16, F32 = torch.bfloat16, torch.float32


def both_ways(z, indices, values, lse, tau):
    """(loss, gradient, gradient from kept statistics)"""
    made = api.distill_top(z, indices, values, teacher_lse=lse, temperature=tau, stats=True)
    back = api.distill_top_backward(z, indices, values, made["stats"], None, teacher_lse=lse,
                                    temperature=tau)
    api.check_device()
    return made["loss"], made["grad"], back


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("rows,vocab,k", [(7, 300, 1), (7, 4099, 40), (5, 70001, 130)])
def test_nan_reaches_loss_and_gradient(rows, vocab, k, tail, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(vocab)
    z = (torch.randn(rows, vocab, generator=g, device="cuda") * 3.0).to(dtype)
    z[0, vocab // 2:] = -INF                    # also where the student masks
    t = api.top_logits(torch.randn(rows, vocab, generator=g, device="cuda") * 3.0, k, temperature=1.5)
    indices, values, lse = t["indices"], t["values"], t["lse"] if tail else None
    clean = both_ways(z, indices, values, lse, 1.5)
    broken = [0, 2]
    values, lse = values.clone(), lse.clone() if tail else None
    values[0, k // 2] = NAN
    values[2, 0] = INF                          # softmax of an infinite logit is not a number
    if tail:
        lse[2] = INF
        lse[4] = NAN
        broken.append(4)
    whole = [r for r in range(rows) if r not in broken]
    for got, was in zip(both_ways(z, indices, values, lse, 1.5), clean):
        assert torch.isnan(got[broken]).all()
        assert torch.equal(got[whole], was[whole])


@pytest.mark.parametrize("tail", [True, False])
def test_the_value_of_an_absent_entry_is_not_read(tail):
    z = torch.randn(3, 500, device="cuda")
    t = api.top_logits(torch.randn(3, 500, device="cuda"), 20)
    indices, lse = t["indices"], t["lse"] if tail else None
    indices[:, 3] = -1
    indices[:, 7] = 500
    clean = both_ways(z, indices, t["values"], lse, 1.0)
    values = t["values"].clone()
    values[:, 3], values[:, 7] = NAN, INF
    for got, was in zip(both_ways(z, indices, values, lse, 1.0), clean):
        assert torch.equal(got, was)


def test_a_teacher_that_overflowed():
    """Through the call that makes the lists: NaN ranks first and stays."""
    z = torch.randn(4, 3001, device="cuda")
    teacher = torch.randn(4, 3001, device="cuda")
    teacher[1, 77], teacher[2] = NAN, NAN
    t = api.top_logits(teacher, 16)
    for lse in (t["lse"], None):
        for got in both_ways(z, t["indices"], t["values"], lse, 1.0):
            assert torch.isnan(got[1:3]).all() and torch.isfinite(got[[0, 3]]).all()
