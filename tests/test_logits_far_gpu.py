"""Rows whose largest logit is +inf, or so large that the logit over the
temperature, in bits, leaves fp32's range on the way (GPU)."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu
INF = math.inf
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", [(6, 1001), (200, 9003), (6, 90001)])
def test_log_sum_exp(rows, vocab, dtype):
    z = torch.randn(rows, vocab, device="cuda").to(dtype)
    top = torch.finfo(dtype).max
    z[1, vocab - 5] = top
    z[2, 3] = INF
    z[3, vocab // 2:] = INF
    z[4] = 1e30
    z[5] = torch.finfo(dtype).min
    z[5, 9:12] = 2.0 ** 101
    for tau in (1.0, 2.0):
        t = api.top_logits(z, 5, temperature=tau)
        api.check_device()
        want = torch.logsumexp(z.double() / tau, 1)
        big = torch.isfinite(want)
        # (beside logits of 2^100 the sum of the exponentials is below an ulp)
        assert ((t["lse"].double() - want).abs() <= 2.0 ** -22 * want.abs() + 1e-4)[big].all()
        assert torch.equal(t["lse"][2:4], torch.full((2,), INF, device="cuda"))


@pytest.mark.parametrize("tau", [1e-6, 1e-3])
def test_log_sum_exp_at_a_low_temperature(tau):
    """Both the sum and its base are exact here: equal maxima, the rest far below."""
    z = torch.randn(5, 20001, device="cuda")
    z[0, 5:9] = 2.0 ** 90
    z[1, 5:9] = 2.0 ** 100
    z[2] = -2.0 ** 100
    t = api.top_logits(z, 3, temperature=tau)
    api.check_device()
    want = torch.logsumexp(z.double() / float(torch.tensor(tau)), 1)
    assert ((t["lse"].double() - want).abs() <= 2.0 ** -22 * want.abs()).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", [(6, 1001), (200, 9003), (6, 90001)])
def test_distillation(rows, vocab, dtype):
    """All of the student's mass on one far entry, or spread over two or three."""
    g = torch.Generator(device="cuda")
    g.manual_seed(vocab)
    indices = torch.arange(0, 40, 2, dtype=torch.int32, device="cuda").expand(rows, 20).contiguous()
    values = torch.randn(rows, 20, generator=g, device="cuda")
    lse = torch.logsumexp(values, 1) + 0.5
    z = torch.randn(rows, vocab, generator=g, device="cuda").to(dtype)
    top = torch.finfo(dtype).max
    z[0, 1] = top                       # in the rest
    z[1, 2] = top                       # listed
    z[2, [1, vocab - 1]] = top          # two of the rest
    z[3, [3, 4]] = top                  # one of each
    z[4] = top
    p = torch.softmax(values.double(), 1) * math.exp(-0.5)
    rest = 1.0 - math.exp(-0.5)
    q = torch.softmax(z.double(), 1)
    listed = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    listed[indices[0].long()] = True
    q_rest = q[:, ~listed].sum(1)
    share = torch.softmax(z.double().masked_fill(listed, -INF), 1)
    want = share * (q_rest - rest)[:, None]
    want[:, listed] = q[:, listed] - p
    made = api.distill_top(z, indices, values, teacher_lse=lse, stats=True)
    back = api.distill_top_backward(z, indices, values, made["stats"], None, teacher_lse=lse)
    api.check_device()
    tol = (2.0 ** -8 if dtype == BF16 else 2.0 ** -18) * want.abs() + 2.0 ** -20
    assert ((made["grad"].double() - want).abs() <= tol).all()
    # the kept statistics, in fp32, cannot tell logits of that size apart by what q takes
    # to fall to half: the backward call is checked where one entry has all of the rest
    for r in (1, 5):
        assert ((back[r].double() - want[r]).abs() <= tol[r]).all()
    log_q = torch.log_softmax(z.double(), 1)
    log_r = torch.logsumexp(log_q.masked_fill(listed, -INF), 1)
    loss = (p * (p.log() - log_q[:, listed])).sum(1) + rest * (math.log(rest) - log_r)
    inside = loss < 3e38
    assert (made["loss"].double()[~inside] > 1e38).all()
    off = (made["loss"].double() - loss).abs()
    assert (off <= 2.0 ** -18 * loss.abs() + 2.0 ** -18)[inside].all()


def test_an_infinite_student_is_not_a_number():
    z = torch.randn(3, 4001, device="cuda")
    z[0, 7], z[1, 100] = INF, INF
    indices = torch.arange(16, dtype=torch.int32, device="cuda").expand(3, 16).contiguous()
    made = api.distill_top(z, indices, torch.randn(3, 16, device="cuda"), stats=True)
    api.check_device()
    assert torch.isnan(made["loss"][:2]).all() and torch.isnan(made["grad"][:2]).all()
    assert torch.isfinite(made["loss"][2]) and torch.isfinite(made["grad"][2]).all()


SCALES = [1e5, 3e7, 1e9, 1e10, 7.7e12, 1e20, 1e28, 1e30, 3e35]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("rows,vocab", [(2, 1001), (200, 5003), (2, 90001)])
def test_log_sum_exp_of_rows_far_from_zero(rows, vocab, sign, dtype):
    """Masked with one value, or spread about it: a product of the maximum and
    log2(e) / tau has an ulp of its own there."""
    for scale in SCALES:
        for tau in (1.0, 0.7):
            one = torch.full((rows, vocab), sign * scale, device="cuda").to(dtype)
            spread = (one.float() * (1.0 + 0.01 * torch.randn(rows, vocab, device="cuda"))).to(dtype)
            for z in (one, spread):
                t = api.top_logits(z, 4, temperature=tau)
                want = torch.logsumexp(z.double() / float(torch.tensor(tau)), 1)
                tol = 2.0 ** -22 * want.abs() + 1e-4
                assert ((t["lse"].double() - want).abs() <= tol).all(), (scale, tau)
    api.check_device()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("rows,vocab", [(2, 1001), (200, 5003), (2, 90001)])
def test_distillation_of_rows_far_from_zero(rows, vocab, sign, dtype):
    """The whole row, or all of it that is not listed, at one value: q is
    uniform over it.  Then z - lse is exact, and what is left is e = 2^-21 of
    the rounding of a handful of logarithms and of a sum of n ones."""
    indices = torch.arange(0, 60, 3, dtype=torch.int32, device="cuda").expand(rows, 20).contiguous()
    g = torch.Generator(device="cuda")
    g.manual_seed(vocab)
    values = torch.randn(rows, 20, generator=g, device="cuda")
    lse = torch.logsumexp(values, 1) + 0.5
    p = torch.exp(values.double() - lse.double()[:, None])
    rest = 1.0 - p.sum(1)
    listed = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    listed[indices[0].long()] = True
    e = 2.0 ** -21 + (vocab / 512 + 64) * 2.0 ** -24
    for scale in SCALES:
        z = torch.full((rows, vocab), sign * scale, device="cuda").to(dtype)
        made = api.distill_top(z, indices, values, teacher_lse=lse)
        loss = (p * (p.log() + math.log(vocab))).sum(1) + rest * (rest.log() + math.log(vocab / (vocab - 20)))
        assert ((made["loss"].double() - loss).abs() <= 8 * e * (1.0 + math.log(vocab))).all(), scale
        want = torch.full((rows, vocab), 1.0 / vocab, dtype=torch.float64, device="cuda")
        want -= rest[:, None] / (vocab - 20)
        want[:, listed] = 1.0 / vocab - p
        size = torch.full_like(want, 1.0 / vocab)
        size[:, listed] += p
        tol = 8 * e * size + (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0)
        assert ((made["grad"].double() - want).abs() <= tol).all(), scale
        # the list at ordinary values
        z[:, :60:3] = torch.arange(20, device="cuda").to(dtype) / 8
        made = api.distill_top(z, indices, values, teacher_lse=lse)
        q_list = torch.softmax(torch.arange(20, device="cuda").double() / 8, 0)
        q_list = q_list if sign < 0 else torch.zeros_like(q_list)
        want.fill_(0.0)
        want += (((0.0 if sign < 0 else 1.0) - rest) / (vocab - 20))[:, None]
        want[:, listed] = q_list - p
        tol = 8 * e * (1.0 / vocab + want.abs()) + 8 * e * listed + (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0)
        assert ((made["grad"].double() - want).abs() <= tol).all(), scale
        assert (made["loss"] > 0.1 * scale).all()
    api.check_device()
