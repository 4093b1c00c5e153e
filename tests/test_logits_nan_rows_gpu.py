"""NaN among a student's or a teacher's logits where everything beside it is
masked with -inf: the row's sum is not a number, whatever its maximum (GPU)."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", [(6, 1001), (200, 9003), (6, 90001)])
def test_log_sum_exp(rows, vocab, dtype):
    z = torch.full((rows, vocab), -INF, dtype=dtype, device="cuda")
    z[1, vocab - 2] = NAN
    z[2, 0] = NAN
    z[2, vocab // 2:] = torch.randn(vocab - vocab // 2, device="cuda").to(dtype)
    z[3] = NAN
    z[4, vocab // 3] = 1.0
    t = api.top_logits(z, 5)
    api.check_device()
    assert torch.isnan(t["lse"][1:4]).all()
    assert torch.isnan(t["values"][1:4, 0]).all()
    assert t["indices"][1:4, 0].tolist() == [vocab - 2, 0, 0]
    assert float(t["lse"][0]) == -INF and abs(float(t["lse"][4]) - 1.0) < 2.0 ** -20


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("rows,vocab", [(5, 1001), (200, 9003), (5, 90001)])
def test_distillation(rows, vocab, tail, dtype):
    """One NaN that is listed or not, the others masked or not: softmax of the
    row is NaN everywhere."""
    g = torch.Generator(device="cuda")
    g.manual_seed(vocab)
    indices = torch.arange(0, 40, 2, dtype=torch.int32, device="cuda").expand(rows, 20).contiguous()
    values = torch.randn(rows, 20, generator=g, device="cuda")
    lse = torch.logsumexp(values, 1) + 0.5 if tail else None
    z = (torch.randn(rows, vocab, generator=g, device="cuda")).to(dtype)

    def run():
        made = api.distill_top(z, indices, values, teacher_lse=lse, stats=True)
        back = api.distill_top_backward(z, indices, values, made["stats"], None, teacher_lse=lse)
        api.check_device()
        return made["loss"], made["grad"], back

    clean = run()
    z[0] = -INF
    z[0, :40:2] = 0.0
    z[0, vocab - 3] = NAN           # the only one of the rest that is not -inf
    z[1, 4] = NAN                   # a listed one
    z[2] = -INF
    z[2, 6] = NAN                   # a listed one, and nothing else
    z[3, vocab // 2] = NAN
    for got, was in zip(run(), clean):
        assert torch.isnan(got[:4]).all()
        assert torch.equal(got[4:], was[4:])
