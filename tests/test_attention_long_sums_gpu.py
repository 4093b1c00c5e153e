"""Attention's sums over very many keys, or rows, of one sign: fp32 however they are packed (GPU).

The tensor core cuts off what a product has below a step (2^-23) of the sum that it is added to, of
each 16 keys.  1,024 key tiles of 128 (8,192 products) lose 2^-10 of a sum at most; tiles beyond go
to another sum, which is joined to the first with roundings of 2^-24."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api
from tests import attention_reference as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
LOST = 2.0 ** -10 + 2.0 ** -13  # of a sum: cut off, and what sums of sums (up to 2^10 of them) and their quotient round
VALUE = 255 / 128               # the eight bits of a bf16


def packed(tokens, keys, others):
    """A sequence of many keys among others of one token and five keys each."""
    return (ref.starts_of([1] * (others // 2) + [tokens] + [1] * (others - others // 2)),
            ref.starts_of([5] * (others // 2) + [keys] + [5] * (others - others // 2)))


# others: so many that CTAs take items, few, none; tokens of one tile (its twin takes every other key
# tile) and of two
@pytest.mark.parametrize("tokens,keys,others,d", [
    (3, 1 << 21, 200, 8), (300, 1 << 21, 200, 8), (300, 1 << 20, 400, 128), (3, 1 << 21, 20, 8),
    (300, 1 << 21, 20, 8), (3, 1 << 22, 0, 8), (40000, 1 << 20, 0, 8), (2, (1 << 21) - 77, 160, 72)])
def test_values_alike(tokens, keys, others, d):
    """q of zeros: y is the mean of the values."""
    starts, key_starts = packed(tokens, keys, others)
    v = torch.full((keys + 5 * others, d), VALUE, dtype=BF16, device="cuda")
    q = torch.zeros(tokens + others, d, dtype=BF16, device="cuda")
    o = api.attention(q, v, v, d, starts=starts, key_starts=key_starts, causal=False, lse=True)
    api.check_device()
    off = (o["y"].double() - VALUE).abs()
    # rounded by half a step at most, 2^-8 of values below 2
    assert (off <= 2.0 ** -8 + LOST * VALUE).all(), off.max().item()
    rows = slice(others // 2, others // 2 + tokens)
    assert ((o["lse"][rows].double() - math.log(keys)).abs() <= 2.0 ** -12 + 24 * 2.0 ** -24).all()
    again = api.attention(q, v, v, d, starts=starts, key_starts=key_starts, causal=False, lse=True)
    assert torch.equal(again["y"], o["y"]) and torch.equal(again["lse"], o["lse"])


@pytest.mark.parametrize("tokens,keys,others,d,heads", [
    (3, 300_001, 160, 64, 1), (130, 300_001, 80, 64, 2), (3, 300_001, 160, 128, 1), (130, 200_001, 80, 128, 2),
    (3, (1 << 21) + 77, 0, 64, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_maxima_that_grow(tokens, keys, others, d, heads, causal):
    """Scores that grow along the keys: what was summed apart follows the maximum too."""
    starts, key_starts = packed(tokens, keys, others)
    g = torch.Generator(device="cuda")
    g.manual_seed(keys)
    total = keys + 5 * others
    q = torch.randn(tokens + others, heads * d, generator=g, device="cuda").abs().to(BF16)
    k = torch.randn(total, d, generator=g, device="cuda") * 0.2
    k += torch.linspace(-0.3, 0.3, total, device="cuda")[:, None]
    k = k.to(BF16)
    v = torch.randn(total, d, generator=g, device="cuda").to(BF16)
    o = api.attention(q, k, v, d, starts=starts, key_starts=key_starts, causal=causal, lse=True)
    api.check_device()
    first = others // 2
    rq, rk = slice(first, first + tokens), slice(5 * first, 5 * first + keys)
    for some in (slice(0, 3), slice(tokens - 2, tokens)):
        # (the mask is aligned at the end: of the first tokens, the last keys aside)
        last = keys - (tokens - some.stop) if causal else keys
        rows = slice(rq.start + some.start, rq.start + some.stop)
        y, lse, e_y, e_lse = ref.forward(q[rows], k[rk][:last], v[rk][:last], d, 1, causal, d ** -0.5)
        assert ((o["y"][rows].double() - y).abs() <= e_y + ref.HALF * (y.abs() + e_y)).all()
        assert ((o["lse"][rows].double() - lse).abs() <= e_lse).all()
