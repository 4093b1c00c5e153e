"""Tokens that see no key have y 0, lse -inf and dq 0 whatever the keys and values of their sequence
hold, and whichever way its rows are dealt out (GPU)."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api
from tests import attention_reference as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

# query lengths, key lengths, heads, kv heads, head_dim: causal, so the first n - m tokens of a
# sequence see nothing
CASES = [
    ([100], [60], 2, 1, 64),                     # beside tokens that see keys, in one tile
    ([20], [3], 4, 1, 128),
    ([300, 7], [170, 5], 4, 2, 128),
    ([60], [59], 32, 8, 128),
    ([1000], [700], 2, 2, 64),                   # some tiles without any key
    ([400] * 40, [399 - i for i in range(40)], 8, 8, 64),
    ([50] * 200, [49] * 200, 8, 8, 80),
]


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf], ids=str)
@pytest.mark.parametrize("what", ["k", "v", "both"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{c[0][0]}-{c[1][0]}-{c[2:]}")
def test_nothing_seen(case, what, value):
    nq, nk, heads, kv_heads, d = case
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    draw = lambda r, c: torch.randn(r, c, generator=g, device="cuda").to(BF16)  # noqa: E731
    q, dy = draw(sum(nq), heads * d), draw(sum(nq), heads * d)
    k, v = draw(sum(nk), kv_heads * d), draw(sum(nk), kv_heads * d)
    if what in ("k", "both"):
        k[:] = value
    if what in ("v", "both"):
        v[:] = value
    kw = dict(starts=ref.starts_of(nq), key_starts=ref.starts_of(nk))
    o = api.attention(q, k, v, d, lse=True, **kw)
    dq = api.attention_backward(dy, q, k, v, o["y"], o["lse"], d, dkv=False, **kw)["dq"]
    api.check_device()
    at = 0
    for n, m in zip(nq, nk):
        none = slice(at, at + n - m)
        assert (o["y"][none] == 0).all() and (o["lse"][none] == -math.inf).all() and (dq[none] == 0).all()
        at += n
    if what == "v":  # scores do not know of it
        y = api.attention(q, k, torch.ones_like(v), d, lse=True, **kw)
        assert torch.equal(y["lse"], o["lse"])
