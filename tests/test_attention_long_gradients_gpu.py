"""Attention's gradients over very many rows, or keys, of one sign: fp32 sums (GPU).

As for the outputs: the tensor core cuts off less than 2^-23 of a sum with each product of 16 columns,
2^-10 over the 1,024 steps of 128 columns that are added to one."""
import pytest
import torch

from paper_2608_13966_gb300 import api
from tests import attention_reference as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
LOST = 2.0 ** -10 + 2.0 ** -13
VALUE = 255 / 128


def close(got, want):
    """Cut off, then rounded to bf16."""
    off = (got.double() / want - 1).abs()
    assert (off <= 2.0 ** -8 + LOST).all(), off.max().item()


@pytest.mark.parametrize("tokens,heads,d", [(1 << 18, 8, 8), (1 << 21, 1, 8), (1 << 17, 16, 128), (30001, 67, 8)])
def test_of_keys(tokens, heads, d):
    """Two keys of zeros (probabilities of 1/2), values of 1 and -1 (D = 0): dk = +-n/2 (255/128)^2,
    dv = n/2 255/128, for n rows of dy and q of 255/128, and nothing in the other columns."""
    q = torch.zeros(tokens, heads, d, dtype=BF16, device="cuda")
    q[:, :, 0] = VALUE
    q = q.view(tokens, heads * d)
    k, v = (torch.zeros(2, d, dtype=BF16, device="cuda") for _ in range(2))
    v[0, 0], v[1, 0] = 1, -1
    kw = dict(causal=False, scale=1.0)
    o = api.attention(q, k, v, d, lse=True, **kw)
    assert (o["y"] == 0).all()
    g = api.attention_backward(q, q, k, v, o["y"], o["lse"], d, dq=False, **kw)
    api.check_device()
    n = tokens * heads
    close(g["dk"][0, 0], n / 2 * VALUE ** 2)
    close(g["dk"][1, 0], -n / 2 * VALUE ** 2)
    close(g["dv"][:, 0], n / 2 * VALUE)
    assert (g["dk"][:, 1:] == 0).all() and (g["dv"][:, 1:] == 0).all()


@pytest.mark.parametrize("tokens,keys,others,d", [(3, 1 << 21, 0, 8), (300, 1 << 21, 200, 8), (130, 1 << 21, 0, 128)])
def test_of_queries(tokens, keys, others, d):
    """Probabilities of 1/n, values of 1 and -1 in turn, keys of +-255/128 with them where q is 0:
    dq = (255/128)^2."""
    total = keys + 2 * others
    sign = 1 - 2 * (torch.arange(total, device="cuda") % 2).float()
    q, k, v = (torch.zeros(n, d, dtype=BF16, device="cuda") for n in (tokens + others, total, total))
    q[:, 0] = VALUE
    k[:, 1] = VALUE * sign
    v[:, 0] = sign
    kw = dict(causal=False, scale=1.0, starts=ref.starts_of([tokens] + [1] * others),
              key_starts=ref.starts_of([keys] + [2] * others))
    o = api.attention(q, k, v, d, lse=True, **kw)
    assert (o["y"] == 0).all()
    g = api.attention_backward(q, q, k, v, o["y"], o["lse"], d, dkv=False, **kw)
    api.check_device()
    close(g["dq"][:, 1], VALUE ** 2)
    assert (g["dq"][:, 0] == 0).all() and (g["dq"][:, 2:] == 0).all()


@pytest.mark.parametrize("case", [
    ([70001], [5], 2, 1, 64, False), ([270001], [4], 1, 1, 8, False), ([5], [140001], 2, 1, 64, False),
    ([131072, 3, 40000], [3, 200, 2], 2, 2, 128, False), ([3, 200], [131073, 200], 4, 2, 96, True),
    ([131072], [3], 1, 1, 64, False), ([131073], [3], 1, 1, 64, False)], ids=str)
def test_steps_apart(case):
    """Sums of a step more than one holds, of exactly as many, of several; random inputs against fp64
    (and twice the same)."""
    nq, nk, heads, kv_heads, d, causal = case
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(nq))
    draw = lambda r, c: torch.randn(r, c, generator=g, device="cuda").to(BF16)  # noqa: E731
    q, dy = draw(sum(nq), heads * d), draw(sum(nq), heads * d)
    k, v = draw(sum(nk), kv_heads * d), draw(sum(nk), kv_heads * d)
    kw = dict(starts=ref.starts_of(nq), key_starts=ref.starts_of(nk), causal=causal)
    o = api.attention(q, k, v, d, lse=True, **kw)
    got = api.attention_backward(dy, q, k, v, o["y"], o["lse"], d, **kw)
    again = api.attention_backward(dy, q, k, v, o["y"], o["lse"], d, **kw)
    api.check_device()
    a = b = 0
    for n, m in zip(nq, nk):
        rq, rk = slice(a, a + n), slice(b, b + m)
        want = ref.backward(dy[rq], q[rq], k[rk], v[rk], d, kv_heads, causal, d ** -0.5)
        for name, rows, x, e in (("dq", rq, want[0], want[3]), ("dk", rk, want[1], want[4]), ("dv", rk, want[2], want[5])):
            off = (got[name][rows].double() - x).abs()
            assert (off <= e + ref.HALF * (x.abs() + e)).all(), (name, off.max().item())
        a, b = a + n, b + m
    assert all(torch.equal(got[n], again[n]) for n in got)
