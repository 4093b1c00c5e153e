"""Attention of more items than the device holds at a time: CTAs take them from those not launched."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api
from paper_2608_13966_gb300 import quasar as Q
from tests import attention_reference as ref
from tests.test_attention_gpu import check, each, make

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

# one tile (its twins take turns), two, and both in a batch; keys from none to many tiles
CASES = [
    ([1] * 50, [(397 * i) % 1500 for i in range(50)], 32, 8, 128, True),
    ([1] * 90, [(131 * i) % 700 + 1 for i in range(90)], 16, 2, 64, False),
    ([1, 33, 20, 64, 70, 0, 32, 31] * 4, [600, 33, 300, 129, 70, 40, 1000, 257] * 4, 32, 8, 128, True),
    ([5] * 40, [128 * (i % 5) + i for i in range(40)], 40, 5, 80, True),
    ([300, 2, 1, 180] * 5, [300, 900, 129, 180] * 5, 12, 12, 64, True),
    ([127] * 30, [129] * 30, 8, 8, 128, True),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_items(case):
    q, k, v, starts, key_starts, nq, nk = make(case)
    d = case[4]
    kw = dict(starts=starts, key_starts=key_starts, causal=case[5])
    o = api.attention(q, k, v, d, lse=True, **kw)
    back = api.attention_backward(q, q, k, v, o["y"], o["lse"], d, **kw)
    api.check_device()
    check(case, o, q, k, v, nq, nk)
    scale = d ** -0.5
    for rq, rk in list(each(nq, nk))[:9]:
        want = ref.backward(q[rq], q[rq], k[rk], v[rk], d, case[3], case[5], scale)
        for name, rows, x, e in (("dq", rq, want[0], want[3]), ("dk", rk, want[1], want[4]), ("dv", rk, want[2], want[5])):
            assert ((back[name][rows].double() - x).abs() <= e + ref.HALF * (x.abs() + e)).all(), (name, rows)
    # two at once, on two streams, and replayed: who takes what does not show
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    many = [api.attention(q, k, v, d, lse=True, stream=s, **kw) for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        many.append(api.attention(q, k, v, d, lse=True, **kw))
        again = api.attention_backward(q, q, k, v, o["y"], o["lse"], d, **kw)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    api.check_device()
    assert all(torch.equal(z["y"], o["y"]) and torch.equal(z["lse"], o["lse"]) for z in many)
    assert all(torch.equal(again[n], back[n]) for n in back)


def test_only_their_columns_are_written():
    """Outputs among other columns, and the lse's rows: nothing beside them changes."""
    case = CASES[2]
    q, k, v, starts, key_starts, nq, nk = make(case)
    heads, kv_heads, d = case[2:5]
    kw = dict(starts=starts, key_starts=key_starts)
    o = api.attention(q, k, v, d, lse=True, **kw)
    want = api.attention_backward(q, q, k, v, o["y"], o["lse"], d, **kw)
    around = lambda rows, cols: torch.full((rows + 2, cols + 48), 7.25, dtype=BF16, device="cuda")  # noqa: E731
    inner = lambda t: t[1:-1, 24:-24]  # noqa: E731
    y, dq = around(len(q), heads * d), around(len(q), heads * d)
    dk, dv = around(len(k), kv_heads * d), around(len(k), kv_heads * d)
    lse = torch.full((len(q) + 2, heads), 7.25, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    Q.quasar_attention(q.data_ptr(), q.stride(0), k.data_ptr(), k.stride(0), v.data_ptr(), v.stride(0), len(q), len(k),
                       heads, kv_heads, d, starts.data_ptr(), key_starts.data_ptr(), len(nq), 1, d ** -0.5,
                       inner(y).data_ptr(), y.stride(0), lse[1:].data_ptr(), stream)
    api.attention_backward(q, q, k, v, o["y"], o["lse"], d, out=(inner(dq), inner(dk), inner(dv)), **kw)
    api.check_device()
    for whole, part in ((y, o["y"]), (dq, want["dq"]), (dk, want["dk"]), (dv, want["dv"])):
        assert torch.equal(inner(whole), part)
        inner(whole)[:] = 7.25
        assert (whole == 7.25).all()
    assert torch.equal(lse[1:-1], o["lse"]) and (lse[0] == 7.25).all() and (lse[-1] == 7.25).all()


def test_an_item_longer_than_a_wait():
    """One of 600 sequences has 2.6e8 keys, which take a CTA over a second: that is no time-out.  With
    q of zeros and values of ones for 2^20 keys and zeros behind, every sum is exact: lse is
    log(2.6e8) but for some roundings of 20, and y their share, rounded to bf16 (twice: as a quotient,
    and as stored).  The others have a token and a key each."""
    far, tokens, others = 260_000_000, 256, 599
    k = torch.zeros(far + others, 8, dtype=BF16, device="cuda")
    k[:1 << 20] = 1
    k[far:] = 3
    q = torch.zeros(tokens + others, 8, dtype=BF16, device="cuda")
    starts, key_starts = ref.starts_of([tokens] + [1] * others), ref.starts_of([far] + [1] * others)
    o = api.attention(q, k, k, 8, starts=starts, key_starts=key_starts, causal=False, lse=True)
    api.check_device()
    assert ((o["lse"][:tokens].double() - math.log(far)).abs() <= 8 * 20 * 2.0 ** -24).all()
    want = (1 << 20) / far
    assert ((o["y"][:tokens].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want).all()
    assert (o["y"][tokens:] == 3).all() and (o["lse"][tokens:] == 0).all()


def test_far_more_keys_than_a_sum_holds():
    """2^21 keys alike, of values with eight bits: what the tensor core cuts off of each stays below
    the rounding of y."""
    v = torch.full((1 << 21, 8), 255 / 128, dtype=BF16, device="cuda")
    for tokens in (3, 152 * 256):
        y = api.attention(torch.zeros(tokens, 8, dtype=BF16, device="cuda"), v, v, 8, causal=False)["y"]
        assert ((y.double() - 255 / 128).abs() <= 2.0 ** -8 * 2).all()


def test_a_wait_that_runs_out_is_reported():
    case = CASES[0]
    q, k, v, starts, key_starts, *_ = make(case)
    kw = dict(starts=starts, key_starts=key_starts)
    want = api.attention(q, k, v, 128, lse=True, **kw)
    grads = api.attention_backward(q, q, k, v, want["y"], want["lse"], 128, **kw)
    api.check_device()
    for call in (lambda: api.attention(q, k, v, 128, **kw),
                 lambda: api.attention_backward(q, q, k, v, want["y"], want["lse"], 128, **kw)):
        Q.quasar_debug_force_timeout(1_000_000)
        try:
            call()
            assert Q.quasar_get_device_status() == Q.QuasarStatus.ERR_TIMEOUT
        finally:
            Q.quasar_debug_force_timeout(0)
    assert torch.equal(api.attention(q, k, v, 128, **kw)["y"], want["y"])
    again = api.attention_backward(q, q, k, v, want["y"], want["lse"], 128, **kw)
    assert all(torch.equal(again[n], grads[n]) for n in grads)
    api.check_device()
