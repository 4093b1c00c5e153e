"""Attention against fp64 (the bounds: attention_reference.py)."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api
from tests import attention_reference as ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# query lengths, key lengths (None: the same), heads, kv heads, head_dim, causal
CASES = [
    ([1], None, 1, 1, 64, True),
    ([1], None, 1, 1, 128, False),
    ([128], None, 1, 1, 128, False),
    ([128], None, 1, 1, 64, True),
    ([5], [3], 2, 1, 128, True),          # the first tokens see nothing
    ([129], None, 2, 2, 64, True),
    ([255], [257], 3, 1, 128, True),
    ([300], [7], 4, 2, 64, True),
    ([64], [1000], 4, 1, 128, False),
    ([77, 1, 0, 200, 128], None, 4, 2, 128, True),
    ([77, 1, 0, 200, 128], [80, 130, 5, 0, 129], 4, 2, 128, True),
    ([3, 500, 17], [600, 500, 18], 8, 1, 64, False),
    ([1, 1, 1, 1, 1], [1000, 1, 129, 0, 2050], 32, 8, 128, True),
    ([1], [5000], 8, 1, 128, True),
    ([1], [5000], 7, 7, 80, True),
    ([2, 3], [3000, 900], 20, 4, 96, True),
    ([700], None, 6, 2, 72, True),
    ([400], None, 5, 1, 8, True),
    ([40, 40], [300, 41], 128, 1, 64, True),  # 128 heads share their keys
    ([513, 511], None, 12, 12, 64, True),
    ([1500], None, 8, 2, 128, True),
    ([1] * 67, [33 * i % 200 for i in range(67)], 4, 2, 64, True),
]


def make(case, seed=0, first=0, behind=0, scale=1.0):
    nq, nk, heads, kv_heads, d, causal = case
    nk = nq if nk is None else nk
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rows, keys = first + sum(nq) + behind, first + sum(nk) + behind
    draw = lambda r, c: (torch.randn(r, c, generator=g, device="cuda") * scale).to(BF16)  # noqa: E731
    q, k, v = draw(rows, heads * d), draw(keys, kv_heads * d), draw(keys, kv_heads * d)
    return q, k, v, ref.starts_of(nq, first), ref.starts_of(nk, first), nq, nk


def each(nq, nk, first=0):
    a = b = first
    for n, m in zip(nq, nk):
        yield slice(a, a + n), slice(b, b + m)
        a, b = a + n, b + m


def check(case, o, q, k, v, nq, nk, first=0, scale=None):
    heads, kv_heads, d, causal = case[2:]
    scale = d ** -0.5 if scale is None else scale
    for rq, rk in each(nq, nk, first):
        if rq.start == rq.stop:
            continue
        y, lse, e_y, e_lse = ref.forward(q[rq], k[rk], v[rk], d, kv_heads, causal, scale)
        off = (o["y"][rq].double() - y).abs()
        assert (off <= e_y + ref.HALF * (y.abs() + e_y)).all(), (case, rq, off.max())
        none = lse == -math.inf
        assert torch.equal(o["lse"][rq] == -math.inf, none), (case, rq)
        off = torch.where(none, 0.0, (o["lse"][rq].double() - lse).abs())
        assert (off <= e_lse).all(), (case, rq, off.max())


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case):
    q, k, v, starts, key_starts, nq, nk = make(case)
    kw = dict(starts=starts, key_starts=key_starts, causal=case[5])
    o = api.attention(q, k, v, case[4], lse=True, **kw)
    api.check_device()
    check(case, o, q, k, v, nq, nk)
    again = api.attention(q, k, v, case[4], lse=True, **kw)
    assert torch.equal(again["y"], o["y"]) and torch.equal(again["lse"], o["lse"])


@pytest.mark.parametrize("case", [CASES[9], CASES[12]], ids=str)
def test_rows_of_no_sequence(case):
    """Rows before the first sequence and behind the last hold NaN: none is read, theirs are empty."""
    q, k, v, starts, key_starts, nq, nk = make(case, first=3, behind=150)
    for t, n in ((q, sum(nq)), (k, sum(nk)), (v, sum(nk))):
        t[:3] = math.nan
        t[3 + n:] = math.nan
    o = api.attention(q, k, v, case[4], starts=starts, key_starts=key_starts, lse=True, causal=case[5])
    check(case, o, q, k, v, nq, nk, first=3)
    for rows in (slice(0, 3), slice(3 + sum(nq), None)):
        assert (o["y"][rows] == 0).all() and (o["lse"][rows] == -math.inf).all()


def test_columns_of_one_buffer_and_default_starts():
    case = ([333], None, 6, 2, 64, True)
    heads, kv_heads, d = case[2:5]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    packed = torch.randn(333, (heads + 2 * kv_heads) * d + 8, generator=g, device="cuda").to(BF16)
    q, k, v, _ = packed.split([heads * d, kv_heads * d, kv_heads * d, 8], 1)
    o = api.attention(q, k, v, d, lse=True)
    check(case, o, q, k, v, [333], [333])
    o = api.attention(q, k, v, d, lse=True, causal=False, scale=0.3)
    check(case[:5] + (False,), o, q, k, v, [333], [333], scale=0.3)
    assert "lse" not in api.attention(q, k, v, d)


def test_large_scores():
    """Maxima that grow by far more than the slack from key tile to key tile, and differ by row."""
    case = ([600], None, 2, 1, 64, True)
    q, k, v, *_ = make(case, seed=3)
    k = (k.float() * torch.linspace(0.1, 30.0, 600, device="cuda")[:, None]).to(BF16)
    o = api.attention(q, k, v, 64, lse=True)
    check(case, o, q, k, v, [600], [600])
    q[::2] *= -1
    o = api.attention(q, k, v, 64, lse=True)
    check(case, o, q, k, v, [600], [600])


def test_not_finite():
    """A NaN or infinity in q or k reaches the rows of its own sequence that see it, and no others."""
    case = ([200, 200], None, 2, 1, 64, True)
    q, k, v, starts, _, nq, nk = make(case)
    want = api.attention(q, k, v, 64, starts=starts)["y"]
    k2 = k.clone()
    k2[150, 3] = math.nan
    got = api.attention(q, k2, v, 64, starts=starts)["y"]
    assert torch.equal(got[:150], want[:150]) and torch.equal(got[200:], want[200:])
    assert got[150:200].isnan().all()
    q2 = q.clone()
    q2[10, 64:] = math.inf
    got = api.attention(q2, k, v, 64, starts=starts)["y"]
    same = torch.ones_like(got, dtype=torch.bool)
    same[10, 64:] = False
    assert torch.equal(got[same], want[same])
    v2 = v.clone()
    v2[200:] = math.nan  # the second sequence's own
    got = api.attention(q, k, v2, 64, starts=starts)["y"]
    assert torch.equal(got[:200], want[:200]) and got[200:].isnan().all()


def test_offsets_out_of_range():
    """Offsets that leave the tensors name no row outside: what they do name is finite."""
    q, k, v, *_ = make(([100], None, 2, 1, 64, True))
    bad = torch.tensor([-50, 40, 1 << 30], dtype=torch.int32, device="cuda")
    y = api.attention(q, k, v, 64, starts=bad)["y"]
    api.check_device()
    want = api.attention(q, k, v, 64, starts=torch.tensor([0, 40, 100], dtype=torch.int32, device="cuda"))["y"]
    assert torch.equal(y, want)
    down = torch.tensor([0, 90, 30, 100], dtype=torch.int32, device="cuda")
    api.attention(q, k, v, 64, starts=down)
    api.check_device()


def test_empty():
    q, k, v, *_ = make(([0], [50], 2, 1, 64, True))
    assert api.attention(q, k, v, 64)["y"].shape == (0, 128)
    q, k, v, *_ = make(([50], [0], 2, 1, 64, True))
    o = api.attention(q, k, v, 64, lse=True)
    assert (o["y"] == 0).all() and (o["lse"] == -math.inf).all()
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    q, k, v, *_ = make(([50], [50], 2, 1, 64, True))
    o = api.attention(q, k, v, 64, starts=none, lse=True)
    assert (o["y"] == 0).all() and (o["lse"] == -math.inf).all()


@pytest.mark.parametrize("many", [300, 3001])
def test_many_sequences(many):
    """One to three tokens a sequence, up to 40 keys."""
    g = torch.Generator()
    g.manual_seed(many)
    nq = torch.randint(0, 4, (many,), generator=g).tolist()
    nk = [n + extra for n, extra in zip(nq, torch.randint(0, 38, (many,), generator=g).tolist())]
    case = (nq, nk, 4, 2, 64, True)
    q, k, v, starts, key_starts, *_ = make(case)
    o = api.attention(q, k, v, 64, starts=starts, key_starts=key_starts, lse=True)
    back = api.attention_backward(q, q, k, v, o["y"], o["lse"], 64, starts=starts, key_starts=key_starts)
    api.check_device()
    some = set(torch.randint(0, many, (40,), generator=g).tolist()) | {0, many - 1}
    for i, (rq, rk) in enumerate(each(nq, nk)):
        if i not in some or rq.start == rq.stop:
            continue
        y, lse, e_y, e_lse = ref.forward(q[rq], k[rk], v[rk], 64, 2, True, 0.125)
        assert ((o["y"][rq].double() - y).abs() <= e_y + ref.HALF * (y.abs() + e_y)).all()
        want = ref.backward(q[rq], q[rq], k[rk], v[rk], 64, 2, True, 0.125)
        for name, rows, x, e in (("dq", rq, want[0], want[3]), ("dk", rk, want[1], want[4]), ("dv", rk, want[2], want[5])):
            assert ((back[name][rows].double() - x).abs() <= e + ref.HALF * (x.abs() + e)).all(), name


def test_far_rows():
    """Rows beyond 2^31 elements of a buffer: a long cache, one head of it wide.  (How many CTAs
    share a row's keys goes by the cache's rows, so sums have another order than over the
    sequence's own rows alone, and both are held to fp64.)"""
    rows, width = 560000, 4096
    cache = torch.empty(rows, width, dtype=BF16, device="cuda")
    case = ([70], [200], 2, 1, 64, True)
    q, k, v, *_ = make(case)
    kk, vv = cache[:, 128:192], cache[:, 4032:]
    kk[-200:], vv[-200:] = k, v
    starts, key_starts = ref.starts_of([70]), torch.tensor([rows - 200, rows], dtype=torch.int32, device="cuda")
    o = api.attention(q, kk, vv, 64, starts=starts, key_starts=key_starts, lse=True)
    check(case, o, q, k, v, [70], [200])
    back = api.attention_backward(q, q, kk, vv, o["y"], o["lse"], 64, starts=starts, key_starts=key_starts)
    want = ref.backward(q, q, k, v, 64, 1, True, 0.125)
    for name, x, e in zip(("dq", "dk", "dv"), want[:3], want[3:]):
        got = back[name][-x.shape[0]:].double()
        assert ((got - x).abs() <= e + ref.HALF * (x.abs() + e)).all(), name
        assert (back[name][:-x.shape[0]] == 0).all()


def test_a_long_sequence():
    """20,001 tokens of one head against fp64 at some of its rows, and in one piece with itself."""
    case = ([20001], None, 1, 1, 64, True)
    q, k, v, *_ = make(case)
    o = api.attention(q, k, v, 64, lse=True)
    for rows in (slice(0, 130), slice(9990, 10010), slice(19900, 20001)):
        y, lse, e_y, e_lse = ref.forward(q[rows], k[:rows.stop], v[:rows.stop], 64, 1, True, 0.125)
        assert ((o["y"][rows].double() - y).abs() <= e_y + ref.HALF * (y.abs() + e_y)).all()
        assert ((o["lse"][rows].double() - lse).abs() <= e_lse).all()


def test_streams_and_graphs():
    case = ([1, 1, 1, 300], [2000, 700, 129, 300], 8, 2, 128, True)
    q, k, v, starts, key_starts, nq, nk = make(case)
    kw = dict(starts=starts, key_starts=key_starts, lse=True)
    want = api.attention(q, k, v, 128, **kw)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    got = api.attention(q, k, v, 128, stream=other, **kw)
    other.synchronize()
    assert torch.equal(got["y"], want["y"])
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, api.attention(q, k, v, 128, **kw)))
    # other lengths in the same buffers
    nq2, nk2 = [2, 0, 200, 101], [100, 900, 1000, 1129]
    starts.copy_(ref.starts_of(nq2))
    key_starts.copy_(ref.starts_of(nk2))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for (graph, _), s in zip(graphs, streams):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    for _, o in graphs:
        check(case, o, q, k, v, nq2, nk2)


def test_a_wait_that_runs_out_is_reported():
    """Forward and both backward kernels: their copies are never asked for."""
    from paper_2608_13966_gb300 import quasar as Q

    for case in (([300], None, 4, 2, 128, True), ([1], [3000], 8, 2, 64, True)):  # (the second: a cluster a row)
        q, k, v, starts, key_starts, nq, nk = make(case)
        kw = dict(starts=starts, key_starts=key_starts)
        want = api.attention(q, k, v, case[4], lse=True, **kw)
        back = lambda: api.attention_backward(q, q, k, v, want["y"], want["lse"], case[4], **kw)  # noqa: E731
        grads = back()
        api.check_device()
        for call in (lambda: api.attention(q, k, v, case[4], **kw), back):
            Q.quasar_debug_force_timeout(1_000_000)
            try:
                call()
                assert Q.quasar_get_device_status() == Q.QuasarStatus.ERR_TIMEOUT
            finally:
                Q.quasar_debug_force_timeout(0)
        assert torch.equal(api.attention(q, k, v, case[4], **kw)["y"], want["y"])
        again = back()
        assert all(torch.equal(again[n], grads[n]) for n in grads)
        api.check_device()
