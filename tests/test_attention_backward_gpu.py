"""The gradients of attention against fp64 (the bounds: attention_reference.py)."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api
from tests import attention_reference as ref
from tests.test_attention_gpu import CASES, each, make

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
MORE = [
    ([63], None, 1, 1, 64, True),
    ([64], None, 3, 1, 128, True),           # 21 tokens a step, one column left over
    ([65, 129], None, 7, 1, 64, False),
    ([40], [30], 96, 1, 64, True),           # 96 heads: two runs of 48
    ([20], [25], 67, 1, 64, True),           # a prime number of heads: one at a time
    ([100], [1000], 4, 1, 128, True),
    ([1000], [100], 4, 1, 128, True),        # 900 tokens see nothing
    ([1000], [100], 4, 1, 128, False),
    ([0, 50, 0], [30, 0, 0], 2, 1, 64, True),
]


def gradients(case, q, k, v, starts, key_starts, dy, **kw):
    common = dict(starts=starts, key_starts=key_starts, causal=case[5], **kw)
    o = api.attention(q, k, v, case[4], lse=True, **common)
    return o, api.attention_backward(dy, q, k, v, o["y"], o["lse"], case[4], **common)


def some_dy(q, seed=5):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(q.shape, generator=g, device="cuda").to(BF16)


def check(case, got, dy, q, k, v, nq, nk, first=0, scale=None):
    heads, kv_heads, d, causal = case[2:]
    scale = d ** -0.5 if scale is None else scale
    for rq, rk in each(nq, nk, first):
        want = ref.backward(dy[rq], q[rq], k[rk], v[rk], d, kv_heads, causal, scale)
        for name, rows, x, e in (("dq", rq, want[0], want[3]), ("dk", rk, want[1], want[4]), ("dv", rk, want[2], want[5])):
            off = (got[name][rows].double() - x).abs()
            bad = ~(off <= e + ref.HALF * (x.abs() + e))
            assert not bad.any(), (case, name, rows, off[bad].max().item(), int(bad.sum()))


@pytest.mark.parametrize("case", CASES + MORE, ids=str)
def test_backward(case):
    q, k, v, starts, key_starts, nq, nk = make(case)
    dy = some_dy(q)
    o, got = gradients(case, q, k, v, starts, key_starts, dy)
    api.check_device()
    check(case, got, dy, q, k, v, nq, nk)
    _, again = gradients(case, q, k, v, starts, key_starts, dy)
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("case", [([300], None, 4, 2, 128, True), ([200, 70], None, 2, 2, 64, False)], ids=str)
def test_whole_norm(case):
    """Each gradient's error relative to its norm: independent roundings of half a step at
    most (2^-8, of root mean square below 2^-8 / sqrt(3)) of P and ds, of y in D and of the
    result itself do not add up to more than 2^-8 sqrt(3) together."""
    q, k, v, starts, key_starts, nq, nk = make(case, seed=2)
    dy = some_dy(q)
    _, got = gradients(case, q, k, v, starts, key_starts, dy)
    for rq, rk in each(nq, nk):
        want = ref.backward(dy[rq], q[rq], k[rk], v[rk], case[4], case[3], case[5], case[4] ** -0.5)
        for name, rows, x in (("dq", rq, want[0]), ("dk", rk, want[1]), ("dv", rk, want[2])):
            assert (got[name][rows].double() - x).norm() < ref.HALF * 3 ** 0.5 * x.norm(), name


def test_against_differences():
    """Differences of the formula in fp64, at a handful of inputs."""
    case = ([9], [12], 2, 1, 16, True)
    q, k, v, starts, key_starts, nq, nk = make(case)
    dy = some_dy(q)
    _, got = gradients(case, q, k, v, starts, key_starts, dy)

    def loss(q, k, v):
        return (ref.forward(q, k, v, 16, 1, True, 0.25)[0] * dy.double()).sum()

    at = [t.double() for t in (q, k, v)]
    h = 1e-4
    for which, name in enumerate(("dq", "dk", "dv")):
        size = got[name].double().abs().max()
        for place in ((0, 0), (3, 7), (8, 15), (8, 31))[:4 if which == 0 else 3]:
            e = torch.zeros_like(at[which])
            e[place] = h
            plus, minus = ([t + s * e if i == which else t for i, t in enumerate(at)] for s in (1, -1))
            slope = (loss(*plus) - loss(*minus)) / (2 * h)
            # a handful of terms, each rounded by 2^-8 at most
            assert abs(float(slope - got[name][place])) < 4 * ref.HALF * float(size)


@pytest.mark.parametrize("case", [CASES[9], CASES[12]], ids=str)
def test_rows_of_no_sequence(case):
    q, k, v, starts, key_starts, nq, nk = make(case, first=3, behind=150)
    dy = some_dy(q)
    for t, n in ((q, sum(nq)), (dy, sum(nq)), (k, sum(nk)), (v, sum(nk))):
        t[:3] = math.nan
        t[3 + n:] = math.nan
    _, got = gradients(case, q, k, v, starts, key_starts, dy)
    check(case, got, dy, q, k, v, nq, nk, first=3)
    for name, n in (("dq", sum(nq)), ("dk", sum(nk)), ("dv", sum(nk))):
        assert (got[name][:3] == 0).all() and (got[name][3 + n:] == 0).all()


def test_large_scores():
    case = ([600], None, 2, 1, 64, True)
    q, k, v, starts, key_starts, nq, nk = make(case, seed=3)
    k = (k.float() * torch.linspace(0.1, 30.0, 600, device="cuda")[:, None]).to(BF16)
    dy = some_dy(q)
    _, got = gradients(case, q, k, v, starts, key_starts, dy)
    check(case, got, dy, q, k, v, nq, nk)


def test_columns_of_one_buffer():
    """q, k, v and their gradients as columns of one buffer each; parts asked for."""
    heads, kv_heads, d, n = 6, 2, 64, 333
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    widths = [heads * d, kv_heads * d, kv_heads * d]
    packed = torch.randn(n, sum(widths), generator=g, device="cuda").to(BF16)
    q, k, v = packed.split(widths, 1)
    dy = some_dy(q)
    o = api.attention(q, k, v, d, lse=True, scale=0.2)
    dz = torch.full_like(packed, math.nan)
    got = api.attention_backward(dy, q, k, v, o["y"], o["lse"], d, scale=0.2, out=dz.split(widths, 1))
    check(([n], None, heads, kv_heads, d, True), got, dy, q, k, v, [n], [n], scale=0.2)
    assert torch.equal(torch.cat([got["dq"], got["dk"], got["dv"]], 1), dz)
    only = api.attention_backward(dy, q, k, v, o["y"], o["lse"], d, scale=0.2, dkv=False)
    assert set(only) == {"dq"} and torch.equal(only["dq"], got["dq"])
    only = api.attention_backward(dy, q, k, v, o["y"], o["lse"], d, scale=0.2, dq=False)
    assert set(only) == {"dk", "dv"} and torch.equal(only["dk"], got["dk"]) and torch.equal(only["dv"], got["dv"])


def test_not_finite():
    """A NaN in one sequence's dy stays in its rows of dq, its keys and its sequence."""
    case = ([200, 200], None, 2, 1, 64, True)
    q, k, v, starts, key_starts, nq, nk = make(case)
    dy = some_dy(q)
    _, want = gradients(case, q, k, v, starts, key_starts, dy)
    dy[250, 70] = math.nan
    _, got = gradients(case, q, k, v, starts, key_starts, dy)
    for n in got:
        assert torch.equal(got[n][:200], want[n][:200])
    same = torch.ones_like(got["dq"], dtype=torch.bool)
    same[250, 64:] = False
    assert torch.equal(got["dq"][same], want["dq"][same]) and got["dq"][250, 64:].isnan().all()
    assert got["dk"][200:251].isnan().all()


def test_empty():
    for nq, nk in ((0, 50), (50, 0)):
        q, k, v, *_ = make(([nq], [nk], 2, 1, 64, True))
        o = api.attention(q, k, v, 64, lse=True)
        got = api.attention_backward(o["y"], q, k, v, o["y"], o["lse"], 64)
        assert all((got[n] == 0).all() for n in got)
        assert got["dq"].shape == (nq, 128) and got["dk"].shape == (nk, 64)


def test_streams_and_graphs():
    case = ([100, 30, 1, 300], [200, 70, 129, 300], 8, 2, 128, True)
    q, k, v, starts, key_starts, nq, nk = make(case)
    dy = some_dy(q)
    _, want = gradients(case, q, k, v, starts, key_starts, dy)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    _, got = gradients(case, q, k, v, starts, key_starts, dy, stream=other)
    other.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in got)
    graphs = []
    for _ in range(2):  # each with a workspace of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, gradients(case, q, k, v, starts, key_starts, dy)[1]))
    nq2, nk2 = [20, 0, 200, 101], [100, 90, 200, 229]
    starts.copy_(ref.starts_of(nq2))
    key_starts.copy_(ref.starts_of(nk2))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for (graph, _), s in zip(graphs, streams):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    for _, got in graphs:
        check(case, got, dy, q, k, v, nq2, nk2)
