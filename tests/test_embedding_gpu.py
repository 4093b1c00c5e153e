"""The embedding and its gradient against fp64.

A looked-up value is one product and one sum in fp32, rounded once; a row of
the gradient is an fp32 sum of its n tokens' rows, off by at most n 2^-24 of the
sum of their sizes, rounded once."""
import pytest
import torch

from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: U}


def rand(*shape, dtype=BF16, seed=0, ld=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + sum(shape))
    x = torch.randn(*shape, generator=g, device="cuda").to(dtype)
    if ld is None:
        return x
    wide = torch.zeros(shape[0], ld, dtype=dtype, device="cuda")
    wide[:, :shape[1]] = x
    return wide[:, :shape[1]]


def some_ids(tokens, vocab, seed=0, dtype=torch.int32, padding=0.1, skew=3.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + tokens)
    ids = (torch.rand(tokens, generator=g, device="cuda") ** skew * vocab).long().clamp(max=vocab - 1)
    out = torch.rand(tokens, generator=g, device="cuda") < padding
    far = torch.tensor([-1, vocab, -2 ** 31, 2 ** 31 - 1], device="cuda")
    return torch.where(out, far[torch.arange(tokens, device="cuda") % 4], ids).to(dtype)


def gradient(dy, ids, vocab, scale):
    """The sums, the sums of sizes and the number of each row's tokens, in fp64."""
    live = (ids >= 0) & (ids < vocab)
    at = ids[live].long()
    total, size = (torch.zeros(vocab, dy.shape[1], dtype=torch.float64, device="cuda") for _ in range(2))
    total.index_add_(0, at, dy[live].double() * scale)
    size.index_add_(0, at, (dy[live].double() * scale).abs())
    return total, size, torch.bincount(at, minlength=vocab)[:, None]


@pytest.mark.parametrize("table_dtype,out", [(BF16, BF16), (F32, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("tokens,vocab,width", [(1, 1, 1), (1, 50001, 4096), (3, 17, 9), (23, 1000, 1003), (4, 5, 2048),
                                                (5, 100, 2056), (1001, 8003, 640), (4097, 300, 4099)])
def test_lookup(tokens, vocab, width, table_dtype, out):
    for id_dtype, ld in ((torch.int32, None), (torch.int64, width + 5)):
        table, ids = rand(vocab, width, dtype=table_dtype, ld=ld), some_ids(tokens, vocab, dtype=id_dtype)
        res = rand(tokens, width, dtype=out, seed=3, ld=ld)
        live = ((ids >= 0) & (ids < vocab))[:, None]
        rows = torch.where(live, table[ids.long().clamp(0, vocab - 1)].double(), 0.0)
        for scale, residual in ((1.0, None), (0.37, res)):
            y = api.embedding(ids, table, scale=scale, residual=residual, out_dtype=out)
            want = rows * torch.tensor(scale, dtype=F32).double().item() + (0 if residual is None else res.double())
            assert ((y.double() - want).abs() <= HALF[out] * want.abs() * 1.001 + U * rows.abs()).all()


@pytest.mark.parametrize("dy_dtype,out", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("tokens,vocab,width", [(1, 1, 1), (1, 5000, 2048), (31, 17, 9), (127, 3, 40), (128, 1, 64),
                                                (129, 513, 1003), (2049, 511, 256), (5000, 131072, 64),
                                                (20000, 700, 136), (3000, 263000, 8)])
def test_gradient(tokens, vocab, width, dy_dtype, out):
    for id_dtype, ld in ((torch.int32, None), (torch.int64, width + 3)):
        dy, ids = rand(tokens, width, dtype=dy_dtype, ld=ld), some_ids(tokens, vocab, dtype=id_dtype)
        for scale in (1.0, 0.37):
            exact_scale = torch.tensor(scale, dtype=F32).double().item()
            want, size, n = gradient(dy, ids, vocab, exact_scale)
            got = api.embedding_backward(dy, ids, vocab, scale=scale, dtable_dtype=out)
            e = (n + 2) * U * size
            assert ((got.double() - want).abs() <= e + HALF[out] * (want.abs() + e)).all()
            assert (got[n[:, 0] == 0] == 0).all()
            assert torch.equal(got, api.embedding_backward(dy, ids, vocab, scale=scale, dtable_dtype=out))
            before = rand(vocab, width, dtype=out, seed=5, ld=ld)
            into = rand(vocab, width, dtype=out, seed=5, ld=ld)
            assert api.embedding_backward(dy, ids, vocab, scale=scale, into=into) is into
            want = want + before.double()
            e = e + U * before.double().abs()
            assert ((into.double() - want).abs() <= e + HALF[out] * (want.abs() + e)).all()
            assert torch.equal(into[n[:, 0] == 0], before[n[:, 0] == 0])


@pytest.mark.parametrize("tokens", [40000, 300000])
def test_one_token_for_all(tokens):
    """Every row into one, and whole numbers: the sum is exact."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    dy = torch.randint(-3, 4, (tokens, 72), generator=g, device="cuda").to(BF16)
    ids = torch.full((tokens,), 77, dtype=torch.int32, device="cuda")
    got = api.embedding_backward(dy, ids, 200, dtable_dtype=F32)
    assert torch.equal(got[77].double(), dy.double().sum(0))
    got[77] = 0
    assert (got == 0).all()


def test_order_of_the_sums():
    """A row's tokens are added in their order: sums that fp32 cannot reorder."""
    tokens, width = 100, 16
    dy = torch.zeros(tokens, width, device="cuda")
    dy[3], dy[50], dy[97] = 1.0, 2.0 ** 25, -(2.0 ** 25)
    ids = torch.zeros(tokens, dtype=torch.int32, device="cuda")
    got = api.embedding_backward(dy, ids, 1, dtable_dtype=F32)
    assert (got == 0.0).all()  # (1 + 2^25) - 2^25 in fp32
    dy[3], dy[50], dy[97] = 2.0 ** 25, -(2.0 ** 25), 1.0
    assert (api.embedding_backward(dy, ids, 1, dtable_dtype=F32) == 1.0).all()


def test_far_rows():
    """Offsets that pass 32 bits: tables of more than 2^31 elements."""
    vocab, width = 600000, 4096
    table = torch.empty(vocab, width, dtype=BF16, device="cuda")
    table[-2:] = rand(2, width)
    ids = torch.tensor([vocab - 1, vocab - 2], device="cuda")
    assert torch.equal(api.embedding(ids, table), table[[vocab - 1, vocab - 2]])
    del table
    dy = rand(2, width)
    got = api.embedding_backward(dy, ids, vocab)
    assert torch.equal(got[-2:], dy.flip(0)) and (got[vocab // 2:-2] == 0).all()


def test_nan_stays_in_its_row():
    dy, ids = rand(400, 100), some_ids(400, 50, padding=0.0)
    dy[7, 3] = float("nan")
    got = api.embedding_backward(dy, ids, 50)
    bad = got.isnan()
    assert bad[ids[7].long(), 3] and bad.sum() == 1


def test_empty():
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert api.embedding(none, rand(10, 8)).shape == (0, 8)
    assert (api.embedding_backward(rand(0, 8), none, 10) == 0).all()
    into = rand(10, 8)
    before = into.clone()
    assert torch.equal(api.embedding_backward(rand(0, 8), none, 10, into=into), before)


def test_streams_and_graphs():
    dy, ids = rand(3000, 200), some_ids(3000, 500)
    want = api.embedding_backward(dy, ids, 500)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    got = api.embedding_backward(dy, ids, 500, stream=other)
    other.synchronize()
    assert torch.equal(got, want)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, api.embedding_backward(dy, ids, 500)))
    ids.copy_(some_ids(3000, 500, seed=4))
    want = api.embedding_backward(dy, ids, 500)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for (graph, _), s in zip(graphs, streams):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for _, o in graphs)
