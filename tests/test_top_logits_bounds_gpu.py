"""Top lists whose first bound is hard to find: more entries asked for than a
small CTA has threads, and rows whose vectors' maxima say nothing about how
many elements reach them (GPU).  Every comparison is of whole values, with
outputs that held a marker before the call, so that a place that is not
written shows."""
import pytest
import torch

from paper_2608_13966_gb300 import api
from paper_2608_13966_gb300 import quasar as Q

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
MARK = -12345


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def check(z, k):
    rows, vocab = z.shape
    values = torch.full((rows, k), float(MARK), device="cuda")
    indices = torch.full((rows, k), MARK, dtype=torch.int32, device="cuda")
    lse = torch.full((rows,), float(MARK), device="cuda")
    st = Q.quasar_top_logits(z, Q.BF16 if z.dtype == BF16 else Q.F32, z.stride(0), rows, vocab, k,
                             1.0, values, indices, lse)
    assert st == Q.QuasarStatus.OK
    api.check_device()
    v, i = torch.sort(z.float(), dim=1, descending=True, stable=True)
    assert (indices != MARK).all(), int((indices == MARK).sum())
    assert torch.equal(indices.long(), i[:, :k])
    assert torch.equal(values, v[:, :k])
    assert (lse != MARK).all()


def peaks(rows, vocab, dtype, every, peak, seed):
    """N(0, 1) with `peak` (a value, or a range to draw from) at each `every`-th place."""
    g = gen(seed)
    z = torch.randn(rows, vocab, generator=g, device="cuda")
    at = z[:, ::every]
    if isinstance(peak, tuple):
        low, high = peak
        at.copy_(low + (high - low) * torch.rand(at.shape, generator=g, device="cuda"))
    else:
        at.fill_(peak)
    return z.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [100, 128, 129, 200, 256])
@pytest.mark.parametrize("vocab", [512, 1000, 1024, 2048, 4092, 4096, 8184, 8192])
@pytest.mark.parametrize("peak", [5.0, (8.0, 12.0), (8.0, 8.1)])
def test_one_peak_a_vector(vocab, k, dtype, peak):
    per = 8 if dtype == BF16 else 4
    check(peaks(3, vocab, dtype, per, peak, vocab + k), k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [129, 200, 256])
@pytest.mark.parametrize("threads", [128, 512])
def test_one_peak_a_thread(threads, k, dtype):
    """As many peaks as a CTA has threads, each in a vector of another."""
    per = 8 if dtype == BF16 else 4
    vocab = min(8 * threads, 1024) * per
    z = torch.full((2, vocab), -1.0, dtype=dtype, device="cuda")
    z[:, :threads * per:per] = 2.0
    check(z, k)
    z[:, :threads * per:per] = (2.0 + torch.arange(threads, device="cuda") / 512).to(dtype)
    check(z, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [129, 256])
@pytest.mark.parametrize("vocab", [1030, 8000])
def test_every_vector_alike(vocab, k, dtype):
    per = 8 if dtype == BF16 else 4
    one = torch.randn(per, generator=gen(k), device="cuda")
    z = one.repeat(vocab // per + 1)[:vocab].repeat(2, 1).to(dtype)
    check(z, k)
    check(torch.full((2, vocab), -0.5, dtype=dtype, device="cuda"), k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [64, 129, 200, 256])
@pytest.mark.parametrize("share", [1016, 1024, 1025])
@pytest.mark.parametrize("ctas", [2, 4, 8])
def test_shares_of_a_cluster(ctas, share, k, dtype):
    """Rows that several CTAs take, shares of about 1,024 vectors each."""
    per = 8 if dtype == BF16 else 4
    vocab = ctas * share * per - per + 1
    check(peaks(1, vocab, dtype, per, 5.0, ctas), k)
    check(peaks(1, vocab, dtype, per, (8.0, 12.0), ctas + 1), k)
    z = torch.full((1, vocab), -1.0, dtype=dtype, device="cuda")
    z[:, -(share - 1) * per::per] = 2.0     # all in the last share
    check(z, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [129, 256])
def test_rows_start_anywhere(k, dtype):
    z = peaks(4, 3000, dtype, 8, 5.0, k)
    for offset in (1, 3, 5):
        flat = torch.full((offset + 4 * 3003 + 16,), 100.0, dtype=dtype, device="cuda")
        view = flat[offset:offset + 4 * 3003].view(4, 3003)[:, :3000]
        view.copy_(z)
        check(view, k)
