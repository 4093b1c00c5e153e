"""Matrix products of small whole numbers, which every kernel must give bit for
bit, and the accuracy of long fp32 sums (GPU).

Operands of -2 to 2 have whole products and sums below 2^24, exact in fp32 in
any order and with any rounding: a term that is dropped, doubled or taken from
the wrong place shows however long the sum is.

For the accuracy: adding n terms of a random sum one by one, rounding each time
to nearest, errs by some 0.6 2^-24 |s_j| at step j with |s_j| ~ sqrt(j): in the
norm 0.6 2^-24 sqrt(n / 2) of the result.  The kernels' fp32 results must not be
worse."""
import pytest
import torch

from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# tokens, features, inputs: one token; each width of the small tiles, shared by one
# to eight CTAs; paired tiles, a round of them and more; sums that end inside a block
SHAPES = [(1, 1003, 4104), (2, 130, 72), (8, 300, 4104), (9, 257, 1032), (16, 128, 8200), (17, 1000, 520),
          (33, 129, 4096), (64, 640, 2056), (65, 130, 8), (100, 1003, 4096), (129, 4096, 136), (300, 700, 14336),
          (1001, 1003, 4096), (2311, 2497, 1032), (4096, 4104, 72)]


def whole(*shape, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(BF16)


def normal(*shape, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(BF16)


def wide(t):
    """The same values in rows that the products can read."""
    rows, cols = t.shape
    made = torch.zeros(rows, -(-cols // 8) * 8, dtype=t.dtype, device=t.device)
    made[:, :cols] = t
    return made[:, :cols]


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("tokens,features,inputs", SHAPES)
def test_whole_numbers(tokens, features, inputs, out):
    x, r = whole(tokens, inputs, seed=1), whole(features, inputs, seed=2)
    dz = wide(whole(tokens, features, seed=3))
    bias = whole(features, seed=4).float()
    made = api.linear(x, r, bias=bias, out_dtype=out)["y"]
    back = api.linear_backward(dz, x, r, bias=True, dx_dtype=out, dr_dtype=out)
    api.check_device()
    assert torch.equal(made, (x.double() @ r.double().t() + bias.double()).to(out))
    assert torch.equal(back["dx"], (dz.double() @ r.double()).to(out))
    assert torch.equal(back["dr"], (dz.double().t() @ x.double()).to(out))
    assert torch.equal(back["dbias"], dz.double().sum(0).float())


@pytest.mark.parametrize("n", [4096, 14336])
@pytest.mark.parametrize("rows,cols", [(24, 512), (300, 257), (2400, 2304)])
def test_long_sums_in_fp32(rows, cols, n):
    """The sum runs over the inputs, the features and the tokens in turn: the
    three layouts of the operands."""
    bound = 0.6 * 2.0 ** -24 * (n / 2) ** 0.5

    def check(got, want):
        off = float((got.double() - want).norm() / want.norm())
        assert off <= bound, off / bound

    x, r = normal(rows, n, seed=1), normal(cols, n, seed=2, scale=0.05)
    check(api.linear(x, r, out_dtype=F32)["y"], x.double() @ r.double().t())
    dz, r = normal(rows, n, seed=3), normal(n, cols // 8 * 8, seed=4, scale=0.05)
    x = normal(rows, cols // 8 * 8, seed=5)
    check(api.linear_backward(dz, x, r, dr=False, dx_dtype=F32)["dx"], dz.double() @ r.double())
    dz, x = wide(normal(n, cols, seed=6)), normal(n, rows // 8 * 8, seed=7)
    r = normal(cols, rows // 8 * 8, seed=8)
    check(api.linear_backward(dz, x, r, dx=False, dr_dtype=F32)["dr"], dz.double().t() @ x.double())
    api.check_device()
