"""Products over nothing: no inputs forward, no features or no tokens backward.  The sum is
0, the epilogue applies, and no operand is looked at (GPU)."""
import pytest
import torch

from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def rand(*shape, seed, dtype=BF16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def nothing(rows, cols):
    return torch.empty(rows, cols, dtype=BF16, device="cuda")


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("tokens", [1, 5, 20, 40, 100, 300])
def test_no_inputs(tokens, out):
    features = 259
    bias, residual = rand(features, seed=1, dtype=F32), rand(tokens, features, seed=2, dtype=out)
    made = api.linear(nothing(tokens, 0), nothing(features, 0), bias=bias, activation="relu",
                      residual=residual, out_dtype=out, save_pre=True)
    api.check_device()
    z = bias.expand(tokens, features)
    assert torch.equal(made["y"], (z.clamp(min=0.0) + residual.float()).to(out))
    assert torch.equal(made["pre"], z.to(BF16))


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("tokens", [1, 5, 40, 100, 300])
def test_no_features(tokens, out):
    inputs = 264
    pre, residual = rand(tokens, inputs, seed=3), rand(tokens, inputs, seed=4, dtype=out)
    made = api.linear_backward(nothing(tokens, 0), rand(tokens, inputs, seed=5), nothing(0, inputs),
                               pre_in=pre, activation_in="silu", residual=residual, dx_dtype=out)
    api.check_device()
    assert torch.equal(made["dx"], residual) and made["dr"].shape == (0, inputs)


@pytest.mark.parametrize("features,inputs", [(24, 16), (300, 1032), (1, 8), (24, 0)])
def test_no_tokens(features, inputs):
    made = api.linear_backward(nothing(0, features), nothing(0, inputs), rand(features, inputs, seed=6),
                               bias=True, dr_dtype=F32)
    api.check_device()
    assert made["dx"].shape == (0, inputs) and made["dr"].shape == (features, inputs)
    assert not made["dr"].any() and not made["dbias"].any()
