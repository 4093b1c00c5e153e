"""The activations and their slopes where a pre-activation is not a number, in
every kernel that applies them: one token, few tiles, shared tiles, paired tiles,
and the gradient through a layer's own activation (GPU)."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan
BF16, F32 = torch.bfloat16, torch.float32
SHAPES = [(1, 300, 72), (40, 300, 72), (130, 257, 2056), (2311, 2497, 72)]


def rand(*shape, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(BF16)


@pytest.mark.parametrize("tokens,features,inputs", SHAPES)
@pytest.mark.parametrize("activation", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("out", [BF16, F32])
def test_nan_goes_through_the_activation(tokens, features, inputs, activation, out):
    x, r = rand(tokens, inputs, seed=1), rand(features, inputs, seed=2, scale=0.1)
    bias = torch.zeros(features, device="cuda")
    clean = api.linear(x, r, bias=bias, activation=activation, out_dtype=out, save_pre=True)
    bias[7], bias[features - 1] = NAN, NAN
    made = api.linear(x, r, bias=bias, activation=activation, out_dtype=out, save_pre=True)
    api.check_device()
    for name in ("y", "pre"):
        assert torch.isnan(made[name][:, [7, features - 1]]).all(), name
        assert torch.equal(made[name][:, 8:-1], clean[name][:, 8:-1]), name


@pytest.mark.parametrize("activation", ["relu", "silu", "gelu"])
def test_nan_goes_through_the_slope(activation):
    dy, pre = rand(9, 301, seed=3), rand(9, 301, seed=4)
    clean = api.activation_grad(dy, pre, activation)
    pre[2, 5] = NAN
    dz = api.activation_grad(dy, pre, activation)
    assert bool(torch.isnan(dz[2, 5]))
    dz[2, 5] = clean[2, 5]
    assert torch.equal(dz, clean)
    for tokens, features, inputs in SHAPES:
        dz, x, r = rand(tokens, features, seed=5), rand(tokens, inputs, seed=6), rand(features, inputs, seed=7)
        pre = rand(tokens, inputs, seed=8)
        pre[tokens - 1, inputs - 2] = NAN
        dx = api.linear_backward(dz, x, r, dr=False, pre_in=pre, activation_in=activation)["dx"]
        api.check_device()
        assert bool(torch.isnan(dx[tokens - 1, inputs - 2])) and int(torch.isnan(dx).sum()) == 1


@pytest.mark.parametrize("activation,low", [("relu", 0.0), ("silu", 0.0), ("gelu", 0.0)])
def test_an_infinite_pre_activation_has_slope_0_or_1(activation, low):
    """A kept pre-activation past bf16's range is infinite: the slope is its limit there."""
    far = torch.tensor([[-INF, -3e38, -200.0, 200.0, 3e38, INF, 0.5]], dtype=BF16, device="cuda")
    got = api.activation_grad(torch.full_like(far, 2.0), far, activation)[0, :6].float()
    assert got.tolist() == [low, low, low, 2.0, 2.0, 2.0]
    for tokens, features, inputs in SHAPES:
        dz, x, r = rand(tokens, features, seed=5), rand(tokens, inputs, seed=6), rand(features, inputs, seed=7)
        pre = torch.full((tokens, inputs), INF, dtype=BF16, device="cuda")
        pre[:, ::3] = -INF
        plain = api.linear_backward(dz, x, r, dr=False)["dx"]
        dx = api.linear_backward(dz, x, r, dr=False, pre_in=pre, activation_in=activation)["dx"]
        api.check_device()
        assert (dx[:, ::3] == 0).all()
        assert torch.equal(dx[:, 1::3], plain[:, 1::3]) and torch.equal(dx[:, 2::3], plain[:, 2::3])
