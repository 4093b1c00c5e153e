"""Rows that hold a NaN or an infinity, in each kernel that a row's length and place choose: such a row
is not finite as the formula has it, and the others are what they are without it (GPU)."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
COLS = [8, 63, 128, 250, 512, 1000, 1003, 1032, 2048, 4096, 4099, 8192, 16384, 16392]


def made(rows, cols, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + cols)
    return torch.randn(rows, cols, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("cols", COLS)
def test_forward(cols, dtype, center):
    x = made(7, cols, dtype, 0)
    clean = api.layer_norm(x, center=center, stats=True)
    x[2, cols // 2] = math.nan
    x[4, cols - 1] = math.inf
    x[5, 0] = -math.inf
    o = api.layer_norm(x, center=center, stats=True)
    y, stats = o["y"], o["stats"]
    assert y[2].isnan().all() and stats[2, 1].isnan()
    if center:  # the mean is not finite: nothing less it is
        assert y[4].isnan().all() and y[5].isnan().all()
    else:       # 1 / rms is 0
        for row, at in ((4, cols - 1), (5, 0)):
            assert y[row, at].isnan() and stats[row, 1] == 0
            assert (y[row, :at] == 0).all() and (y[row, at + 1:] == 0).all()
    for row in (0, 1, 3, 6):
        assert torch.equal(y[row], clean["y"][row]) and torch.equal(stats[row], clean["stats"][row])


@pytest.mark.parametrize("cols", COLS)
def test_backward(cols):
    """A NaN in dy: its row of dx, and its column of the sums over the rows, no others."""
    x, dy = made(7, cols, BF16, 0), made(7, cols, BF16, 3)
    stats = api.layer_norm(x, stats=True)["stats"]
    clean = api.layer_norm_backward(dy, x, None, stats, dbias=True)
    at = cols // 2
    dy[2, at] = math.nan
    o = api.layer_norm_backward(dy, x, None, stats, dbias=True)
    assert o["dx"][2].isnan().all()
    rows, columns = (torch.arange(n, device="cuda") for n in (7, cols))
    assert torch.equal(o["dx"][rows != 2], clean["dx"][rows != 2])
    for name in ("dweight", "dbias"):
        assert o[name][at].isnan() and torch.equal(o[name][columns != at], clean[name][columns != at])
