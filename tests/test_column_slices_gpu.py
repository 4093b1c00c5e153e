"""Operands and results that are columns of one buffer: they share no byte, and the calls take
them (GPU).  Results are compared bit for bit with those of separate buffers."""
import pytest
import torch

from paper_2608_13966_gb300 import api
from paper_2608_13966_gb300 import quasar as Q

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
OK, INVALID = Q.QuasarStatus.OK, Q.QuasarStatus.ERR_INVALID_ARG


def rand(*shape, seed, dtype=BF16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def side_by_side(*parts, gap=0):
    """The matrices as columns of one buffer, `gap` marked columns after each."""
    rows = parts[0].shape[0]
    buffer = torch.full((rows, sum(p.shape[1] + gap for p in parts)), 77.0, dtype=parts[0].dtype, device="cuda")
    views, at = [], 0
    for p in parts:
        view = buffer[:, at:at + p.shape[1]]
        view.copy_(p)
        views.append(view)
        at += p.shape[1] + gap
    return buffer, views


@pytest.mark.parametrize("gap", [0, 8])
@pytest.mark.parametrize("tokens,features,inputs", [(1, 64, 72), (30, 72, 264), (300, 520, 136), (2400, 2304, 72)])
def test_linear(tokens, features, inputs, gap):
    x, r = rand(tokens, inputs, seed=1), rand(features, inputs, seed=2)
    res = rand(tokens, features, seed=3)
    want = api.linear(x, r, activation="silu", residual=res, save_pre=True)
    empty = torch.zeros(tokens, features, dtype=BF16, device="cuda")
    buffer, (y, x, pre, res) = side_by_side(empty, x, empty, res, gap=gap)
    ld = buffer.stride(0)
    st = Q.quasar_linear(x, ld, r, inputs, None, "silu", res, ld, tokens, features, inputs, y, Q.BF16, ld, pre, ld)
    assert st == OK
    api.check_device()
    assert torch.equal(y, want["y"]) and torch.equal(pre, want["pre"])
    assert (buffer == 77.0).sum() >= 4 * gap * tokens


@pytest.mark.parametrize("tokens,features,inputs", [(1, 64, 72), (7, 64, 72), (30, 72, 264), (300, 520, 136)])
def test_linear_backward(tokens, features, inputs):
    dz, x, r = rand(tokens, features, seed=1), rand(tokens, inputs, seed=2), rand(features, inputs, seed=3)
    pre, res = rand(tokens, inputs, seed=4), rand(tokens, inputs, seed=5)
    want = api.linear_backward(dz, x, r, pre_in=pre, activation_in="gelu", residual=res)
    _, (dx, dz, x, pre, res) = side_by_side(torch.zeros_like(x), dz, x, pre, res)
    _, (r, dr) = side_by_side(r, torch.zeros_like(r))
    ld, ld_r = dz.stride(0), r.stride(0)
    assert Q.quasar_linear_grad_input(dz, ld, r, ld_r, pre, ld, "gelu", res, ld, tokens, features, inputs, dx,
                                      Q.BF16, ld) == OK
    assert Q.quasar_linear_grad_weight(dz, ld, x, ld, tokens, features, inputs, dr, Q.BF16, ld_r) == OK
    dy, _ = rand(tokens, features, seed=6), None
    grad = api.activation_grad(dy, dz, "silu")
    _, (dy, p, out) = side_by_side(dy, dz, torch.zeros_like(dy))
    assert Q.quasar_activation_grad(dy, dy.stride(0), p, dy.stride(0), "silu", tokens, features, out,
                                    dy.stride(0)) == OK
    api.check_device()
    assert torch.equal(dx, want["dx"]) and torch.equal(dr, want["dr"]) and torch.equal(out, grad)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", [(1, 1003), (9, 1003), (200, 5001), (3, 70001)])
def test_logits(rows, vocab, dtype):
    z = rand(rows, vocab, seed=1, dtype=dtype)
    t = api.top_logits(rand(rows, vocab, seed=2, dtype=dtype), 20)
    _, (grad, z, back) = side_by_side(torch.zeros_like(z), z, torch.zeros_like(z), gap=1)
    # (of the same rows: where a row starts within 16 bytes orders its sums)
    want = api.distill_top(z, t["indices"], t["values"], stats=True)
    made = api.distill_top(z, t["indices"], t["values"], stats=True, out=grad)
    api.distill_top_backward(z, t["indices"], t["values"], made["stats"], None, out=back)
    api.check_device()
    assert torch.equal(grad, want["grad"]) and torch.equal(made["loss"], want["loss"])
    again = api.distill_top_backward(z, t["indices"], t["values"], made["stats"], None)
    assert torch.equal(back, again)


def test_columns_that_meet_are_still_refused():
    buffer = torch.zeros(8, 200, dtype=BF16, device="cuda")
    x, r = buffer[:, :64], torch.zeros(32, 64, dtype=BF16, device="cuda")

    def linear(y, ld=200, **kw):
        return Q.quasar_linear(x, 200, r, 64, None, "none", None, 0, 8, 32, 64, y, Q.BF16, ld, **kw)

    assert linear(buffer[:, 64:]) == OK
    assert linear(buffer[:, 63:]) == INVALID
    assert linear(buffer[:, 169:]) == INVALID          # the last column is the next row's first
    assert linear(buffer[:, 64:], ld=192) == INVALID   # other strides: by the bytes they span
    assert linear(buffer[:, 64:], pre=buffer[:, 95:], ld_pre=200) == INVALID
    assert linear(buffer[:, 64:], pre=buffer[:, 96:], ld_pre=200) == OK
    torch.cuda.synchronize()
