"""Tensors of one call on two devices, or on one that is not current, are refused before
anything is allocated or launched (host: stand-ins that only describe a tensor)."""
import pytest
import torch

from paper_2608_13966_gb300 import api

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Described:
    """What the checks ask of a tensor."""

    def __init__(self, *shape, dtype=BF16, at=0):
        self.shape, self.dtype, self.at = torch.Size(shape), dtype, at
        self.is_cuda, self.device = True, torch.device("cuda", at)

    def stride(self):
        return (self.shape[1], 1) if len(self.shape) == 2 else (1,)

    def get_device(self):
        return self.at

    def is_contiguous(self):
        return True


def calls():
    """Every call with all of its tensors, by name."""
    m, n, k, v = 4, 32, 64, 100

    def linear(t):
        return lambda: api.linear(t["x"], t["r"], bias=t["bias"], residual=t["residual"])

    def activation_grad(t):
        return lambda: api.activation_grad(t["dy"], t["pre"], "silu")

    def linear_backward(t):
        return lambda: api.linear_backward(t["dz"], t["x"], t["r"], pre_in=t["pre_in"],
                                           activation_in="silu", residual=t["residual"])

    def top_logits(t):
        return lambda: api.top_logits(t["logits"], 3)

    def distill_top(t):
        return lambda: api.distill_top(t["logits"], t["indices"], t["values"],
                                       teacher_lse=t["teacher_lse"], row_weight=t["row_weight"])

    def distill_top_backward(t):
        return lambda: api.distill_top_backward(t["logits"], t["indices"], t["values"], t["stats"],
                                                t["row_weight"], teacher_lse=t["teacher_lse"])

    lists = {"logits": ((m, v), F32), "indices": ((m, 3), I32), "values": ((m, 3), F32),
             "teacher_lse": ((m,), F32), "row_weight": ((m,), F32)}
    return [
        (linear, {"x": ((m, k), BF16), "r": ((n, k), BF16), "bias": ((n,), F32),
                  "residual": ((m, n), BF16)}),
        (activation_grad, {"dy": ((m, n), BF16), "pre": ((m, n), BF16)}),
        (linear_backward, {"dz": ((m, n), BF16), "x": ((m, k), BF16), "r": ((n, k), BF16),
                           "pre_in": ((m, k), BF16), "residual": ((m, k), BF16)}),
        (top_logits, {"logits": ((m, v), F32)}),
        (distill_top, lists),
        (distill_top_backward, lists | {"stats": ((m, 2), F32)}),
    ]


@pytest.mark.parametrize("call,tensors", calls(), ids=lambda x: getattr(x, "__name__", ""))
def test_tensors_elsewhere(call, tensors, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    names = list(tensors)
    for odd in names[1:]:
        made = {n: Described(*tensors[n][0], dtype=tensors[n][1], at=int(n == odd)) for n in names}
        with pytest.raises(ValueError, match=f"{odd} must be on cuda:0.*not on cuda:1"):
            call(made)()


@pytest.mark.parametrize("call,tensors", calls(), ids=lambda x: getattr(x, "__name__", ""))
def test_all_of_them_elsewhere(call, tensors, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    made = {n: Described(*shape, dtype=dtype, at=1) for n, (shape, dtype) in tensors.items()}
    with pytest.raises(ValueError, match="on cuda:1, but the current device is cuda:0"):
        call(made)()
