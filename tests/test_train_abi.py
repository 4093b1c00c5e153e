"""Refusals of the operators around the reconstruction, on the host: bad
arguments return a status and launch nothing (no GPU needed; addresses are
fake, so nothing here may pass validation except no-ops)."""
import pytest
import torch

from paper_2608_13966_gb300 import api
from paper_2608_13966_gb300 import build as qbuild
from paper_2608_13966_gb300 import quasar as Q

A, B, C, D, E, F = (0x10000000 * (i + 1) for i in range(6))
OK, INVALID, UNSUPPORTED = (Q.QuasarStatus.OK, Q.QuasarStatus.ERR_INVALID_ARG,
                            Q.QuasarStatus.ERR_UNSUPPORTED)


@pytest.fixture(scope="module", autouse=True)
def lib():
    qbuild.build()
    return Q.load(build_if_missing=False)


def _linear(**kw):
    args = dict(x=A, ld_x=64, r=B, ld_r=64, bias=None, activation="none", residual=None,
                ld_residual=0, tokens=4, features=32, inputs=64, y=C, y_dtype=Q.BF16, ld_y=32,
                pre=None, ld_pre=0, stream=0)
    args.update(kw)
    return Q.quasar_linear(**args)


@pytest.mark.parametrize("kw,expect", [
    (dict(x=None), INVALID),
    (dict(r=None), INVALID),
    (dict(y=None), INVALID),
    (dict(x=A + 8), INVALID),                        # operands are 16-byte aligned
    (dict(r=B + 2), INVALID),
    (dict(ld_x=68), INVALID),                        # and so are their rows
    (dict(ld_r=65), INVALID),
    (dict(ld_x=56), INVALID),                        # a row stride below the row
    (dict(ld_y=31), INVALID),
    (dict(y=C + 1), INVALID),
    (dict(bias=D + 2), INVALID),
    (dict(activation=4), INVALID),
    (dict(activation=-1), INVALID),
    (dict(y_dtype=2), INVALID),
    (dict(tokens=-1), INVALID),
    (dict(tokens=1 << 32), INVALID),
    (dict(features=1 << 31, ld_y=1 << 31), INVALID),
    (dict(y=A + 128), INVALID),                      # y overlaps x
    (dict(y=B + 128), INVALID),                      # y overlaps r
    (dict(residual=C + 2, ld_residual=32), INVALID),  # y overlaps the residual, shifted
    (dict(residual=C, ld_residual=40), INVALID),      # ... with another stride
    (dict(residual=D, ld_residual=16), INVALID),
    (dict(pre=C + 64, ld_pre=32), INVALID),           # pre overlaps y
    (dict(pre=A, ld_pre=32), INVALID),                # pre overlaps x
    (dict(pre=D, ld_pre=8), INVALID),
    (dict(tokens=0), OK),
    (dict(features=0, ld_y=0), OK),
])
def test_linear_arguments(kw, expect):
    assert _linear(**kw) == expect


def _grad_input(**kw):
    args = dict(dz=A, ld_dz=32, r=B, ld_r=64, pre_in=None, ld_pre_in=0, activation_in="none",
                residual=None, ld_residual=0, tokens=4, features=32, inputs=64, dx=C,
                dx_dtype=Q.BF16, ld_dx=64, stream=0)
    args.update(kw)
    return Q.quasar_linear_grad_input(**args)


@pytest.mark.parametrize("kw,expect", [
    (dict(dz=None), INVALID),
    (dict(dz=A + 4), INVALID),
    (dict(ld_dz=33), INVALID),
    (dict(r=None), INVALID),
    (dict(dx=None), INVALID),
    (dict(ld_dx=60), INVALID),
    (dict(activation_in="silu"), INVALID),                           # no pre-activation
    (dict(activation_in="silu", pre_in=D, ld_pre_in=8), INVALID),
    (dict(activation_in=9), INVALID),
    (dict(dx=A), INVALID),
    (dict(dx=B + 512), INVALID),
    (dict(activation_in="gelu", pre_in=C, ld_pre_in=64, dx_dtype=Q.F32), INVALID),
    (dict(activation_in="gelu", pre_in=C + 2, ld_pre_in=64), INVALID),
    (dict(residual=C + 64, ld_residual=64), INVALID),
    (dict(tokens=0), OK),
])
def test_grad_input_arguments(kw, expect):
    assert _grad_input(**kw) == expect


def _grad_weight(**kw):
    args = dict(dz=A, ld_dz=32, x=B, ld_x=64, tokens=4, features=32, inputs=64, dr=C,
                dr_dtype=Q.F32, ld_dr=64, dbias=D, stream=0)
    args.update(kw)
    return Q.quasar_linear_grad_weight(**args)


@pytest.mark.parametrize("kw,expect", [
    (dict(dz=None), INVALID),
    (dict(x=None), INVALID),
    (dict(x=B + 8), INVALID),
    (dict(ld_x=63), INVALID),
    (dict(ld_dr=63), INVALID),
    (dict(dr=C + 2), INVALID),
    (dict(dr_dtype=3), INVALID),
    (dict(dr=A), INVALID),
    (dict(dr=B + 64), INVALID),
    (dict(dbias=D + 1), INVALID),
    (dict(dbias=C + 4), INVALID),
    (dict(dbias=A), INVALID),
    (dict(dr=None, dbias=None), OK),
    (dict(features=0, ld_dz=0), OK),
])
def test_grad_weight_arguments(kw, expect):
    assert _grad_weight(**kw) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(dy=None), INVALID),
    (dict(dz=None), INVALID),
    (dict(pre=None), INVALID),
    (dict(activation=7), INVALID),
    (dict(ld_dy=15), INVALID),
    (dict(ld_pre=15), INVALID),
    (dict(dz=A + 2), INVALID),
    (dict(dz=B + 2), INVALID),
    (dict(rows=0), OK),
])
def test_activation_grad_arguments(kw, expect):
    args = dict(dy=A, ld_dy=16, pre=B, ld_pre=16, activation="silu", rows=4, cols=16, dz=C,
                ld_dz=16, stream=0)
    args.update(kw)
    assert Q.quasar_activation_grad(**args) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(logits=None), INVALID),
    (dict(logits=A + 1), INVALID),
    (dict(dtype=5), INVALID),
    (dict(ld=99), INVALID),
    (dict(k=0), INVALID),
    (dict(k=101), INVALID),
    (dict(vocab=1000, ld=1000, k=257), UNSUPPORTED),
    (dict(vocab=0, k=1), INVALID),
    (dict(temperature=0.0), INVALID),
    (dict(temperature=-1.0), INVALID),
    (dict(temperature=float("nan")), INVALID),
    (dict(temperature=float("inf")), INVALID),
    (dict(values=None), INVALID),
    (dict(indices=None), INVALID),
    (dict(indices=C + 2), INVALID),
    (dict(values=A + 16), INVALID),
    (dict(lse=B + 4), INVALID),
    (dict(indices=B), INVALID),
    (dict(rows=0), OK),
])
def test_top_logits_arguments(kw, expect):
    args = dict(logits=A, dtype=Q.BF16, ld=100, rows=4, vocab=100, k=8, temperature=1.0, values=B,
                indices=C, lse=D, stream=0)
    args.update(kw)
    assert Q.quasar_top_logits(**args) == expect


def _distill(**kw):
    args = dict(logits=A, dtype=Q.F32, ld=100, rows=4, vocab=100, indices=B, values=C, k=8,
                teacher_lse=None, row_weight=None, temperature=1.0, loss=D, stats=E, grad=F,
                ld_grad=100, stream=0)
    args.update(kw)
    return Q.quasar_distill_top(**args)


@pytest.mark.parametrize("kw,expect", [
    (dict(logits=None), INVALID),
    (dict(logits=A + 2), INVALID),
    (dict(indices=None), INVALID),
    (dict(values=None), INVALID),
    (dict(loss=None), INVALID),
    (dict(k=0), INVALID),
    (dict(k=101), INVALID),
    (dict(vocab=1000, ld=1000, ld_grad=1000, k=257), UNSUPPORTED),
    (dict(temperature=0.0), INVALID),
    (dict(ld_grad=99), INVALID),
    (dict(grad=F + 2), INVALID),
    (dict(grad=A + 400), INVALID),            # overlaps the logits, shifted
    (dict(grad=A, ld_grad=104), INVALID),     # ... with another stride
    (dict(grad=B), INVALID),
    (dict(loss=A + 16), INVALID),
    (dict(stats=D), INVALID),
    (dict(loss=C), INVALID),
    (dict(row_weight=D + 4), INVALID),
    (dict(teacher_lse=E), INVALID),
    (dict(rows=0), OK),
])
def test_distill_arguments(kw, expect):
    assert _distill(**kw) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(stats=None), INVALID),
    (dict(grad=None), INVALID),
    (dict(grad=D), INVALID),                  # the statistics are read
    (dict(grad=C), INVALID),
    (dict(rows=0), OK),
])
def test_distill_backward_arguments(kw, expect):
    args = dict(logits=A, dtype=Q.F32, ld=100, rows=4, vocab=100, indices=B, values=C, k=8,
                teacher_lse=None, stats=D, row_weight=None, temperature=1.0, grad=F, ld_grad=100,
                stream=0)
    args.update(kw)
    assert Q.quasar_distill_top_backward(**args) == expect


def test_api_refuses_what_it_cannot_pass_on():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        api.linear(x, x)
    with pytest.raises(ValueError, match="2-D"):
        api.linear(x[0], x)
    with pytest.raises(ValueError, match="contiguous rows"):
        api.top_logits(x.t(), 2)
    with pytest.raises(ValueError, match="CUDA"):
        api.distill_top(x, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))
