"""Refusals of embedding, layer norm and attention on the host: bad arguments return a
status and launch nothing (no GPU needed; addresses are fake, so nothing here may pass
validation except no-ops)."""
import pytest
import torch

from paper_2608_13966_gb300 import api
from paper_2608_13966_gb300 import build as qbuild
from paper_2608_13966_gb300 import quasar as Q
from tests.test_devices import BF16, F32, I32, Described

A, B, C, D, E, F, G, H = (0x10000000 * (i + 1) for i in range(8))
OK, INVALID, UNSUPPORTED = (Q.QuasarStatus.OK, Q.QuasarStatus.ERR_INVALID_ARG,
                            Q.QuasarStatus.ERR_UNSUPPORTED)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def lib():
    qbuild.build()
    return Q.load(build_if_missing=False)


@pytest.mark.parametrize("kw,expect", [
    (dict(ids=None), INVALID),
    (dict(ids=A + 2), INVALID),
    (dict(ids=A + 4, ids_type=Q.I64), INVALID),
    (dict(ids_type=2), INVALID),
    (dict(table=None), INVALID),
    (dict(table=B + 1), INVALID),
    (dict(table_dtype=7), INVALID),
    (dict(ld_table=63), INVALID),
    (dict(y=None), INVALID),
    (dict(y_dtype=-1), INVALID),
    (dict(ld_y=63), INVALID),
    (dict(tokens=-1), INVALID),
    (dict(vocab=1 << 31), INVALID),
    (dict(residual=D, ld_residual=60), INVALID),
    (dict(residual=C + 2, ld_residual=64), INVALID),   # y overlaps the residual, shifted
    (dict(residual=C, ld_residual=72), INVALID),
    (dict(y=B + 128), INVALID),
    (dict(y=A), INVALID),
    (dict(tokens=0), OK),
    (dict(width=0, ld_table=0, ld_y=0), OK),
    (dict(width=1 << 28, ld_table=1 << 28, ld_y=1 << 28, vocab=1, tokens=1, y=H << 8), UNSUPPORTED),
])
def test_embedding_arguments(kw, expect):
    args = dict(ids=A, ids_type=Q.I32, tokens=4, table=B, table_dtype=Q.BF16, ld_table=64, vocab=10, width=64,
                scale=1.0, residual=None, ld_residual=0, y=C, y_dtype=Q.BF16, ld_y=64, stream=0)
    assert Q.quasar_embedding(**(args | kw)) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(dy=None), INVALID),
    (dict(dy=A + 1), INVALID),
    (dict(ld_dy=60), INVALID),
    (dict(ids=None), INVALID),
    (dict(ids_type=3), INVALID),
    (dict(dtable=None), INVALID),
    (dict(ld_dtable=3), INVALID),
    (dict(dtable_dtype=9), INVALID),
    (dict(accumulate=2), INVALID),
    (dict(workspace=None), INVALID),
    (dict(workspace=D + 8), INVALID),
    (dict(workspace_bytes=63), INVALID),
    (dict(dtable=A + 64), INVALID),
    (dict(workspace=C + 64), INVALID),
    (dict(workspace=A), INVALID),
    (dict(tokens=0, accumulate=1), OK),
    (dict(vocab=0), OK),
])
def test_embedding_backward_arguments(kw, expect):
    args = dict(dy=A, dy_dtype=Q.BF16, ld_dy=64, ids=B, ids_type=Q.I32, tokens=4, vocab=10, width=64, scale=1.0,
                dtable=C, dtable_dtype=Q.BF16, ld_dtable=64, accumulate=0, workspace=D, workspace_bytes=64, stream=0)
    assert Q.quasar_embedding_backward(**(args | kw)) == expect


def test_embedding_workspace():
    assert Q.quasar_embedding_backward_workspace(4, 64) == 4 * 16
    assert Q.quasar_embedding_backward_workspace(300, 7) == 4 * 1200 + 9 * 4 * 7
    with pytest.raises(Q.QuasarError):
        Q.quasar_embedding_backward_workspace(-1, 7)


@pytest.mark.parametrize("kw,expect", [
    (dict(x=None), INVALID),
    (dict(x=A + 1), INVALID),
    (dict(x_dtype=4), INVALID),
    (dict(ld_x=60), INVALID),
    (dict(y=None), INVALID),
    (dict(ld_y=60), INVALID),
    (dict(eps=-1e-5), INVALID),
    (dict(eps=NAN), INVALID),
    (dict(eps=INF), INVALID),
    (dict(center=2), INVALID),
    (dict(weight=C + 2), INVALID),
    (dict(bias=D + 1), INVALID),
    (dict(stats=E + 2), INVALID),
    (dict(y=A + 2), INVALID),
    (dict(y=A, y_dtype=Q.F32), INVALID),               # in place only of the same type
    (dict(y=C), INVALID),
    (dict(stats=A), INVALID),
    (dict(stats=B), INVALID),
    (dict(cols=0, ld_x=0, ld_y=0), INVALID),
    (dict(rows=0), OK),
])
def test_layer_norm_arguments(kw, expect):
    args = dict(x=A, x_dtype=Q.BF16, ld_x=64, weight=C, bias=D, rows=4, cols=64, center=1, eps=1e-5, y=B,
                y_dtype=Q.BF16, ld_y=64, stats=E, stream=0)
    assert Q.quasar_layer_norm(**(args | kw)) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(dy=None), INVALID),
    (dict(x=None), INVALID),
    (dict(ld_dy=60), INVALID),
    (dict(ld_x=60), INVALID),
    (dict(stats=None), INVALID),
    (dict(stats=D + 2), INVALID),
    (dict(center=-1), INVALID),
    (dict(dx=E + 1), INVALID),
    (dict(dx_dtype=6), INVALID),
    (dict(ld_dx=63), INVALID),
    (dict(residual=F, ld_residual=63), INVALID),
    (dict(dx=None, residual=F, ld_residual=64), INVALID),
    (dict(dx=A + 2), INVALID),
    (dict(dx=A, dx_dtype=Q.F32), INVALID),
    (dict(dx=C), INVALID),
    (dict(dweight=A), INVALID),
    (dict(dweight=G + 1), INVALID),
    (dict(dbias=G + 4), INVALID),
    (dict(cols=0, ld_dy=0, ld_x=0, ld_dx=0), INVALID),
    (dict(dx=None, dweight=None), OK),
])
def test_layer_norm_backward_arguments(kw, expect):
    args = dict(dy=A, dy_dtype=Q.BF16, ld_dy=64, x=B, x_dtype=Q.BF16, ld_x=64, weight=C, stats=D, rows=4, cols=64,
                center=1, residual=None, ld_residual=0, dx=E, dx_dtype=Q.BF16, ld_dx=64, dweight=G, dbias=None,
                workspace=None, workspace_bytes=0, stream=0)
    assert Q.quasar_layer_norm_backward(**(args | kw)) == expect


ATTENTION = dict(q=A, ld_q=256, k=B, ld_k=128, v=C, ld_v=128, tokens=10, keys=12, heads=4, kv_heads=2, head_dim=64,
                 starts=D, key_starts=E, sequences=2, causal=1, scale=0.125, y=F, ld_y=256, lse=G, stream=0)
SHARED = [
    (dict(q=None), INVALID),
    (dict(q=A + 8), INVALID),                          # operands are 16-byte aligned
    (dict(k=B + 2), INVALID),
    (dict(ld_k=132), INVALID),                         # and so are their rows
    (dict(ld_q=248), INVALID),
    (dict(v=None), INVALID),
    (dict(y=None), INVALID),
    (dict(y=F + 8), INVALID),
    (dict(heads=3), INVALID),
    (dict(heads=0), INVALID),
    (dict(kv_heads=0), INVALID),
    (dict(head_dim=60), INVALID),
    (dict(head_dim=0), INVALID),
    (dict(head_dim=136, ld_q=544, ld_k=272, ld_v=272, ld_y=544, ld_dy=544, ld_dq=544, ld_dk=272, ld_dv=272), UNSUPPORTED),
    (dict(heads=258, ld_q=258 * 64, ld_y=258 * 64, ld_dy=258 * 64, ld_dq=258 * 64, tokens=1), UNSUPPORTED),
    (dict(sequences=-1), INVALID),
    (dict(sequences=1 << 25), INVALID),
    (dict(starts=None), INVALID),
    (dict(key_starts=None), INVALID),
    (dict(starts=None, key_starts=None, sequences=0), INVALID),
    (dict(starts=D + 2), INVALID),
    (dict(causal=2), INVALID),
    (dict(scale=0.0), INVALID),
    (dict(scale=-1.0), INVALID),
    (dict(scale=INF), INVALID),
    (dict(scale=3e38), INVALID),  # not finite in bits
    (dict(scale=NAN), INVALID),
    (dict(lse=G + 2), INVALID),
    (dict(tokens=-1), INVALID),
]


@pytest.mark.parametrize("kw,expect", SHARED + [
    (dict(y=A), INVALID),
    (dict(y=B + 16), INVALID),
    (dict(y=D), INVALID),
    (dict(lse=A), INVALID),
    (dict(lse=F + 16), INVALID),
    (dict(tokens=0), OK),
])
def test_attention_arguments(kw, expect):
    kw = {k: v for k, v in kw.items() if k in ATTENTION}
    assert Q.quasar_attention(**(ATTENTION | kw)) == expect


@pytest.mark.parametrize("kw,expect", SHARED + [
    (dict(dy=None), INVALID),
    (dict(lse=None), INVALID),
    (dict(dk=None), INVALID),
    (dict(dv=None), INVALID),
    (dict(dq=H + 8), INVALID),
    (dict(ld_dk=120), INVALID),
    (dict(dk=9 * A, dv=9 * A + 128), INVALID),
    (dict(dq=A), INVALID),
    (dict(dq=F), INVALID),
    (dict(dk=B), INVALID),
    (dict(workspace=None), INVALID),
    (dict(workspace=11 * A + 8), INVALID),
    (dict(workspace=H), INVALID),
    (dict(workspace_bytes=319), INVALID),
    (dict(dq=None, dk=None, dv=None), OK),
    (dict(tokens=0, keys=0), OK),
])
def test_attention_backward_arguments(kw, expect):
    args = ATTENTION | dict(dy=12 * A, ld_dy=256, dq=H, ld_dq=256, dk=9 * A, ld_dk=128, dv=10 * A, ld_dv=128,
                            workspace=11 * A, workspace_bytes=1 << 20)
    if kw.get("workspace_bytes"):
        kw = kw | {}
    assert Q.quasar_attention_backward(**(args | kw)) == expect


def test_columns_of_one_buffer_are_no_overlap():
    """dq, dk and dv as columns of one buffer pass the checks (no rows: nothing is launched)."""
    args = ATTENTION | dict(dy=12 * A, ld_dy=256, dq=H, ld_dq=512, dk=H + 512, ld_dk=512, dv=H + 768, ld_dv=512,
                            workspace=11 * A, workspace_bytes=1 << 20, tokens=0, keys=0)
    assert Q.quasar_attention_backward(**args) == OK


# -- what the convenience layer refuses ----------------------------------------------

def tensors():
    n, w, v, d = 6, 32, 20, 16
    return {
        "embedding": (lambda t: api.embedding(t["ids"], t["table"], residual=t["residual"]),
                      {"ids": ((n,), I32), "table": ((v, w), BF16), "residual": ((n, w), BF16)}),
        "embedding_backward": (lambda t: api.embedding_backward(t["dy"], t["ids"], v, into=t["into"]),
                               {"dy": ((n, w), BF16), "ids": ((n,), I32), "into": ((v, w), F32)}),
        "layer_norm": (lambda t: api.layer_norm(t["x"], t["weight"], bias=t["bias"]),
                       {"x": ((n, w), BF16), "weight": ((w,), F32), "bias": ((w,), F32)}),
        "layer_norm_backward": (lambda t: api.layer_norm_backward(t["dy"], t["x"], t["weight"], t["stats"],
                                                                  residual=t["residual"]),
                                {"dy": ((n, w), BF16), "x": ((n, w), BF16), "weight": ((w,), F32),
                                 "stats": ((n, 2), F32), "residual": ((n, w), BF16)}),
        "attention": (lambda t: api.attention(t["q"], t["k"], t["v"], d, starts=t["starts"],
                                              key_starts=t["key_starts"]),
                      {"q": ((n, 64), BF16), "k": ((9, w), BF16), "v": ((9, w), BF16), "starts": ((3,), I32),
                       "key_starts": ((3,), I32)}),
        "attention_backward": (lambda t: api.attention_backward(t["dy"], t["q"], t["k"], t["v"], t["y"], t["lse"], d,
                                                                starts=t["starts"], key_starts=t["key_starts"],
                                                                out=(t["dq"], t["dk"], t["dv"])),
                               {"q": ((n, 64), BF16), "k": ((9, w), BF16), "v": ((9, w), BF16), "starts": ((3,), I32),
                                "key_starts": ((3,), I32), "dy": ((n, 64), BF16), "y": ((n, 64), BF16),
                                "lse": ((n, 4), F32), "dq": ((n, 64), BF16), "dk": ((9, w), BF16),
                                "dv": ((9, w), BF16)}),
    }


def described(of, **changed):
    return {k: changed.get(k) or Described(*shape, dtype=dtype) for k, (shape, dtype) in of.items()}


@pytest.mark.parametrize("name", list(tensors()))
def test_tensors_elsewhere(name, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(api, "_alone", False)
    call, of = tensors()[name]
    for odd in list(of)[1:]:
        made = described(of, **{odd: Described(*of[odd][0], dtype=of[odd][1], at=1)})
        with pytest.raises(ValueError, match=f"{odd} must be on cuda:0.*not on cuda:1"):
            call(made)
    made = {k: Described(*shape, dtype=dtype, at=1) for k, (shape, dtype) in of.items()}
    with pytest.raises(ValueError, match="on cuda:1, but the current device is cuda:0"):
        call(made)


@pytest.mark.parametrize("name", list(tensors()))
def test_shapes_and_types(name):
    call, of = tensors()[name]
    for odd, (shape, dtype) in of.items():
        with pytest.raises(ValueError, match=odd):
            call(described(of, **{odd: Described(*shape, dtype=torch.float16)}))
        with pytest.raises(ValueError, match=odd):
            call(described(of, **{odd: Described(*shape, 1, dtype=dtype)}))
        if odd not in ("ids", "dy", "x", "q", "table", "k", "starts"):  # those set the others' shapes
            with pytest.raises(ValueError, match=odd):
                call(described(of, **{odd: Described(shape[0] + 1, *shape[1:], dtype=dtype)}))


def test_other_refusals():
    call, of = tensors()["attention"]
    made = described(of)
    with pytest.raises(ValueError, match="key_starts is needed"):
        api.attention(made["q"], made["k"], made["v"], 16, starts=made["starts"])
    with pytest.raises(ValueError, match="goes with starts"):
        api.attention(made["q"], made["k"], made["v"], 16, key_starts=made["starts"])
    with pytest.raises(ValueError, match="whole heads"):
        api.attention(made["q"], made["k"], made["v"], 24)
    with pytest.raises(ValueError, match="cannot share"):
        api.attention(Described(6, 48), made["k"], made["v"], 16)
    with pytest.raises(ValueError, match="ids 6"):
        api.embedding_backward(Described(7, 32), Described(6, dtype=I32), 20)
    with pytest.raises(ValueError, match="dx=True"):
        api.layer_norm_backward(*(Described(6, 32),) * 2, None, Described(6, 2, dtype=F32), dx=False,
                                residual=Described(6, 32))
