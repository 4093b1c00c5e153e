"""The norm's dweight and dbias are [cols] fp32 wherever a float may lie: slices of one flat buffer of
gradients, at each of the four places within 16 bytes (GPU)."""
import pytest
import torch

from paper_2608_13966_gb300 import api
from paper_2608_13966_gb300 import quasar as Q

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
CODES = {BF16: Q.BF16, F32: Q.F32}


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("cols", [128, 1024, 1032, 2048, 4096, 4099, 8192, 16384, 16392])
@pytest.mark.parametrize("rows", [1, 2, 33])
def test_sums_at_any_float(rows, cols, dtype):
    """The same bits as in tensors of their own, and the floats around them stay."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + cols)
    x, dy = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(2))
    w = torch.randn(cols, generator=g, device="cuda")
    stats = api.layer_norm(x, w, stats=True)["stats"]
    want = api.layer_norm_backward(dy, x, w, stats, dbias=True)
    if rows == 1:  # the sum of one row is dy itself
        assert torch.equal(want["dbias"], dy[0].float())
    need = Q.quasar_layer_norm_backward_workspace(rows, cols)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    for first, second in ((1, 0), (0, 1), (2, 3), (3, 2)):
        flat = torch.full((2 * cols + 24,), 99.0, device="cuda")
        dw = flat[4 + first:4 + first + cols]
        at = -(-(12 + first + cols) // 4) * 4 + second
        db = flat[at:at + cols]
        dx = torch.empty(rows, cols, dtype=BF16, device="cuda")
        assert dw.data_ptr() % 16 == 4 * first and db.data_ptr() % 16 == 4 * second
        st = Q.quasar_layer_norm_backward(dy, CODES[dtype], cols, x, CODES[dtype], cols, w, stats, rows, cols, 1, None, 0,
                                          dx, Q.BF16, cols, dw, db, ws, need)
        assert st == Q.QuasarStatus.OK
        api.check_device()
        assert torch.equal(dx, want["dx"]) and torch.equal(dw, want["dweight"]) and torch.equal(db, want["dbias"])
        dw[:] = 99.0
        db[:] = 99.0
        assert (flat == 99).all()
