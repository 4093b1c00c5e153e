"""Layer norm and its gradients against fp64.

Tolerances: an output of fewer bits is off by half a step of its value (bf16
2^-8), an fp32 sum of n terms by at most n 2^-24 of the sum of their sizes, and
x - mean by 2^-24 of |x| + |mean| and by the error of the mean."""
import pytest
import torch

from paper_2608_13966_gb300 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: U}
COLS = [1, 2, 7, 8, 63, 64, 65, 128, 250, 257, 512, 1000, 1003, 1025, 2048, 2051, 4096, 4099, 5000, 8192, 12288,
        16384, 16385, 20001]


def made(rows, cols, dtype, seed=0, ld=None, offset=0.0, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed + 7 * rows + cols)
    x = torch.randn(rows, cols, generator=g, device=device) + offset
    if ld is None:
        return x.to(dtype)
    wide = torch.full((rows, ld), 7.0, dtype=dtype, device=device)
    wide[:, :cols] = x
    return wide[:, :cols]


def check(got, want, tol, what):
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), (what, off[bad].max().item(), tol.expand_as(off)[bad].min().item(), int(bad.sum()))


def forward_bounds(x, w, b, center, eps):
    """Exact y and stats, and how far each may be off before y is rounded."""
    n = x.shape[1]
    x = x.double()
    mean = x.mean(1, keepdim=True) if center else torch.zeros_like(x[:, :1])
    d = x - mean
    rstd = (d.square().mean(1, keepdim=True) + eps).rsqrt()
    e_mean = (n + 4) * U * x.abs().mean(1, keepdim=True) * (1.0 if center else 0.0)
    e_d = 2 * U * (x.abs() + mean.abs()) + e_mean
    # of the mean square: from d, and from summing
    e_rel = (2 * d.abs() * e_d + e_d.square()).mean(1, keepdim=True) * rstd.square() + (n + 8) * U
    xh = d * rstd
    y = xh * w + b
    e_y = (e_d * rstd + xh.abs() * (0.5 * e_rel + 4 * U)) * w.abs() * (1 + 1e-3) + 2 * U * ((xh * w).abs() + b.abs())
    return y, mean, rstd, e_y, e_mean + 2 * U * mean.abs(), rstd * (0.5 * e_rel + 4 * U) * (1 + 1e-3)


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", COLS)
def test_forward(cols, dtype, center):
    for rows, ld in ((1, None), (37, None), (5, cols + 3), (700 if cols < 3000 else 311, -(-cols // 8) * 8)):
        x = made(rows, cols, dtype, ld=ld, offset=0.5)
        w, b = (made(1, cols, F32, seed=s)[0].contiguous() for s in (1, 2))
        for weight, bias, out in ((w, b, BF16), (None, None, F32), (w, None, F32)):
            o = api.layer_norm(x, weight, bias=bias, center=center, out_dtype=out, stats=True)
            ones = torch.ones(cols, dtype=torch.float64, device="cuda")
            y, mean, rstd, e_y, e_mean, e_rstd = forward_bounds(
                x, ones if weight is None else w.double(), 0 * ones if bias is None else b.double(), center, 1e-5)
            check(o["y"], y, e_y + HALF[out] * (y.abs() + e_y), (rows, cols, ld, "y"))
            check(o["stats"][:, :1], mean, e_mean, (rows, cols, "mean"))
            check(o["stats"][:, 1:], rstd, e_rstd, (rows, cols, "rstd"))


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("x_dtype,dy_dtype,dx_dtype", [(BF16, BF16, BF16), (F32, BF16, F32), (BF16, F32, BF16),
                                                       (F32, F32, BF16)])
@pytest.mark.parametrize("cols", COLS)
def test_backward(cols, x_dtype, dy_dtype, dx_dtype, center):
    for rows, ld in ((1, None), (37, cols + 3), (700 if cols < 3000 else 311, -(-cols // 8) * 8)):
        x = made(rows, cols, x_dtype, ld=ld, offset=0.5)
        dy = made(rows, cols, dy_dtype, seed=3, ld=ld)
        res = made(rows, cols, dx_dtype, seed=4, ld=ld)
        w = made(1, cols, F32, seed=1)[0].contiguous()
        stats = api.layer_norm(x, w, center=center, stats=True)["stats"]
        for residual, weight in ((res, w), (None, None)):
            o = api.layer_norm_backward(dy, x, weight, stats, center=center, dbias=True, residual=residual,
                                        dx_dtype=dx_dtype)
            again = api.layer_norm_backward(dy, x, weight, stats, center=center, dbias=True, residual=residual,
                                            dx_dtype=dx_dtype)
            assert all(torch.equal(o[k], again[k]) for k in o)
            mean, rstd = stats.double().split(1, 1)
            xd, dyd = x.double(), dy.double()
            xh, big = (xd - mean) * rstd, (xd.abs() + mean.abs()) * rstd
            u = dyd * (1.0 if weight is None else w.double())
            mu, mux = u.mean(1, keepdim=True) * float(center), (u * xh).mean(1, keepdim=True)
            r = 0.0 if residual is None else res.double()
            dx = rstd * (u - mu - xh * mux) + r
            n = cols + 16
            size = rstd * (u.abs() + u.abs().mean(1, keepdim=True) + big * (u.abs() * big).mean(1, keepdim=True))
            e = n * U * size + 2 * U * dx.abs()
            check(o["dx"], dx, e + HALF[dx_dtype] * (dx.abs() + e), (rows, cols, ld, "dx"))
            check(o["dweight"], (dyd * xh).sum(0), (rows + 16) * U * (dyd.abs() * big).sum(0), (rows, cols, "dw"))
            check(o["dbias"], dyd.sum(0), (rows + 16) * U * dyd.abs().sum(0), (rows, cols, "db"))


def test_gradient_against_differences():
    x = made(3, 50, F32).double()
    w, b, dy = (made(k, 50, F32, seed=s) for k, s in ((1, 1), (1, 2), (3, 3)))
    w, b = w[0].contiguous(), b[0].contiguous()
    for center in (True, False):
        def loss(x, w, b):
            x = x.double()
            d = x - x.mean(1, keepdim=True) if center else x
            return (d * (d.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w.double() + b.double()).mul(dy.double()).sum()
        stats = api.layer_norm(x.float(), w, bias=b, center=center, stats=True)["stats"]
        o = api.layer_norm_backward(dy, x.float(), w, stats, center=center, dbias=True, dx_dtype=F32)
        h = 1e-5
        for (i, j) in ((0, 0), (1, 17), (2, 49)):
            e = torch.zeros_like(x)
            e[i, j] = h
            slope = (loss(x + e, w, b) - loss(x - e, w, b)) / (2 * h)
            # h^2 of the third derivative, 64-bit rounding over h, fp32 of the kernel
            assert abs(float(slope - o["dx"][i, j])) < 1e-5 * (1 + abs(float(slope)))
            e = torch.zeros(50, dtype=torch.float64, device="cuda")
            e[j] = h
            for name, at in (("dweight", (w + e, b)), ("dbias", (w, b + e))):
                slope = (loss(x, *at) - loss(x, w, b)) / h
                assert abs(float(slope - o[name][j])) < 1e-5 * (1 + abs(float(slope)))


def test_rows_far_from_zero():
    """A mean 1000 times the deviation: the variance is summed about it."""
    x = made(64, 4096, F32, offset=1000.0)
    o = api.layer_norm(x, center=True, stats=True, out_dtype=F32)
    y, mean, rstd, e_y, e_mean, e_rstd = forward_bounds(x, torch.ones(4096, device="cuda").double(),
                                                        torch.zeros(4096, device="cuda").double(), True, 1e-5)
    check(o["y"], y, e_y + U * y.abs(), "y")
    assert ((o["stats"][:, 1:].double() - rstd).abs() / rstd).max() < 1e-3


def test_special_rows():
    x = made(6, 1000, BF16)
    x[1] = 3.0       # no variance
    x[2, 5] = float("nan")
    x[4, 7] = float("inf")
    y = api.layer_norm(x)["y"].float()
    assert (y[1] == 0).all()
    assert y[2].isnan().all() and not y[4].isfinite().any() or y[4].isnan().any()
    for r in (0, 3, 5):
        assert y[r].isfinite().all()
    assert torch.equal(y[0], api.layer_norm(x[:1])["y"][0].float())


def test_empty():
    x = made(0, 64, BF16).reshape(0, 64)
    o = api.layer_norm(x, stats=True)
    assert o["y"].shape == (0, 64) and o["stats"].shape == (0, 2)
    g = api.layer_norm_backward(x, x, None, o["stats"], dbias=True)
    assert g["dx"].shape == (0, 64) and (g["dweight"] == 0).all() and (g["dbias"] == 0).all()


def test_parts_asked_for():
    x, dy = made(300, 700, BF16), made(300, 700, BF16, seed=3)
    stats = api.layer_norm(x, stats=True)["stats"]
    whole = api.layer_norm_backward(dy, x, None, stats, dbias=True)
    for kw in (dict(dx=False), dict(dweight=False), dict(dbias=False), dict(dx=False, dweight=False),
               dict(dweight=False, dbias=False)):
        o = api.layer_norm_backward(dy, x, None, stats, **(dict(dbias=True) | kw))
        for k in o:
            assert torch.equal(o[k], whole[k])
        assert set(o) == {k for k in ("dx", "dweight", "dbias") if kw.get(k, True)}


def test_streams_and_graphs():
    x, dy = made(500, 1003, BF16), made(500, 1003, BF16, seed=3)
    w = made(1, 1003, F32, seed=1)[0].contiguous()
    stats = api.layer_norm(x, w, stats=True)["stats"]
    want = api.layer_norm_backward(dy, x, w, stats, dbias=True)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    on = api.layer_norm_backward(dy, x, w, stats, dbias=True, stream=other)
    other.synchronize()
    assert all(torch.equal(on[k], want[k]) for k in want)
    graphs = []
    for _ in range(2):  # two graphs, each with a workspace of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s = api.layer_norm(x, w, stats=True)
            o = api.layer_norm_backward(dy, x, w, s["stats"], dbias=True)
        graphs.append((graph, o))
    x2 = made(500, 1003, BF16, seed=9)
    x.copy_(x2)
    want = api.layer_norm_backward(dy, x, w, api.layer_norm(x, w, stats=True)["stats"], dbias=True)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for (graph, _), s in zip(graphs, streams):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    for _, o in graphs:
        assert all(torch.equal(o[k], want[k]) for k in want)


def test_a_wait_that_runs_out_is_reported():
    from paper_2608_13966_gb300 import quasar as Q

    for rows in (3, 5000):
        x, dy = made(rows, 4096, BF16), made(rows, 4096, BF16, seed=3)
        want = api.layer_norm(x, stats=True)
        grads = api.layer_norm_backward(dy, x, None, want["stats"], dbias=True)
        api.check_device()
        for call in (lambda: api.layer_norm(x), lambda: api.layer_norm_backward(dy, x, None, want["stats"])):
            Q.quasar_debug_force_timeout(1_000_000)
            try:
                call()
                assert Q.quasar_get_device_status() == Q.QuasarStatus.ERR_TIMEOUT
            finally:
                Q.quasar_debug_force_timeout(0)
        assert torch.equal(api.layer_norm(x)["y"], want["y"])
        again = api.layer_norm_backward(dy, x, None, want["stats"], dbias=True)
        assert all(torch.equal(again[k], grads[k]) for k in grads)
        api.check_device()


@pytest.mark.parametrize("cols", [64, 1003, 2048, 8192, 16384, 20000])
def test_in_place(cols):
    """y in x's place; dx in dy's, x's or the residual's; guards around them stay."""
    from paper_2608_13966_gb300 import quasar as Q

    rows, ld = 700, cols + 8
    def wide(seed, dtype=BF16):
        t = torch.full((rows, ld), 99.0, dtype=dtype, device="cuda")
        t[:, :cols] = made(rows, cols, dtype, seed=seed)
        return t
    x = wide(0)
    o = api.layer_norm(x[:, :cols], stats=True)
    assert Q.quasar_layer_norm(x, Q.BF16, ld, None, None, rows, cols, 1, 1e-5, x, Q.BF16, ld) == Q.QuasarStatus.OK
    assert torch.equal(x[:, :cols], o["y"]) and (x[:, cols:] == 99).all()
    need = Q.quasar_layer_norm_backward_workspace(rows, cols)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    for place in range(3):
        x, dy, res = wide(0), wide(3), wide(4)
        want = api.layer_norm_backward(dy[:, :cols], x[:, :cols], None, o["stats"], dbias=True, residual=res[:, :cols])
        dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        dx = (dy, x, res)[place]
        assert Q.quasar_layer_norm_backward(dy, Q.BF16, ld, x, Q.BF16, ld, None, o["stats"], rows, cols, 1, res, ld, dx,
                                            Q.BF16, ld, dw, db, ws, need) == Q.QuasarStatus.OK
        assert torch.equal(dx[:, :cols], want["dx"]) and (dx[:, cols:] == 99).all()
        assert torch.equal(dw, want["dweight"]) and torch.equal(db, want["dbias"])
