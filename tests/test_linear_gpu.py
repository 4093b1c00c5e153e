"""The matrix products against fp64 (GPU).

Tolerance, per element: a product of two bf16 values is exact in fp32, and a
sum of n of them kept in fp32 is off by at most n 2^-24 sum |a b| (one
rounding or truncation of at most an ulp a term), to which the epilogue adds
a few ulps of what it adds.  Activations have slopes of at most 1.13; their
own fp32 evaluation is good to a few ulps of their operands.  An output in
bf16 must be the bf16 rounding of some value within that distance of the
exact one."""

import pytest
import torch

from paper_2608_13966_gb300 import api
from paper_2608_13966_gb300 import quasar as Q
from tests.bands import outside

pytestmark = pytest.mark.gpu

ACT = {
    "none": lambda z: z,
    "relu": lambda z: z.clamp(min=0.0),
    "silu": lambda z: z * torch.special.expit(z),
    "gelu": lambda z: z * torch.special.ndtr(z),
}


def slope(z, name):
    z = z.clone().requires_grad_(True)
    ACT[name](z).sum().backward()
    return torch.where(z == 0, 0.0, z.grad) if name == "relu" else z.grad


def rand(*shape, scale=1.0, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def strided(t, ld):
    """t's values in rows ld apart."""
    wide = torch.full((t.shape[0], ld), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def close(got, want, mag, terms, bf16):
    assert got.dtype == (torch.bfloat16 if bf16 else torch.float32)
    tol = 1.2 * (terms + 32) * 2.0 ** -24 * mag + 1e-30
    bad = outside(got, want, tol)
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() / tol).max()))


SHAPES = [(1, 128, 64), (1, 1, 8), (2, 1003, 8), (3, 64, 4096), (16, 128, 64), (17, 130, 72),
          (31, 257, 520), (64, 100, 1032), (100, 1024, 264), (129, 129, 136), (257, 515, 648),
          (300, 512, 2048)]


@pytest.mark.parametrize("tokens,features,inputs", SHAPES)
@pytest.mark.parametrize("activation,bias,residual,out,pre", [
    ("none", False, False, torch.float32, False),
    ("none", True, True, torch.bfloat16, False),
    ("relu", False, True, torch.bfloat16, True),
    ("silu", True, False, torch.float32, True),
    ("gelu", True, True, torch.float32, False),
])
def test_linear(tokens, features, inputs, activation, bias, residual, out, pre):
    x, r = rand(tokens, inputs, seed=1), rand(features, inputs, scale=0.05, seed=2)
    b = rand(features, seed=3, dtype=torch.float32) if bias else None
    res = rand(tokens, features, seed=4, dtype=out) if residual else None
    made = api.linear(x, r, bias=b, activation=activation, residual=res, out_dtype=out,
                      save_pre=pre)
    z = x.double() @ r.double().t()
    mag = x.double().abs() @ r.double().abs().t()
    if bias:
        z, mag = z + b.double(), mag + b.double().abs()
    y = ACT[activation](z)
    if residual:
        y = y + res.double()
        mag = mag + res.double().abs()
    api.check_device()
    close(made["y"], y, mag, inputs, out == torch.bfloat16)
    if pre:
        close(made["pre"], z, mag, inputs, True)
        assert made["pre"].stride(0) % 8 == 0 or tokens == 1


@pytest.mark.parametrize("tokens,features,inputs", SHAPES)
@pytest.mark.parametrize("activation,residual,dx_type,dr_type", [
    ("none", False, torch.bfloat16, torch.float32),
    ("silu", True, torch.float32, torch.bfloat16),
    ("gelu", False, torch.float32, torch.float32),
    ("relu", True, torch.bfloat16, torch.float32),
])
def test_linear_backward(tokens, features, inputs, activation, residual, dx_type, dr_type):
    dz, x = rand(tokens, features, seed=5), rand(tokens, inputs, seed=6)
    r = rand(features, inputs, scale=0.05, seed=7)
    pre = rand(tokens, inputs, seed=8) if activation != "none" else None
    res = rand(tokens, inputs, seed=9, dtype=dx_type) if residual else None
    made = api.linear_backward(dz, x, r, bias=True, pre_in=pre, activation_in=activation,
                               residual=res, dx_dtype=dx_type, dr_dtype=dr_type)
    dx = dz.double() @ r.double()
    mag = dz.double().abs() @ r.double().abs()
    if pre is not None:
        dx = dx * slope(pre.double(), activation)
        mag = mag * 1.2
    if residual:
        dx, mag = dx + res.double(), mag + res.double().abs()
    api.check_device()
    close(made["dx"], dx, mag, features, dx_type == torch.bfloat16)
    close(made["dr"], dz.double().t() @ x.double(), dz.double().abs().t() @ x.double().abs(),
          tokens, dr_type == torch.bfloat16)
    close(made["dbias"], dz.double().sum(0), dz.double().abs().sum(0), tokens, False)


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,features,inputs", [(2311, 2497, 72), (2500, 2304, 1032), (4097, 2200, 8)])
def test_linear_of_many_tiles(tokens, features, inputs, out):
    """Enough 256 x 256 tiles for every pair of SMs, with ragged edges."""
    x, r = rand(tokens, inputs, seed=1), rand(features, inputs, scale=0.05, seed=2)
    b, res = rand(features, seed=3, dtype=torch.float32), rand(tokens, features, seed=4, dtype=out)
    made = api.linear(x, r, bias=b, activation="gelu", residual=res, out_dtype=out, save_pre=True)
    z = x.double() @ r.double().t() + b.double()
    mag = x.double().abs() @ r.double().abs().t() + b.double().abs()
    api.check_device()
    close(made["pre"], z, mag, inputs, True)
    close(made["y"], ACT["gelu"](z) + res.double(), mag + res.double().abs(), inputs,
          out == torch.bfloat16)


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,features,inputs", [(2311, 2497, 2312), (2305, 2560, 4104)])
def test_linear_backward_of_many_tiles(tokens, features, inputs, out):
    dz, x = rand(tokens, features, seed=5), rand(tokens, inputs, seed=6)
    r = rand(features, inputs, scale=0.05, seed=7)
    pre, res = rand(tokens, inputs, seed=8), rand(tokens, inputs, seed=9, dtype=out)
    made = api.linear_backward(dz, x, r, bias=True, pre_in=pre, activation_in="silu", residual=res,
                               dx_dtype=out, dr_dtype=out)
    api.check_device()
    dx = dz.double() @ r.double() * slope(pre.double(), "silu") + res.double()
    mag = 1.2 * (dz.double().abs() @ r.double().abs()) + res.double().abs()
    close(made["dx"], dx, mag, features, out == torch.bfloat16)
    close(made["dr"], dz.double().t() @ x.double(), dz.double().abs().t() @ x.double().abs(),
          tokens, out == torch.bfloat16)
    close(made["dbias"], dz.double().sum(0), dz.double().abs().sum(0), tokens, False)


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,features,inputs", [
    (4999, 200, 1976), (2299, 333, 1600), (2500, 130, 2376), (2300, 141, 2688), (2300, 130, 2632), (60, 3001, 1352)])
def test_linear_of_tiles_several_ctas_share(tokens, features, inputs, out):
    """2 to 8 CTAs a tile, by what the device holds at once."""
    x, r = rand(tokens, inputs, seed=32), rand(features, inputs, scale=0.05, seed=33)
    b = rand(features, seed=34, dtype=torch.float32)
    made = api.linear(x, r, bias=b, out_dtype=out)
    api.check_device()
    close(made["y"], x.double() @ r.double().t() + b.double(),
          x.double().abs() @ r.double().abs().t() + b.double().abs(), inputs, out == torch.bfloat16)


def test_a_large_product_whose_wait_runs_out_is_reported():
    x, r = rand(2311, 72, seed=1), rand(2497, 72, seed=2)
    want = api.linear(x, r, out_dtype=torch.float32)["y"]
    api.check_device()
    Q.quasar_debug_force_timeout(1_000_000)
    try:
        api.linear(x, r, out_dtype=torch.float32)
        assert Q.quasar_get_device_status() == Q.QuasarStatus.ERR_TIMEOUT
    finally:
        Q.quasar_debug_force_timeout(0)
    assert torch.equal(api.linear(x, r, out_dtype=torch.float32)["y"], want)
    api.check_device()


@pytest.mark.parametrize("tokens,features,inputs", [(5, 77, 200), (90, 300, 1032), (513, 640, 128)])
def test_strides_and_guards(tokens, features, inputs):
    """Strided operands and results; nothing outside the results is written,
    nothing outside the operands (NaN there) is used."""
    x = strided(rand(tokens, inputs, seed=1), inputs + 24)
    r = strided(rand(features, inputs, scale=0.05, seed=2), inputs + 8)
    res = strided(rand(tokens, features, seed=3, dtype=torch.float32), features + 5)
    ld, off = features + 3, 7
    for y_dtype, code in ((torch.float32, Q.F32), (torch.bfloat16, Q.BF16)):
        y = torch.full(((tokens + 1) * ld + off,), 12345.0, dtype=y_dtype, device="cuda")
        pre = torch.full(((tokens + 1) * ld + off,), 12345.0, dtype=torch.bfloat16, device="cuda")
        rr = res.to(y_dtype)
        rr = strided(rr, features + 5)
        at = y.data_ptr() + off * y.element_size()
        st = Q.quasar_linear(x, inputs + 24, r, inputs + 8, None, "silu", rr, features + 5, tokens,
                             features, inputs, at, code, ld, pre.data_ptr() + 2 * off, ld)
        assert st == Q.QuasarStatus.OK
        z = x.double() @ r.double().t()
        mag = x.double().abs() @ r.double().abs().t() + rr.double().abs()
        view = y[off:off + tokens * ld].view(tokens, ld)
        close(view[:, :features], ACT["silu"](z) + rr.double(), mag, inputs, code == Q.BF16)
        pv = pre[off:off + tokens * ld].view(tokens, ld)
        close(pv[:, :features], z, mag, inputs, True)
        for whole, v in ((y, view), (pre, pv)):
            assert (whole[:off] == 12345.0).all() and (v[:, features:] == 12345.0).all()
            assert (whole[off + tokens * ld:] == 12345.0).all()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 7, 8, 9])
@pytest.mark.parametrize("features,inputs,ld", [(33, 13, 13), (70, 2061, 2064), (31, 4104, 4107), (100, 2048, 2048)])
def test_weight_gradient_of_a_few_tokens(tokens, features, inputs, ld, out):
    """Also with inputs that end inside a vector and rows of dr that start
    anywhere; nothing outside dr is written."""
    dz = strided(rand(tokens, features, seed=1), features // 8 * 8 + 8)
    x = strided(rand(tokens, inputs, seed=2), inputs // 8 * 8 + 16)
    flat = torch.full((features * ld + 40,), 12345.0, dtype=out, device="cuda")
    off = 3 if ld % 8 else 0
    dbias = torch.full((features + 8,), 12345.0, device="cuda")
    st = Q.quasar_linear_grad_weight(dz, dz.stride(0), x, x.stride(0), tokens, features, inputs,
                                     flat.data_ptr() + off * flat.element_size(),
                                     Q.F32 if out == torch.float32 else Q.BF16, ld, dbias)
    assert st == Q.QuasarStatus.OK
    api.check_device()
    dr = flat[off:off + features * ld].view(features, ld)
    close(dr[:, :inputs], dz.double().t() @ x.double(), dz.double().abs().t() @ x.double().abs(),
          tokens, out == torch.bfloat16)
    close(dbias[:features], dz.double().sum(0), dz.double().abs().sum(0), tokens, False)
    assert (dr[:, inputs:] == 12345.0).all() and (flat[:off] == 12345.0).all()
    assert (flat[off + features * ld:] == 12345.0).all() and (dbias[features:] == 12345.0).all()


def test_results_in_place_of_what_they_add():
    tokens, features, inputs = 70, 200, 136
    x, r = rand(tokens, inputs, seed=1), rand(features, inputs, scale=0.05, seed=2)
    y = rand(tokens, features, seed=3)
    want = (x.double() @ r.double().t() + y.double())
    mag = x.double().abs() @ r.double().abs().t() + y.double().abs()
    st = Q.quasar_linear(x, inputs, r, inputs, None, "none", y, features, tokens, features, inputs, y,
                         Q.BF16, features)
    assert st == Q.QuasarStatus.OK
    close(y, want, mag, inputs, True)
    dz, pre = rand(tokens, features, seed=5), rand(tokens, inputs, seed=6)
    want = dz.double() @ r.double() * slope(pre.double(), "gelu")
    mag = 1.2 * (dz.double().abs() @ r.double().abs())
    st = Q.quasar_linear_grad_input(dz, features, r, inputs, pre, inputs, "gelu", None, 0, tokens,
                                    features, inputs, pre, Q.BF16, inputs)
    assert st == Q.QuasarStatus.OK
    close(pre, want, mag, features, True)


@pytest.mark.parametrize("activation", ["none", "relu", "silu", "gelu"])
def test_activation_grad(activation):
    dy, pre = strided(rand(37, 301, seed=1), 305), strided(rand(37, 301, scale=3.0, seed=2), 303)
    dz = api.activation_grad(dy, pre, activation)
    want = dy.double() * slope(pre.double(), activation)
    close(dz, want, dy.double().abs(), 4, True)
    assert dz.stride(0) % 8 == 0
    # an extreme pre-activation has slope 0 or 1, not NaN
    far = torch.tensor([[-1e30, -200.0, 200.0, 1e30, float("inf"), 0.0]], dtype=torch.bfloat16,
                       device="cuda")
    got = api.activation_grad(torch.ones_like(far), far, activation)[0, :5].float()
    if activation == "none":
        assert (got == 1.0).all()
    else:
        assert got[:4].tolist() == [0.0, 0.0, 1.0, 1.0]


def test_empty_reductions():
    r = torch.empty(24, 0, dtype=torch.bfloat16, device="cuda")
    x = torch.empty(5, 0, dtype=torch.bfloat16, device="cuda")
    b = rand(24, seed=1, dtype=torch.float32)
    y = torch.empty(5, 24, dtype=torch.float32, device="cuda")
    st = Q.quasar_linear(x, 0, r, 0, b, "relu", None, 0, 5, 24, 0, y, Q.F32, 24)
    assert st == Q.QuasarStatus.OK
    assert torch.equal(y, b.clamp(min=0).expand(5, 24))
    dz = torch.empty(0, 24, dtype=torch.bfloat16, device="cuda")
    made = api.linear_backward(dz, torch.empty(0, 16, dtype=torch.bfloat16, device="cuda"),
                               rand(24, 16), bias=True, dr_dtype=torch.float32)
    assert made["dx"].shape == (0, 16)
    assert not made["dr"].any() and not made["dbias"].any()


def test_the_same_bits_every_time():
    dz, x = rand(600, 264, seed=1), rand(600, 1032, seed=2)
    r = rand(264, 1032, scale=0.05, seed=3)
    first = api.linear_backward(dz, x, r, bias=True, dx_dtype=torch.float32, dr_dtype=torch.float32)
    y = api.linear(x, r, out_dtype=torch.float32)["y"]
    for _ in range(5):
        again = api.linear_backward(dz, x, r, bias=True, dx_dtype=torch.float32,
                                    dr_dtype=torch.float32)
        for name in first:
            assert torch.equal(first[name], again[name]), name
        assert torch.equal(y, api.linear(x, r, out_dtype=torch.float32)["y"])


def test_gradients_are_those_of_the_forward():
    """dx, dr and dbias against central differences of the fp64 loss at the
    same point (the gradient of a linear form is exact in its differences up
    to rounding, h^2 terms coming from the activation alone)."""
    tokens, features, inputs = 6, 40, 24
    x, r = rand(tokens, inputs, seed=1), rand(features, inputs, scale=0.2, seed=2)
    b = rand(features, seed=3, dtype=torch.float32)
    up = rand(tokens, features, seed=4)

    def loss(x_, r_, b_):
        return (ACT["silu"](x_ @ r_.t() + b_) * up.double()).sum()

    made = api.linear(x, r, bias=b, activation="silu", save_pre=True, out_dtype=torch.float32)
    dz = api.activation_grad(up, made["pre"], "silu")
    grads = api.linear_backward(dz, x, r, bias=True, dx_dtype=torch.float32, dr_dtype=torch.float32)
    at = [x.double(), r.double(), b.double()]
    h = 1e-4
    # dz carries two bf16 roundings (z kept in bf16, dz itself): 2^-8 and 2^-9
    # of the magnitudes summed
    size = up.double().abs() * (1.0 + (x.double().abs() @ r.double().abs().t() + b.double().abs()))
    mags = [size @ r.double().abs(), size.t() @ x.double().abs(), size.sum(0)]
    for which, name in enumerate(("dx", "dr", "dbias")):
        got = grads[name].double().flatten()
        for j in range(0, got.numel(), max(1, got.numel() // 12)):
            step = torch.zeros_like(at[which]).flatten()
            step[j] = h
            hi, lo = list(at), list(at)
            hi[which] = at[which] + step.view_as(at[which])
            lo[which] = at[which] - step.view_as(at[which])
            want = float((loss(*hi) - loss(*lo)) / (2 * h))
            assert abs(float(got[j]) - want) <= 2.0 ** -7 * float(mags[which].flatten()[j]) + 1e-6


@pytest.mark.parametrize("tokens,features,inputs", [(1, 70, 72), (5, 70, 72), (300, 260, 136)])
def test_offsets_past_32_bits(tokens, features, inputs):
    """Rows so far apart that element offsets pass 2^32 (operands, results and
    what is added)."""
    apart = (1 << 32) // max(tokens - 1, 1) // 8 * 8 + 8
    wide = torch.empty((tokens - 1) * apart + 1024, dtype=torch.bfloat16, device="cuda")
    wide2 = torch.empty((tokens - 1) * apart + 1024, dtype=torch.bfloat16, device="cuda")
    x = wide.as_strided((tokens, inputs), (apart, 1))
    y = wide2.as_strided((tokens, features), (apart, 1))
    x.copy_(rand(tokens, inputs, seed=1))
    y.copy_(rand(tokens, features, seed=2))
    r = rand(features, inputs, scale=0.05, seed=3)
    want = x.double() @ r.double().t() + y.double()
    mag = x.double().abs() @ r.double().abs().t() + y.double().abs()
    st = Q.quasar_linear(x, apart, r, inputs, None, "none", y, apart, tokens, features, inputs, y, Q.BF16,
                         apart)
    assert st == Q.QuasarStatus.OK
    api.check_device()
    close(y, want, mag, inputs, True)
    if tokens > 1:  # y is dz now
        made = api.linear_backward(y, x, r, bias=True, dr_dtype=torch.float32)
        close(made["dr"], y.double().t() @ x.double(), y.double().abs().t() @ x.double().abs(), tokens,
              False)
        close(made["dbias"], y.double().sum(0), y.double().abs().sum(0), tokens, False)


def test_two_streams_at_once():
    """Products of different kinds side by side, many of them, and the same
    bits as alone."""
    cases = [(1, 1000, 520), (40, 700, 2056), (200, 333, 1032), (2600, 2600, 136)]
    data = [(rand(t, i, seed=n), rand(f, i, scale=0.05, seed=n + 9)) for n, (t, f, i) in enumerate(cases)]
    alone = [api.linear(x, r, out_dtype=torch.float32)["y"] for x, r in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    made = []
    for turn in range(12):
        for n, (x, r) in enumerate(data):
            made.append((n, api.linear(x, r, out_dtype=torch.float32, stream=streams[(turn + n) % 3])["y"]))
    torch.cuda.synchronize()
    api.check_device()
    for n, y in made:
        assert torch.equal(y, alone[n])


def test_in_a_graph():
    x, r = rand(70, 264, seed=1), rand(200, 264, scale=0.05, seed=2)
    api.linear(x, r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = api.linear(x, r, activation="silu", save_pre=True)
        dz = api.activation_grad(y["y"], y["pre"], "silu")
        made = api.linear_backward(dz, x, r, bias=True)
    for seed in (3, 4):
        x.copy_(rand(70, 264, seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        again = api.linear(x, r, activation="silu", save_pre=True)
        assert torch.equal(again["y"], y["y"]) and torch.equal(again["pre"], y["pre"])
        back = api.linear_backward(api.activation_grad(again["y"], again["pre"], "silu"), x, r, bias=True)
        for name in back:
            assert torch.equal(back[name], made[name]), name


def test_another_stream():
    side = torch.cuda.Stream()
    x, r = rand(40, 264, seed=1), rand(72, 264, seed=2)
    side.wait_stream(torch.cuda.current_stream())
    y = api.linear(x, r, out_dtype=torch.float32, stream=side)["y"]
    z = api.linear(x, r, out_dtype=torch.float32)["y"]
    side.synchronize()
    assert torch.equal(y, z)


def test_a_wait_that_runs_out_is_reported():
    x, r = rand(200, 264, seed=1), rand(300, 264, seed=2)
    want = api.linear(x, r, out_dtype=torch.float32)["y"]
    api.check_device()
    Q.quasar_debug_force_timeout(1_000_000)
    try:
        api.linear(x, r, out_dtype=torch.float32)
        assert Q.quasar_get_device_status() == Q.QuasarStatus.ERR_TIMEOUT
    finally:
        Q.quasar_debug_force_timeout(0)
    assert torch.equal(api.linear(x, r, out_dtype=torch.float32)["y"], want)
    api.check_device()
