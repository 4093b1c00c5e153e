"""Top logits and distillation against fp64 (GPU).

Tolerances.  With e = 2^-22 (2 + zmax), zmax the largest |logit / temperature|
or |log-sum-exp| of the row: forming z - lse costs at most a few roundings of
numbers of that size, so log p and log q are good to e, and p and q to a
relative e.  The derivative of p log(p/q) - p + q is p log(p/q) in log p and
q - p in log q, which gives the loss e (sum p |log p/q| + sum |p - q|) plus
rounding of its terms (2^-21 of their sum).  A listed entry's gradient P q - p
is off by e (q + p), an unlisted one's u (P q_r - p_r) by u e (q_r + p_r),
both times the row's weight over the temperature; a bf16 gradient must be the
bf16 rounding of a value within that distance.  A log-sum-exp adds at most V / 512 + 64 terms in a row: that
many 2^-24, plus e."""
import math

import pytest
import torch

from paper_2608_13966_gb300 import api
from paper_2608_13966_gb300 import quasar as Q
from tests.bands import outside

pytestmark = pytest.mark.gpu
INF = math.inf
BF16, F32 = torch.bfloat16, torch.float32


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def placed(t, ld, offset):
    """t's values in rows ld apart, the first `offset` elements into storage."""
    rows, cols = t.shape
    flat = torch.full((offset + rows * ld + 16,), float("nan"), dtype=t.dtype, device=t.device)
    view = flat[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(t)
    return view


def check_top(z, k, temperature=1.0):
    made = api.top_logits(z, k, temperature=temperature)
    api.check_device()
    v, i = torch.sort(z.float(), dim=1, descending=True, stable=True)
    assert torch.equal(made["values"], v[:, :k])
    assert torch.equal(made["indices"].long(), i[:, :k])
    want = torch.logsumexp(z.double() / temperature, 1)
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(made["lse"]), finite)
    scaled = z.double() / temperature
    zmax = scaled.abs().masked_fill(~torch.isfinite(scaled), 0.0).amax(1)
    e = 2.0 ** -22 * (2 + torch.maximum(zmax, want.abs()))
    tol = e + (z.shape[1] / 512 + 64) * 2.0 ** -24
    assert ((made["lse"].double() - want).abs() <= tol)[finite].all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,k", [
    (1, 1, 1), (3, 7, 7), (2, 100, 1), (5, 512, 256), (4, 513, 33), (3, 2049, 200), (300, 1000, 64),
    (2, 9001, 256), (7, 50001, 100), (1, 131072, 64), (2, 200003, 128),
])
def test_top_logits(rows, vocab, k, dtype):
    z = (torch.randn(rows, vocab, generator=gen(vocab), device="cuda") * 3.0).to(dtype)
    check_top(z, k)
    check_top(z, k, temperature=2.5)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset,ld", [(0, 5003), (1, 5003), (3, 5001), (5, 5008), (7, 5007)])
def test_top_logits_rows_start_anywhere(offset, ld, dtype):
    z = (torch.randn(6, 5001, generator=gen(offset), device="cuda") * 3.0).to(dtype)
    check_top(placed(z, ld, offset), 40)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_top_logits_of_ties(dtype):
    g = gen(3)
    few = torch.randint(0, 3, (4, 40000), generator=g, device="cuda").to(dtype)
    check_top(few, 256)
    check_top(torch.full((3, 70001), 1.5, dtype=dtype, device="cuda"), 100)   # one value
    zeros = torch.zeros(2, 3001, dtype=dtype, device="cuda")
    zeros[:, ::2] = -0.0                                                       # both zeros tie
    check_top(zeros, 50)
    steps = (torch.arange(20000, device="cuda") // 97).to(dtype).expand(2, -1)
    check_top(steps.contiguous(), 120)                                         # rising
    check_top(steps.flip(1).contiguous(), 120)                                 # falling


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_top_logits_of_masked_rows(dtype):
    z = (torch.randn(5, 30011, generator=gen(4), device="cuda") * 3.0).to(dtype)
    z[0] = -INF                         # nothing left
    z[1, 5:] = -INF                     # fewer left than asked for
    z[2, :-3] = -INF
    z[3, 100:20000] = -INF
    z[4] = torch.finfo(dtype).min       # masked with the lowest value
    z[4, 17] = 2.0
    check_top(z, 64)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_top_logits_of_rows_that_keep_rising(dtype):
    """Rows whose first part says little about the rest: more is put aside
    than the lists hold."""
    g = gen(31)
    vocab = 100003
    ramp = torch.linspace(-300.0, 300.0, vocab, device="cuda").expand(2, -1)
    check_top((ramp + torch.randn(2, vocab, generator=g, device="cuda")).to(dtype), 100)
    check_top((ramp.flip(1) + torch.randn(2, vocab, generator=g, device="cuda")).to(dtype), 100)
    late = torch.randn(2, vocab, generator=g, device="cuda")
    late[:, 70000:] += 50.0
    check_top(late.to(dtype), 256)
    few = torch.randn(3, vocab, generator=g, device="cuda")
    few[:, 9000:] = few[:, 9000:].round()           # ties of a handful of values
    check_top(few.to(dtype), 200)
    down = -torch.randn(2, vocab, generator=g, device="cuda").abs() - 1.0   # negative values only
    down[1, 30000:] = -1.0
    check_top(down.to(dtype), 77)


def test_top_logits_never_leaves_the_row():
    """NaN and inf give unspecified values, but places inside the row, and
    outputs that end where they should."""
    z = torch.randn(4, 5001, generator=gen(5), device="cuda")
    z[0] = float("nan")
    z[1, ::3] = float("nan")
    z[2, 7] = INF
    z[3, ::2] = -float("nan")
    made = api.top_logits(z, 30)
    api.check_device()
    assert ((made["indices"] >= 0) & (made["indices"] < 5001)).all()
    assert made["indices"][2, 0] == 7
    vals = torch.full((4 * 30 + 8,), 7.0, device="cuda")
    idx = torch.full((4 * 30 + 8,), 7, dtype=torch.int32, device="cuda")
    lse = torch.full((4 + 8,), 7.0, device="cuda")
    st = Q.quasar_top_logits(z, Q.F32, 5001, 4, 5001, 30, 1.0, vals, idx, lse)
    assert st == Q.QuasarStatus.OK
    assert (vals[120:] == 7.0).all() and (idx[120:] == 7).all() and (lse[4:] == 7.0).all()


# -- distillation ------------------------------------------------------------------

def reference(logits, indices, values, teacher_lse, weight, tau):
    """(loss, grad, loss tolerance, grad tolerance) in fp64, rows one by one."""
    rows, vocab = logits.shape
    loss = torch.zeros(rows, dtype=torch.float64, device="cuda")
    grad = torch.zeros(rows, vocab, dtype=torch.float64, device="cuda")
    t_loss, t_grad = torch.zeros_like(loss), torch.zeros_like(grad)
    for r in range(rows):
        w = 1.0 if weight is None else float(weight[r])
        if w == 0.0:
            continue
        z = logits[r].double() / tau
        here = (indices[r] >= 0) & (indices[r] < vocab)
        at = indices[r][here].long()
        t = values[r][here].double() / tau
        rest = torch.ones(vocab, dtype=torch.bool, device="cuda")
        rest[at] = False
        lse = torch.logsumexp(z, 0)
        log_q = z - lse
        q = log_q.exp()
        q_r = q[rest].sum()
        log_q_r = torch.logsumexp(log_q[rest], 0) if bool(rest.any()) else torch.tensor(-INF)
        if teacher_lse is None:
            if at.numel() == 0 or not bool((t > -INF).any()):
                continue
            log_p = t - torch.logsumexp(t, 0)
            p_r = torch.tensor(0.0, dtype=torch.float64, device="cuda")
        else:
            log_p = t - teacher_lse[r].double()
            p_r = (1.0 - log_p.exp().sum()).clamp(min=0.0) * bool(rest.any())
        p = log_p.exp()
        parts = torch.where(p > 0, p * (log_p - log_q[at]), 0.0)
        loss[r] = parts.sum()
        slack = parts.abs().sum() + (p - q[at]).abs().sum() + (p_r - q_r).abs()
        if float(p_r) > 0:
            loss[r] += p_r * (p_r.log() - log_q_r)
            slack = slack + (p_r * (p_r.log() - log_q_r)).abs()
        mass = p.sum() + p_r
        u = torch.where(rest, (log_q - log_q_r).exp(), 0.0) if float(log_q_r) > -INF else torch.zeros_like(q)
        d = u * (mass * q_r - p_r)
        d[at] = mass * q[at] - p
        grad[r] = d * w / tau
        zf = z[torch.isfinite(z)].abs()
        top = max(float(zf.max()) if zf.numel() else 0.0, abs(float(lse)) if math.isfinite(float(lse)) else 0.0,
                  float(t[torch.isfinite(t)].abs().max()) if bool(torch.isfinite(t).any()) else 0.0)
        e = 2.0 ** -22 * (2 + top)
        t_loss[r] = 2 * e * (slack + 1e-6) + 2.0 ** -21 * loss[r].abs()
        if float(p_r) > 0:  # p_r = 1 - sum p carries the error of every p
            t_loss[r] += e * p.sum() * (log_q_r - p_r.log()).abs()
        tg = u * e * (q_r + p_r + (p.sum() if teacher_lse is not None else 0.0))
        tg[at] = e * (q[at] + p)
        t_grad[r] = 2 * tg * abs(w) / tau + 1e-30
    return loss, grad, t_loss, t_grad


def teacher_of(z, k, tau, seed, noise=0.5):
    t = z.float() + noise * torch.randn(z.shape, generator=gen(seed + 1000), device="cuda")
    v, i = torch.topk(t, k, dim=1)
    return i.int(), v, torch.logsumexp(t / tau, 1)


def check_distill(z, indices, values, teacher_lse, weight, tau):
    loss, grad, t_loss, t_grad = reference(z, indices, values, teacher_lse, weight, tau)
    made = api.distill_top(z, indices, values, teacher_lse=teacher_lse, row_weight=weight,
                           temperature=tau, stats=True)
    api.check_device()
    finite = torch.isfinite(loss)
    assert torch.equal(torch.isfinite(made["loss"]), finite)
    off = (made["loss"].double() - loss).abs()
    assert (off <= t_loss)[finite].all(), float((off / t_loss)[finite].max())
    bad = outside(made["grad"], grad, t_grad)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:3].tolist())
    alone = api.distill_top(z, indices, values, teacher_lse=teacher_lse, row_weight=weight,
                            temperature=tau, grad=False)
    assert torch.equal(alone["loss"], made["loss"])
    back = api.distill_top_backward(z, indices, values, made["stats"], weight,
                                    teacher_lse=teacher_lse, temperature=tau)
    bad = outside(back, grad, t_grad)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:3].tolist())
    return made


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("rows,vocab,k,tau", [
    (1, 2, 1, 1.0), (3, 9, 4, 1.0), (5, 1000, 256, 0.7), (40, 511, 20, 2.0), (3, 4099, 64, 1.0),
    (2, 32003, 100, 2.0), (2, 131072, 64, 1.0), (1, 200001, 200, 1.3),
])
def test_distill(rows, vocab, k, tau, tail, dtype):
    z = (torch.randn(rows, vocab, generator=gen(vocab + k), device="cuda") * 3.0).to(dtype)
    indices, values, lse = teacher_of(z, k, tau, vocab)
    weight = torch.rand(rows, generator=gen(1), device="cuda") + 0.1
    check_distill(z, indices, values, lse if tail else None, weight, tau)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset,ld,ld_grad,off_grad", [
    (0, 3001, 3001, 0), (1, 3001, 3001, 1), (1, 3003, 3008, 0), (4, 3008, 3001, 3), (7, 3004, 3004, 3)])
def test_distill_rows_start_anywhere(offset, ld, ld_grad, off_grad, dtype):
    z = (torch.randn(5, 3001, generator=gen(offset), device="cuda") * 3.0).to(dtype)
    indices, values, lse = teacher_of(z, 30, 1.0, 2)
    _, grad, _, t_grad = reference(z, indices, values, lse, None, 1.0)
    size = off_grad + 5 * ld_grad + 16
    flat = torch.full((size,), 77.0, dtype=dtype, device="cuda")
    out = flat[off_grad:off_grad + 5 * ld_grad].view(5, ld_grad)
    api.distill_top(placed(z, ld, offset), indices, values, teacher_lse=lse, out=out[:, :3001])
    api.check_device()
    assert not outside(out[:, :3001], grad, t_grad).any()
    assert (out[:, 3001:] == 77.0).all()
    assert (flat[:off_grad] == 77.0).all() and (flat[off_grad + 5 * ld_grad:] == 77.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("backward", [False, True])
def test_distill_in_place(dtype, backward):
    z = (torch.randn(9, 20003, generator=gen(8), device="cuda") * 3.0).to(dtype)
    indices, values, lse = teacher_of(z, 50, 1.0, 9)
    made = api.distill_top(z, indices, values, teacher_lse=lse, stats=True)
    mine = z.clone()
    if backward:
        want = api.distill_top_backward(z, indices, values, made["stats"], None, teacher_lse=lse)
        api.distill_top_backward(mine, indices, values, made["stats"], None, teacher_lse=lse, out=mine)
    else:
        want = made["grad"]
        api.distill_top(mine, indices, values, teacher_lse=lse, out=mine)
    assert torch.equal(mine, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [True, False])
def test_distill_ragged_lists(dtype, tail):
    """Rows that list fewer than k entries, or none."""
    z = (torch.randn(6, 5003, generator=gen(10), device="cuda") * 3.0).to(dtype)
    indices, values, lse = teacher_of(z, 40, 1.0, 11)
    indices[0, 7:] = -1
    indices[1] = -1
    indices[2, ::2] = 5003           # just past the vocabulary
    indices[3, 0] = 2**31 - 1
    values[4] = -INF                 # listed, without mass
    values[5, 3:] = -INF
    made = check_distill(z, indices, values, lse if tail else None, None, 1.0)
    if not tail:
        for r in (1, 4):
            assert float(made["loss"][r]) == 0.0 and not made["grad"][r].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("backward", [False, True])
def test_rows_that_count_nothing_are_not_read(dtype, backward):
    z = (torch.randn(6, 4001, generator=gen(12), device="cuda") * 3.0).to(dtype)
    indices, values, lse = teacher_of(z, 40, 1.0, 13)
    weight = torch.tensor([1.0, 0.0, 0.5, 0.0, -0.0, 2.0], device="cuda")
    clean = api.distill_top(z, indices, values, teacher_lse=lse, row_weight=weight, stats=True)
    z[1], values[1], lse[1] = float("nan"), float("nan"), float("nan")
    z[3] = INF
    if backward:
        got = api.distill_top_backward(z, indices, values, clean["stats"], weight, teacher_lse=lse)
        want = api.distill_top_backward(torch.nan_to_num(z), indices, torch.nan_to_num(values),
                                        clean["stats"], weight, teacher_lse=torch.nan_to_num(lse))
        assert torch.equal(got, want)
    else:
        made = api.distill_top(z, indices, values, teacher_lse=lse, row_weight=weight)
        assert torch.equal(made["loss"], clean["loss"]) and torch.equal(made["grad"], clean["grad"])
        got = made["grad"]
        assert (made["loss"][[1, 3, 4]] == 0).all()
    assert not got[[1, 3, 4]].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [True, False])
def test_distill_masked_logits(dtype, tail):
    vocab = 3000
    z = (torch.randn(5, vocab, generator=gen(14), device="cuda") * 3.0).to(dtype)
    indices, values, lse = teacher_of(z, 20, 1.0, 15)
    rest = torch.ones(5, vocab, dtype=torch.bool, device="cuda").scatter_(1, indices.long(), False)
    z[0][rest[0]] = -INF                        # the student has nothing outside the list
    z[1, int(indices[1, 4])] = -INF             # nor at one listed entry: the loss is inf
    z[2, 1500:][rest[2, 1500:]] = -INF          # half the vocabulary masked
    z[3][rest[3]] = torch.finfo(dtype).min      # masked with the lowest value
    indices[4] = -1
    made = check_distill(z, indices, values, lse if tail else None, None, 1.0)
    assert float(made["loss"][1]) == INF
    assert torch.isfinite(made["grad"]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tau", [0.7, 1.3, 2.5, 3.0])
def test_distill_masked_logits_at_any_temperature(dtype, tau):
    z = (torch.randn(3, 2005, generator=gen(32), device="cuda") * 3.0).to(dtype)
    indices, values, lse = teacher_of(z, 20, tau, 33)
    rest = torch.ones(3, 2005, dtype=torch.bool, device="cuda").scatter_(1, indices.long(), False)
    z[:, 900:][rest[:, 900:]] = -INF
    made = check_distill(z, indices, values, lse, None, tau)
    assert torch.isfinite(made["grad"]).all()


def test_distill_with_everything_listed():
    z = torch.randn(4, 200, generator=gen(16), device="cuda") * 3.0
    indices, values, lse = teacher_of(z, 200, 1.0, 17)
    both = check_distill(z, indices, values, lse, None, 1.0)
    alone = check_distill(z, indices, values, None, None, 1.0)
    assert torch.allclose(both["loss"], alone["loss"], rtol=1e-4, atol=1e-6)


def test_distill_far_apart():
    """A student that puts the rest (or the list) far below what fp32 can hold
    beside the other."""
    z = torch.randn(3, 4000, generator=gen(18), device="cuda")
    indices, values, lse = teacher_of(z, 16, 1.0, 19)
    z[0].scatter_(0, indices[0].long(), 300.0)
    z[1].scatter_(0, indices[1].long(), -300.0)
    z[2] *= 40.0
    check_distill(z, indices, values, lse, None, 1.0)
    check_distill(z, indices, values, None, None, 1.0)


@pytest.mark.parametrize("tail", [True, False])
def test_the_gradient_is_that_of_the_loss(tail):
    """Central differences of the fp64 loss, in random directions and single
    entries: the error of a difference is h^2 times a third derivative (below
    1 for these sums) and rounding."""
    vocab, k, tau = 60, 9, 1.5
    z = (torch.randn(3, vocab, generator=gen(20), device="cuda") * 2.0)
    indices, values, lse = teacher_of(z, k, tau, 21)
    weight = torch.tensor([1.0, 0.3, 2.0], device="cuda")
    made = api.distill_top(z, indices, values, teacher_lse=lse if tail else None, row_weight=weight,
                           temperature=tau)

    def total(zz):
        loss = reference(zz, indices, values, lse if tail else None, None, tau)[0]
        return float((loss * weight.double()).sum())

    h = 1e-4
    g = gen(22)
    steps = [torch.randn(3, vocab, generator=g, device="cuda").double() for _ in range(4)]
    for at in (0, 5, int(indices[0, 0]), int(indices[0, k - 1])):
        one = torch.zeros(3, vocab, dtype=torch.float64, device="cuda")
        one[0, at] = 1.0
        steps.append(one)
    for s in steps:
        want = (total(z.double() + h * s) - total(z.double() - h * s)) / (2 * h)
        got = float((made["grad"].double() * s).sum())
        assert abs(got - want) <= 1e-5 * float(s.norm())


def test_top_logits_feed_the_distillation():
    z = (torch.randn(8, 9001, generator=gen(23), device="cuda") * 3.0).to(BF16)
    t = api.top_logits(z, 64, temperature=2.0)
    made = api.distill_top(z, t["indices"], t["values"], teacher_lse=t["lse"], temperature=2.0)
    # the student is the teacher
    assert (made["loss"].abs() <= 2.0 ** -22 * (2 + z.float().abs().max()) * 4).all()
    scale = api.distill_top(z, t["indices"], t["values"] + 1.0, teacher_lse=t["lse"], temperature=2.0)
    assert made["grad"].float().abs().max() < 1e-4 < scale["grad"].float().abs().max()


def test_the_same_bits_every_time():
    z = (torch.randn(64, 40001, generator=gen(24), device="cuda") * 3.0).to(BF16)
    t = api.top_logits(z, 100)
    w = torch.rand(64, generator=gen(25), device="cuda")
    first = api.distill_top(z, t["indices"], t["values"], row_weight=w, stats=True)
    for _ in range(5):
        again = api.distill_top(z, t["indices"], t["values"], row_weight=w, stats=True)
        for name in first:
            assert torch.equal(first[name], again[name]), name
        assert torch.equal(api.top_logits(z, 100)["lse"], t["lse"])


@pytest.mark.parametrize("dtype,vocab", [(F32, 1 << 20), (BF16, 1500007)])
def test_long_rows(dtype, vocab):
    z = (torch.randn(2, vocab, generator=gen(27), device="cuda") * 3.0).to(dtype)
    check_top(z, 200)
    indices, values, lse = teacher_of(z, 200, 1.0, 28)
    check_distill(z, indices, values, lse, None, 1.0)


def test_many_long_rows():
    """More rows than SMs, each longer than one CTA can describe."""
    vocab, rows = (1 << 20) + 3, 160
    z = torch.randn(rows, vocab, generator=gen(34), device="cuda")
    t = api.top_logits(z, 20)
    made = api.distill_top(z, t["indices"], t["values"] + 0.5, stats=True)
    api.check_device()
    for r in (0, 77, 159):
        v, i = torch.sort(z[r], descending=True, stable=True)
        assert torch.equal(t["values"][r], v[:20]) and torch.equal(t["indices"][r].long(), i[:20])
        row = slice(r, r + 1)
        loss, grad, t_loss, t_grad = reference(z[row], t["indices"][row], t["values"][row] + 0.5, None,
                                               None, 1.0)
        assert ((made["loss"][row].double() - loss).abs() <= t_loss).all()
        assert not outside(made["grad"][row], grad, t_grad).any()


def test_offsets_past_32_bits():
    """Rows so far apart that element offsets pass 2^32."""
    rows, vocab, ld = 3, 5003, (1 << 31) + 5
    logits = torch.empty((rows - 1) * ld + vocab + 8, dtype=BF16, device="cuda")
    out = torch.empty((rows - 1) * ld + vocab + 8, dtype=BF16, device="cuda")
    z = logits[3:].as_strided((rows, vocab), (ld, 1))
    g = out[1:].as_strided((rows, vocab), (ld, 1))
    z.copy_(torch.randn(rows, vocab, generator=gen(35), device="cuda") * 3.0)
    check_top(z, 40)
    indices, values, lse = teacher_of(z, 40, 1.0, 36)
    _, grad, _, t_grad = reference(z, indices, values, lse, None, 1.0)
    api.distill_top(z, indices, values, teacher_lse=lse, out=g)
    api.check_device()
    assert not outside(g, grad, t_grad).any()


def test_in_a_graph():
    """Captured once, replayed on new values: a step's calls in their order."""
    z = (torch.randn(40, 9001, generator=gen(37), device="cuda") * 3.0).to(BF16)
    grad, side = torch.empty_like(z), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        t = api.top_logits(z, 32)
        api.distill_top(z, t["indices"], t["values"], teacher_lse=t["lse"], out=grad)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t = api.top_logits(z, 32)
        made = api.distill_top(z, t["indices"], t["values"] - 0.25, teacher_lse=t["lse"], out=grad)
    for seed in (38, 39):
        z.copy_(torch.randn(40, 9001, generator=gen(seed), device="cuda") * 3.0)
        graph.replay()
        torch.cuda.synchronize()
        again = api.top_logits(z, 32)
        assert torch.equal(again["indices"], t["indices"]) and torch.equal(again["lse"], t["lse"])
        want = api.distill_top(z, again["indices"], again["values"] - 0.25, teacher_lse=again["lse"])
        assert torch.equal(want["loss"], made["loss"]) and torch.equal(want["grad"], grad)


def test_a_row_without_a_finite_logit():
    z = torch.full((2, 5000), -INF, device="cuda")
    z[1] = torch.randn(5000, generator=gen(29), device="cuda")
    indices = torch.arange(20, dtype=torch.int32, device="cuda").expand(2, 20).contiguous()
    values = torch.randn(2, 20, generator=gen(30), device="cuda")
    made = api.distill_top(z, indices, values, stats=True)
    assert float(made["loss"][0]) == INF and math.isfinite(float(made["loss"][1]))
    assert not made["grad"][0].any() and torch.isfinite(made["grad"]).all()
    back = api.distill_top_backward(z, indices, values, made["stats"], None)
    assert not back[0].any() and torch.isfinite(back).all()


def test_a_wait_that_runs_out_is_reported():
    z = (torch.randn(4, 9001, generator=gen(26), device="cuda") * 3.0).to(BF16)
    want = api.top_logits(z, 8)
    d = api.distill_top(z, want["indices"], want["values"])
    api.check_device()
    for call in (lambda: api.top_logits(z, 8),
                 lambda: api.distill_top(z, want["indices"], want["values"])):
        Q.quasar_debug_force_timeout(1_000_000)
        try:
            call()
            assert Q.quasar_get_device_status() == Q.QuasarStatus.ERR_TIMEOUT
        finally:
            Q.quasar_debug_force_timeout(0)
    assert torch.equal(api.top_logits(z, 8)["values"], want["values"])
    assert torch.equal(api.distill_top(z, want["indices"], want["values"])["loss"], d["loss"])
    api.check_device()
