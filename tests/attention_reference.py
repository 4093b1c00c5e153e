"""Attention over packed sequences in fp64, and how far a kernel may be off.

With u = 2^-24: a score is a sum of d exact products, truncated as the tensor
core accumulates (a step, 2u, of the sum of sizes per instruction of 16), times
the scale; the exponent's argument is rounded at its own size, and exp2 is good
to 4u.  e_p is what that makes of a probability, relative to it.  Rounded to
bf16, a probability is off by half a step, 2^-8 of it, and sums over n keys are
truncated in n / 16 instructions."""
import torch

U = 2.0 ** -24
HALF = 2.0 ** -8  # of bf16


def starts_of(lengths, first=0, device="cuda"):
    at = [first]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device=device)


def by_head(t, d, kv_heads):
    return t.double().reshape(t.shape[0], kv_heads, t.shape[1] // (kv_heads * d), d).permute(1, 2, 0, 3)


def together(t):
    return t.permute(2, 0, 1, 3).reshape(t.shape[2], t.shape[0] * t.shape[1] * t.shape[3])


def scores(q, k, d, kv_heads, causal, scale):
    """s, the seen pairs and e_p of one sequence, [kv_heads, group, n, m]."""
    qs, ks = by_head(q, d, kv_heads), by_head(k, d, kv_heads)
    s = qs @ ks.transpose(2, 3) * scale
    size = qs.abs() @ ks.abs().transpose(2, 3) * scale
    n, m = s.shape[2:]
    seen = torch.ones(n, m, dtype=torch.bool, device=s.device)
    if causal:
        seen = seen.tril(m - n)
    top = s.masked_fill(~seen, 0.0).abs().amax(3, keepdim=True) if m else 0.0
    e_p = size * (d / 16 + 4) * 2 * U + (s.abs() + top) * 4 * U + 8 * U
    return s.masked_fill(~seen, -torch.inf), seen, e_p


def softmax(s):
    if s.shape[3] == 0:
        return s, torch.full_like(s.sum(3, keepdim=True), -torch.inf)
    lse = torch.logsumexp(s, 3, keepdim=True)
    p = torch.exp(s - lse)
    return torch.where(lse == -torch.inf, 0.0, p), lse


def forward(q, k, v, d, kv_heads, causal, scale):
    """y, lse and the bounds of both, before y is rounded."""
    s, seen, e_p = scores(q, k, d, kv_heads, causal, scale)
    p, lse = softmax(s)
    vs = by_head(v, d, kv_heads)
    m = s.shape[3]
    y = p @ vs
    mean_e = (p * e_p).sum(3, keepdim=True)  # of the sum of probabilities
    e_y = (p * (HALF + e_p + mean_e + (m / 16 + 16) * 2 * U)) @ vs.abs()
    e_lse = mean_e + (m / 32 + 16) * U + 4 * U * lse.abs().nan_to_num(0, 0, 0)
    return together(y), together(lse), together(e_y), together(e_lse)


def backward(dy, q, k, v, d, kv_heads, causal, scale):
    """dq, dk, dv and their bounds, before they are rounded.  The kernel reads y
    rounded to bf16 (half a step) for the row's sum of dy y."""
    s, seen, e_p = scores(q, k, d, kv_heads, causal, scale)
    p, lse = softmax(s)
    n, m = s.shape[2:]
    qs, ks, vs, dys = (by_head(t, d, kv_heads) for t in (q, k, v, dy))
    dp = dys @ vs.transpose(2, 3)
    dp_size = dys.abs() @ vs.abs().transpose(2, 3)
    y = p @ vs
    e_y = (p * (HALF + e_p + (p * e_p).sum(3, keepdim=True) + (m / 16 + 16) * 2 * U)) @ vs.abs()
    delta = (dys * y).sum(3, keepdim=True)
    e_delta = (dys.abs() * (e_y + HALF * (y.abs() + e_y))).sum(3, keepdim=True) + (d + 8) * U * (dys * y).abs().sum(3, keepdim=True)
    e_p = e_p + (p * e_p).sum(3, keepdim=True) + 8 * U + 4 * U * lse.abs().nan_to_num(0, 0, 0)  # (the lse is rounded, too)
    ds = p * (dp - delta) * scale
    e_ds = scale * p * ((e_p + HALF) * (dp - delta).abs() + (1 + HALF) * ((d / 16 + 8) * 2 * U * dp_size + e_delta)) + \
        (HALF + 8 * U) * ds.abs()
    sums = lambda count: (count / 16 + 16) * 2 * U  # noqa: E731
    dq = ds @ ks
    e_dq = (e_ds + sums(m) * ds.abs()) @ ks.abs()
    group = qs.shape[1]
    dk = (ds.transpose(2, 3) @ qs).sum(1, keepdim=True)
    e_dk = ((e_ds + sums(n * group) * ds.abs()).transpose(2, 3) @ qs.abs()).sum(1, keepdim=True)
    dv = (p.transpose(2, 3) @ dys).sum(1, keepdim=True)
    e_dv = ((p * (HALF + e_p + sums(n * group))).transpose(2, 3) @ dys.abs()).sum(1, keepdim=True)
    return tuple(together(t) for t in (dq, dk, dv, e_dq, e_dk, e_dv))
