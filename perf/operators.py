"""Cases of the training-step operators around the reconstruction.

Four operators, in two directions where training needs them:

- ``linear``: y = act(x r^T + bias) + residual, with r the reconstructed
  weights the forward pass reads;
- ``linear_backward``: from dz, the gradient at the product, the gradients of
  the product's input (times the derivative of the activation that made that
  input, where one did), of r (the g that the next reconstruction reads) and
  of the bias;
- ``top_logits``: a teacher's k largest logits of each row with their indices
  and the row's log-sum-exp;
- ``distill``: the forward KL divergence of a student's logits from a
  teacher's top logits, its gradient, or both in one call.

``own`` chooses between the plain form (elementary torch operations in 32
bits) and the package's kernels.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# -- cases ---------------------------------------------------------------------

def _linear(name, tokens, features, inputs, activation="none", bias=False, residual=False,
            out="bf16", save_pre=False):
    return {"name": name, "op": "linear", "tokens": tokens, "features": features,
            "inputs": inputs, "activation": activation, "bias": bias, "residual": residual,
            "out": out, "save_pre": save_pre}


def _linear_backward(name, tokens, features, inputs, activation="none", bias=False, dr="bf16"):
    return {"name": name, "op": "linear_backward", "tokens": tokens, "features": features,
            "inputs": inputs, "activation": activation, "bias": bias, "dr": dr}


def _top_logits(name, rows, vocab, k, dtype="bf16", temperature=1.0):
    return {"name": name, "op": "top_logits", "rows": rows, "vocab": vocab, "k": k,
            "dtype": dtype, "temperature": temperature}


def _distill(name, rows, vocab, k, direction="both", dtype="bf16", tail=True, temperature=1.0,
             padded=False):
    return {"name": name, "op": "distill", "rows": rows, "vocab": vocab, "k": k,
            "direction": direction, "dtype": dtype, "tail": tail, "temperature": temperature,
            "padded": padded}


def listed():
    return [
        # one new token through the gate projection of the 4096-wide layer: serving's step
        _linear("linear_1_token", 1, 14336, 4096, activation="silu"),
        # a small batch of new tokens through the down projection, added to the stream
        _linear("linear_23_tokens", 23, 4096, 14336, residual=True),
        # a ragged batch into an odd number of outputs, in 32 bits, with a bias (a head)
        _linear("linear_ragged", 1001, 1003, 4096, bias=True, out="f32"),
        # a training batch through the gate projection; the pre-activation is kept
        _linear("linear_8192_tokens", 8192, 14336, 4096, activation="silu", bias=True,
                save_pre=True),
        # a short batch back through the key projection, the weight's gradient in 32 bits
        _linear_backward("linear_backward_short", 77, 1024, 4096, bias=True, dr="f32"),
        # a training batch back through the down projection and the activation before it
        _linear_backward("linear_backward_4096_tokens", 4096, 4096, 12288, activation="silu"),
        # one row: the teacher's answer for one new token
        _top_logits("top_logits_1_row", 1, 131072, 64),
        # an odd vocabulary in 32 bits (rows start at any 4-byte address)
        _top_logits("top_logits_odd_f32", 301, 50001, 128, dtype="f32", temperature=2.0),
        # a teacher's training batch
        _top_logits("top_logits_2048_rows", 2048, 131072, 64),
        # a handful of rows in 32 bits, the loss alone (evaluation)
        _distill("distill_loss_few_rows", 7, 131072, 64, direction="loss", dtype="f32"),
        # odd rows with padding tokens, renormalised over the k, the gradient from kept
        # statistics (the way autograd calls it)
        _distill("distill_grad_odd", 511, 50001, 100, direction="grad", tail=False,
                 temperature=2.0, padded=True),
        # a training batch: loss and gradient in one call
        _distill("distill_4096_rows", 4096, 131072, 64, padded=True),
    ]


def _between(rng, low, high):
    """A whole number, spread over the logarithm of [low, high]."""
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["linear", "linear_backward", "top_logits", "distill"])
    if op in ("linear", "linear_backward"):
        most = 8192 * 14336 * 4096 if op == "linear" else 4096 * 4096 * 12288
        while True:
            tokens = _between(rng, 1, 8192)
            features = _between(rng, 64, 14336)
            inputs = 8 * _between(rng, 8, 1792)
            if tokens * features * inputs <= most and 3072 not in (tokens, features, inputs):
                break
        activation = rng.choice(["none", "relu", "gelu", "silu"])
        if op == "linear":
            return _linear("", tokens, features, inputs, activation, rng.random() < 0.5,
                           rng.random() < 0.5, rng.choice(["bf16", "f32"]),
                           rng.random() < 0.5) | {"name": "drawn"}
        return _linear_backward("drawn", tokens, features, inputs, activation,
                                rng.random() < 0.5, rng.choice(["bf16", "f32"]))
    most = 2048 * 131072 if op == "top_logits" else 4096 * 131072
    while True:
        rows, vocab = _between(rng, 1, 4096), _between(rng, 1000, 200000)
        dtype = rng.choice(["bf16", "f32"])
        if rows * vocab * (2 if dtype == "f32" else 1) <= most and 3072 not in (rows, vocab):
            break
    temperature = rng.choice([1.0, 1.0, 2.0, 0.7])
    if op == "top_logits":
        return _top_logits("drawn", rows, vocab, _between(rng, 1, 128), dtype, temperature)
    return _distill("drawn", rows, vocab, _between(rng, 1, 256),
                    rng.choice(["both", "both", "loss", "grad"]), dtype, rng.random() < 0.6,
                    temperature, rng.random() < 0.5)


# -- inputs --------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _levels(g, features, inputs):
    """Weights as a 3-bit reconstruction leaves them: eight levels a q + b in each group of a
    row, in bf16.  Groups of 128, or of the largest power of two that divides the row."""
    group = 8 * math.gcd(inputs // 8, 16)
    w = (torch.randn(features, inputs, generator=g, device="cuda") * 0.02).view(-1, group)
    low, high = w.amin(1, keepdim=True), w.amax(1, keepdim=True)
    step = (high - low) / 7
    return (torch.round((w - low) / step) * step + low).view(features, inputs).to(torch.bfloat16)


def _padded_rows(t, multiple=8):
    """The same values in storage whose rows start at 16-byte boundaries, as a program that
    goes on to differentiate keeps its activations."""
    rows, cols = t.shape
    wide = torch.zeros(rows, -(-cols // multiple) * multiple, dtype=t.dtype, device=t.device)
    wide[:, :cols] = t
    return wide[:, :cols]


def _logits(g, rows, vocab, dtype):
    """A student's logits, and its teacher's: nearby, with a few clear favourites a row."""
    student = torch.randn(rows, vocab, generator=g, device="cuda") * 2.0
    favourites = torch.randint(0, vocab, (rows, 16), generator=g, device="cuda")
    lift = torch.rand(rows, 16, generator=g, device="cuda") * 10.0
    student.scatter_add_(1, favourites, lift)
    teacher = student + torch.randn(rows, vocab, generator=g, device="cuda") * 0.5
    return student.to(dtype), teacher


def prepare(case, seed):
    g = _generator(seed)
    state = {"case": case}
    if case["op"] == "linear":
        tokens, features, inputs = case["tokens"], case["features"], case["inputs"]
        state["x"] = _normal(g, tokens, inputs)
        state["r"] = _levels(g, features, inputs)
        state["bias"] = _normal(g, features, scale=0.1, dtype=torch.float32) if case["bias"] else None
        state["residual"] = (_normal(g, tokens, features, dtype=DTYPES[case["out"]])
                             if case["residual"] else None)
    elif case["op"] == "linear_backward":
        tokens, features, inputs = case["tokens"], case["features"], case["inputs"]
        state["dz"] = _padded_rows(_normal(g, tokens, features, scale=1e-2))
        state["x"] = _normal(g, tokens, inputs)
        state["r"] = _levels(g, features, inputs)
        state["pre"] = _normal(g, tokens, inputs) if case["activation"] != "none" else None
    elif case["op"] == "top_logits":
        state["logits"] = _logits(g, case["rows"], case["vocab"], DTYPES[case["dtype"]])[0]
    else:
        rows, k, tau = case["rows"], case["k"], case["temperature"]
        student, teacher = _logits(g, rows, case["vocab"], DTYPES[case["dtype"]])
        values, indices = torch.topk(teacher, k, dim=1)
        state["logits"], state["values"] = student, values
        state["indices"] = indices.to(torch.int32)
        state["teacher_lse"] = torch.logsumexp(teacher / tau, 1) if case["tail"] else None
        # what a row counts in the mean over the tokens; padding tokens count nothing
        live = torch.ones(rows, device="cuda")
        if case["padded"]:
            live = (torch.rand(rows, generator=g, device="cuda") < 0.9).float()
        state["row_weight"] = live / live.sum().clamp(min=1.0)
        state["stats"] = None
        if case["direction"] == "grad":
            scaled = student.float() / tau
            rest = scaled.scatter(1, indices, -math.inf)
            state["stats"] = torch.stack([torch.logsumexp(scaled, 1), torch.logsumexp(rest, 1)], 1)
    return state


# -- the operators -------------------------------------------------------------

def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_derivative(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
                + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi))
    return torch.ones_like(z)


def _plain_linear(state, case):
    z = state["x"].float() @ state["r"].float().t()
    if state["bias"] is not None:
        z = z + state["bias"]
    y = _act(z, case["activation"])
    if state["residual"] is not None:
        y = y + state["residual"].float()
    result = {"y": y.to(DTYPES[case["out"]])}
    if case["save_pre"]:
        result["pre"] = z.to(torch.bfloat16)
    return result


def _plain_linear_backward(state, case):
    dz = state["dz"].float()
    dx = dz @ state["r"].float()
    if state["pre"] is not None:
        dx = dx * _act_derivative(state["pre"].float(), case["activation"])
    result = {"dx": dx.to(torch.bfloat16),
              "dr": (dz.t() @ state["x"].float()).to(DTYPES[case["dr"]])}
    if case["bias"]:
        result["dbias"] = dz.sum(0)
    return result


def _lse(z):
    top = z.amax(1, keepdim=True)
    return (top + torch.log(torch.exp(z - top).sum(1, keepdim=True))).squeeze(1)


def _plain_top_logits(state, case):
    z = state["logits"].float()
    ranked, order = torch.sort(z, dim=1, descending=True, stable=True)
    k = case["k"]
    return {"values": ranked[:, :k].contiguous(), "indices": order[:, :k].to(torch.int32),
            "lse": _lse(z / case["temperature"])}


def _plain_distill(state, case):
    tau, direction = case["temperature"], case["direction"]
    z = state["logits"].float() / tau
    listed_ = state["indices"].long()
    t = state["values"] / tau
    if case["tail"]:
        log_p = t - state["teacher_lse"][:, None]
        p = torch.exp(log_p)
        rest_p = (1.0 - p.sum(1)).clamp(min=0.0)
    else:
        log_p = t - _lse(t)[:, None]
        p = torch.exp(log_p)
        rest_p = torch.zeros_like(p[:, 0])
    if state["stats"] is not None:
        lse, rest_lse = state["stats"][:, 0], state["stats"][:, 1]
    else:
        lse, rest_lse = _lse(z), _lse(z.scatter(1, listed_, -math.inf))
    live = state["row_weight"] != 0
    result = {}
    if direction != "grad":
        # p log(p / q) - p + q summed over the entries and the rest: the same sum, because both
        # distributions sum to one, without its cancellation (no term is negative)
        log_q = torch.cat([z.gather(1, listed_), rest_lse[:, None]], 1) - lse[:, None]
        every_p = torch.cat([p, rest_p[:, None]], 1)
        every_log_p = torch.cat([log_p, torch.log(rest_p)[:, None]], 1)
        d = every_log_p - log_q
        term = torch.where(d > -1.0, every_p * (d + torch.expm1(-d)),
                           every_p * (d - 1.0) + torch.exp(log_q))
        loss = torch.where(every_p > 0, term, torch.exp(log_q)).sum(1)
        result["loss"] = torch.where(live, loss, torch.zeros_like(loss))
    if direction != "loss":
        q = torch.exp(z - lse[:, None])
        mass = p.sum(1) + rest_p
        d = q * (mass - rest_p * torch.exp(lse - rest_lse))[:, None]
        d.scatter_(1, listed_, mass[:, None] * q.gather(1, listed_) - p)
        d = d * (state["row_weight"] / tau)[:, None]
        result["grad"] = torch.where(live[:, None], d, torch.zeros_like(d)).to(state["logits"].dtype)
    return result


def _own_run(state, case):
    from paper_2608_13966_gb300 import api

    if case["op"] == "linear":
        return api.linear(state["x"], state["r"], bias=state["bias"],
                          activation=case["activation"], residual=state["residual"],
                          out_dtype=DTYPES[case["out"]], save_pre=case["save_pre"])
    if case["op"] == "linear_backward":
        return api.linear_backward(state["dz"], state["x"], state["r"], pre_in=state["pre"],
                                   activation_in=case["activation"], bias=case["bias"],
                                   dr_dtype=DTYPES[case["dr"]])
    if case["op"] == "top_logits":
        return api.top_logits(state["logits"], case["k"], temperature=case["temperature"])
    common = dict(teacher_lse=state["teacher_lse"], temperature=case["temperature"])
    if case["direction"] == "grad":
        return {"grad": api.distill_top_backward(state["logits"], state["indices"],
                                                 state["values"], state["stats"],
                                                 state["row_weight"], **common)}
    made = api.distill_top(state["logits"], state["indices"], state["values"],
                           row_weight=state["row_weight"], grad=case["direction"] == "both",
                           **common)
    return {name: made[name] for name in ("loss", "grad") if name in made}


def run(state):
    case = state["case"]
    if own:
        return _own_run(state, case)
    return {"linear": _plain_linear, "linear_backward": _plain_linear_backward,
            "top_logits": _plain_top_logits, "distill": _plain_distill}[case["op"]](state, case)


# -- what a pass cannot do without ------------------------------------------------

def work(case):
    if case["op"] in ("linear", "linear_backward"):
        m, n, k = case["tokens"], case["features"], case["inputs"]
        flops = 2.0 * m * n * k
        if case["op"] == "linear":
            out = 2 if case["out"] == "bf16" else 4
            size = 2 * (m * k + n * k) + out * m * n * (2 if case["residual"] else 1)
            size += (4 * n if case["bias"] else 0) + (2 * m * n if case["save_pre"] else 0)
            return {"bytes": size, "flops": flops}
        size = 2 * (m * n + m * k + n * k) + 2 * m * k + (2 if case["dr"] == "bf16" else 4) * n * k
        size += (2 * m * k if case["activation"] != "none" else 0) + (4 * n if case["bias"] else 0)
        return {"bytes": size, "flops": 2 * flops}
    rows, k = case["rows"], case["k"]
    read = rows * case["vocab"] * (2 if case["dtype"] == "bf16" else 4)
    if case["op"] == "top_logits":
        return {"bytes": read + rows * (8 * k + 4), "flops": 2.0 * rows * case["vocab"]}
    live = 0.9 if case["padded"] else 1.0  # padding rows are not read
    size = live * read + rows * (8 * k + 4 + (4 if case["tail"] else 0))
    size += rows * 4 if case["direction"] != "grad" else rows * 8
    size += read if case["direction"] != "loss" else 0
    return {"bytes": size, "flops": 3.0 * rows * case["vocab"]}


# -- the definitions in 64 bits -----------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "linear":
        z = torch.mm(state["x"].double(), state["r"].double().T)
        if state["bias"] is not None:
            z += state["bias"].double()
        y = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0.0),
             "silu": lambda v: v * torch.special.expit(v),
             "gelu": lambda v: v * torch.special.ndtr(v)}[case["activation"]](z)
        if state["residual"] is not None:
            y = y + state["residual"].double()
        return {"y": y, "pre": z} if case["save_pre"] else {"y": y}
    if case["op"] == "linear_backward":
        dz = state["dz"].double()
        dx = torch.mm(dz, state["r"].double())
        if state["pre"] is not None:
            v = state["pre"].double()
            if case["activation"] == "relu":
                dx = torch.where(v > 0, dx, 0.0)
            elif case["activation"] == "silu":
                dx = dx * (torch.special.expit(v) + v * torch.special.expit(v) * torch.special.expit(-v))
            else:
                density = (v.square() * -0.5).exp() * (2.0 * math.pi) ** -0.5
                dx = dx * (torch.special.ndtr(v) + v * density)
        result = {"dx": dx, "dr": torch.mm(dz.T, state["x"].double())}
        if case["bias"]:
            result["dbias"] = torch.einsum("mn->n", dz)
        return result
    z = state["logits"].double() / case["temperature"]
    if case["op"] == "top_logits":
        # ties go to the lowest index, so a row's indices have one right answer
        order = torch.argsort(-state["logits"].double(), dim=1, stable=True)[:, : case["k"]]
        return {"values": state["logits"].double().gather(1, order),
                "indices": order.to(torch.int32), "lse": torch.logsumexp(z, 1)}
    chosen = torch.zeros_like(z, dtype=torch.bool).scatter_(1, state["indices"].long(), True)
    log_q = torch.log_softmax(z, 1)
    rest_log_q = torch.logsumexp(log_q.masked_fill(chosen, -math.inf), 1)
    t = state["values"].double() / case["temperature"]
    if case["tail"]:
        p = (t - state["teacher_lse"].double()[:, None]).exp()
        rest_p = (1.0 - p.sum(1)).clamp(min=0.0)
    else:
        p = torch.softmax(t, 1)
        rest_p = torch.zeros(case["rows"], dtype=torch.float64, device=z.device)
    live = state["row_weight"] != 0
    result = {}
    if case["direction"] != "grad":
        cross = -(p * log_q.gather(1, state["indices"].long())).sum(1)
        cross -= torch.where(rest_p > 0, rest_p * rest_log_q, 0.0)
        entropy = torch.special.entr(p).sum(1) + torch.special.entr(rest_p)
        result["loss"] = torch.where(live, cross - entropy, 0.0)
    if case["direction"] != "loss":
        # d loss / d z = q (sum of p) - p, with the rest's mass spread as the student spreads it
        spread = (rest_p[:, None] * (log_q - rest_log_q[:, None]).exp()).masked_fill(chosen, 0.0)
        target = spread.scatter_add(1, state["indices"].long(), p)
        d = log_q.exp() * (p.sum(1) + rest_p)[:, None] - target
        result["grad"] = d * (state["row_weight"].double() / case["temperature"])[:, None]
    return result
