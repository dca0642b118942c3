"""What is measured of the low-bit student's operators: 4-bit microscaled quantisation, the linear layer on it, and
distillation from a teacher's top logits.

Every case is one pass through an operator as a user's program calls it.  `own` chooses between the plain form
(elementary torch operations in 32 bits) and the framework's kernels.
"""
import math

import torch

own = False

F32, F16, BF16 = "float32", "float16", "bfloat16"
_BYTES = {F32: 4, F16: 2, BF16: 2}
_MX4_BITS = 4 + 8 / 32           # an element and its share of the block's scale


# ---- the cases -------------------------------------------------------------------------------------------
def _quantize(name, rows, cols, dtype, both):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "both": both}


def _linear(name, tokens, k, n, dtype):
    return {"name": name, "op": "linear", "tokens": tokens, "k": k, "n": n, "dtype": dtype}


def _train(name, tokens, k, n, dtype):
    return {"name": name, "op": "train", "tokens": tokens, "k": k, "n": n, "dtype": dtype}


def _distill(name, op, rows, vocab, width, top, dtype, tail, labels, temperature):
    return {"name": name, "op": op, "rows": rows, "vocab": vocab, "width": width, "top": top, "dtype": dtype,
            "tail": tail, "labels": labels, "temperature": temperature}


def listed():
    return [
        # Activations of a few tokens, BERT-Large's hidden width: what latency is worth.
        _quantize("quantize_few_tokens", 16, 1024, BF16, False),
        # A large batch at the width of BERT-Large's feed-forward layer, both orientations, as a training step needs them.
        _quantize("quantize_both_large", 16384, 4096, BF16, True),
        # Generation of one token through the first feed-forward product of the GPT-2 1.5B shape.
        _linear("linear_one_token", 1, 1600, 6400, BF16),
        # A short prompt, or a few requests at once, through the second one: a ragged number of blocks, an odd number of tokens.
        _linear("linear_short_prompt", 77, 6400, 1600, BF16),
        # Evaluation of a large batch at a generic width.
        _linear("linear_large", 16384, 4096, 8192, BF16),
        # One sequence of a small micro-batch through BERT-Large's first feed-forward product, forward and backward.
        _train("train_one_sequence", 512, 1024, 4096, BF16),
        # Odd sizes everywhere and 32-bit gradients.
        _train("train_ragged_f32", 1777, 1001, 1333, F32),
        # A training micro-batch of the GPT-2 1.5B shape.
        _train("train_large", 16384, 1600, 6400, BF16),
        # Validation loss of masked-token predictions: few rows of 32-bit logits, loss alone.
        _distill("distill_loss_masked_tokens", "distill_loss", 76, 30522, 30522, 16, F32, False, True, 1.0),
        # Validation loss of a long batch.
        _distill("distill_loss_large", "distill_loss", 8192, 50257, 50257, 64, BF16, True, False, 2.0),
        # The gradient for a few rows, logits in a padded head.
        _distill("distill_grad_few_rows", "distill_grad", 24, 30522, 30592, 32, F16, False, True, 2.0),
        # The training step's loss and gradient at the GPT-2 vocabulary, every part of the loss in use.
        _distill("distill_grad_large", "distill_grad", 8192, 50257, 50257, 64, BF16, True, True, 2.0),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "train", "distill_loss", "distill_grad"])
    dtype = rng.choice([BF16, BF16, F16, F32])
    if op == "quantize":
        rows, cols = _log_int(rng, 1, 16384), _log_int(rng, 33, 6400)
        cols = min(cols, 16384 * 4096 // rows)
        case = _quantize("", rows, cols, dtype, rng.random() < 0.5)
    elif op in ("linear", "train"):
        tokens, k, n = _log_int(rng, 1, 16384), _log_int(rng, 100, 6400), _log_int(rng, 100, 8192)
        if rng.random() < 0.5:
            k, n = 32 * max(4, k // 32), 64 * max(2, n // 64)
        if op == "train":
            n = min(n, 16384 * 1600 * 6400 // (tokens * k))
        case = _linear("", tokens, k, n, dtype) if op == "linear" else _train("", tokens, k, n, dtype)
    else:
        rows, vocab = _log_int(rng, 1, 8192), _log_int(rng, 1000, 50257)
        if dtype == F32:
            rows = min(rows, 4096)
        width = vocab if rng.random() < 0.5 else 64 * (vocab // 64 + 1)
        case = _distill("", op, rows, vocab, width, _log_int(rng, 1, 64), dtype, rng.random() < 0.5, rng.random() < 0.5,
                        rng.choice([1.0, 1.5, 2.0, 4.0]))
    del case["name"]
    return case


def work(case):
    op = case["op"]
    e = _BYTES[case["dtype"]]
    q = _MX4_BITS / 8
    if op == "quantize":       # read the input; write codes and scales, and the values that are read back from them
        size = case["rows"] * case["cols"]
        sides = 2 if case["both"] else 1
        return {"bytes": size * (e + sides * (2 * q + e)), "flops": 4 * size * sides}
    if op == "linear":         # read x and the 4-bit weight, write y
        m, k, n = case["tokens"], case["k"], case["n"]
        return {"bytes": m * k * e + n * k * q + m * n * e, "flops": 2 * m * k * n}
    if op == "train":          # read x, w, dy; write y, dx, dw; the 4-bit forms of x, w, dy each way are written and read once
        m, k, n = case["tokens"], case["k"], case["n"]
        return {"bytes": 2 * e * (m * k + n * k + m * n) + 4 * q * (m * k + n * k + m * n), "flops": 6 * m * k * n}
    size = case["rows"] * case["vocab"]
    extra = case["rows"] * (case["top"] * (4 + e) + 16)
    return {"bytes": size * e * (2 if op == "distill_grad" else 1) + extra, "flops": size * (12 if op == "distill_grad" else 6)}


# ---- inputs ----------------------------------------------------------------------------------------------
def prepare(case, seed):
    """What a user's program holds before the call.  For `linear` that includes the weight in its 4-bit form: the
    values that it stands for in the plain form, the framework's tensor where the framework runs."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = getattr(torch, case["dtype"])

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    op = case["op"]
    if op == "quantize":
        # Activations: channels of unlike sizes, some rows all zero (padding tokens).
        x = normal(case["rows"], case["cols"]) * torch.exp(normal(1, case["cols"]))
        x[torch.rand(case["rows"], generator=g, device="cuda") < 0.02] = 0
        return {"case": case, "x": x.to(dtype)}
    if op in ("linear", "train"):
        m, k, n = case["tokens"], case["k"], case["n"]
        x = (normal(m, k) * torch.exp(0.5 * normal(1, k))).to(dtype)
        w = (normal(n, k) * 0.02).to(dtype)
        if op == "linear":
            w = _on_grid(w.float()).to(dtype)
            state = {"case": case, "x": x, "w": w}
            if own:
                from paper_2202_06009_b200 import mx4_quantize
                state["w"] = mx4_quantize(w)
            return state
        # Gradients of the output: small, and of unlike sizes from token to token.
        dy = (normal(m, n) * 1e-3 * torch.exp(normal(m, 1))).to(dtype)
        return {"case": case, "x": x, "w": w, "dy": dy}
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    # The teacher's best `top` tokens of each row, best first, and their logits; the last ones are missing (-1) in some
    # rows, all of them in a few.
    start = torch.randint(0, vocab, (rows, 1), generator=g, device="cuda")
    hop = torch.randint(1, max(2, vocab // top), (rows, 1), generator=g, device="cuda")
    index = (start + hop * torch.arange(top, device="cuda")) % vocab
    falls = torch.empty(rows, top, device="cuda").exponential_(2.0, generator=g)
    teacher = (14.0 - falls.cumsum(1)).to(dtype)
    # A student that agrees with it in part.
    logits = 2.0 * normal(rows, case["width"])
    at = torch.arange(rows, device="cuda")[:, None]
    logits[at, index] += 0.6 * teacher.float()
    logits = logits.to(dtype)[:, :vocab]
    short = (torch.rand(rows, 1, generator=g, device="cuda") < 0.1) & (torch.arange(top, device="cuda") >= (top + 1) // 2)
    index = torch.where(short | (torch.rand(rows, 1, generator=g, device="cuda") < 0.02), -1, index).to(torch.int32)
    state = {"case": case, "logits": logits, "index": index, "teacher": teacher,
             "weight": (torch.rand(rows, generator=g, device="cuda") >= 0.05).float() / rows, "lse": None, "labels": None}
    if case["tail"]:           # the teacher's log-sum-exp over its whole vocabulary: 2% to 30% of its mass lies outside the list
        outside = 0.02 + 0.28 * torch.rand(rows, generator=g, device="cuda")
        known = (teacher.float() / case["temperature"]).masked_fill(index < 0, float("-inf"))
        state["lse"] = torch.logsumexp(known, 1).nan_to_num(neginf=0.0) - torch.log1p(-outside)
    if case["labels"]:         # the right token where it is known
        state["labels"] = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.1, -100,
                                      torch.randint(0, vocab, (rows,), generator=g, device="cuda")).to(torch.int32)
    return state


# ---- one pass --------------------------------------------------------------------------------------------
_SOFT, _HARD = 0.7, 0.3        # shares of the two parts of the loss where there are labels


def run(state):
    case = state["case"]
    op = case["op"]
    dtype = getattr(torch, case["dtype"])
    if op == "quantize":
        return _run_quantize(state["x"], case["both"], dtype)
    if op == "linear":
        return _run_linear(state["x"], state["w"], dtype)
    if op == "train":
        return _run_train(state["x"], state["w"], state["dy"], dtype)
    return _run_distill(state, op == "distill_grad")


def _run_quantize(x, both, dtype):
    if own:
        from paper_2202_06009_b200 import mx4_quantize, mx4_quantize_both
        if not both:
            return {"values": mx4_quantize(x).dequantize(dtype)}
        rows, cols = mx4_quantize_both(x)
        return {"values": rows.dequantize(dtype), "values_t": cols.dequantize(dtype)}
    out = {"values": _on_grid(x.float()).to(dtype)}
    if both:
        out["values_t"] = _on_grid(x.float().t()).to(dtype)
    return out


def _run_linear(x, w, dtype):
    if own:
        from paper_2202_06009_b200 import mx4_linear
        return {"y": mx4_linear(x, w)}
    return {"y": (_on_grid(x.float()) @ w.float().t()).to(dtype)}


def _run_train(x, w, dy, dtype):
    if own:
        from paper_2202_06009_b200 import mx4_linear_backward, mx4_linear_forward
        y, saved = mx4_linear_forward(x, w)
        dx, dw = mx4_linear_backward(dy, saved)
        return {"y": y, "dx": dx, "dw": dw}
    x, w, dy = x.float(), w.float(), dy.float()
    y = _on_grid(x) @ _on_grid(w).t()
    dx = _on_grid(dy) @ _on_grid(w.t()).t()
    dw = _on_grid(dy.t()) @ _on_grid(x.t()).t()
    return {"y": y.to(dtype), "dx": dx.to(dtype), "dw": dw.to(dtype)}


def _run_distill(state, grad):
    case = state["case"]
    soft, hard = (_SOFT, _HARD) if case["labels"] else (1.0, 0.0)
    if own:
        from paper_2202_06009_b200 import distill_topk, distill_topk_grad
        call = distill_topk_grad if grad else distill_topk
        out = call(state["logits"], state["index"], state["teacher"], labels=state["labels"], row_weight=state["weight"],
                   teacher_lse=state["lse"], temperature=case["temperature"], soft_weight=soft, hard_weight=hard)
        return {"loss": out[0], "grad": out[1]} if grad else {"loss": out}
    return _plain_distill(state, soft, hard, grad)


# ---- plain forms -----------------------------------------------------------------------------------------
def _on_grid(x):
    """x (32-bit, [rows, cols]) rounded to 4-bit microscaled form along its rows, as the values that this stands for.

    A block is 32 neighbours of a row.  Its scale is 2^(floor(log2 max|x|) - 2), at least 2^-127; its elements are
    rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale (ties to the even code), 6 being the most.
    A block that holds a NaN or an infinity is NaN."""
    rows, cols = x.shape
    blocks = torch.nn.functional.pad(x, (0, -cols % 32)).reshape(rows, -1, 32)
    most = blocks.abs().amax(2, keepdim=True)
    # most / mantissa is a power of two without rounding, the one above `most`; an eighth of it is the scale.
    scale = torch.where(most > 0, most / torch.frexp(most).mantissa * 0.125, 0.0).clamp(min=2.0 ** -127)
    size = blocks.abs() / scale
    code = ((size > 0.25).to(torch.int8) + (size >= 0.75) + (size > 1.25) + (size >= 1.75) + (size > 2.5) + (size >= 3.5)
            + (size > 5.0))
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=x.device)
    values = torch.copysign(grid[code.int()] * scale, blocks)
    values = torch.where(torch.isfinite(most), values, float("nan"))
    return values.reshape(rows, -1)[:, :cols]


def _plain_distill(state, soft, hard, grad):
    case = state["case"]
    z, index, temperature = state["logits"].float(), state["index"].long(), case["temperature"]
    listed_ = index >= 0
    at = index.clamp(min=0)
    some = listed_.any(1)
    t = (state["teacher"].float() / temperature).masked_fill(~listed_, float("-inf"))
    most = z.amax(1, keepdim=True)
    e = torch.exp((z - most) / temperature)
    total = e.sum(1, keepdim=True)
    log_q = (z.gather(1, at) - most) / temperature - torch.log(total)
    if state["lse"] is None:
        high = t.amax(1, keepdim=True).clamp(min=-3e38)
        log_p = t - high - torch.log(torch.exp(t - high).sum(1, keepdim=True))
    else:
        log_p = t - state["lse"][:, None]
    p = torch.where(listed_, torch.exp(log_p), 0.0)
    loss = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
    weight = state["weight"]
    if state["lse"] is not None:
        outside = torch.ones_like(z, dtype=torch.bool)
        rows, columns = listed_.nonzero(as_tuple=True)
        outside[rows, at[rows, columns]] = False
        rest = torch.where(outside, e, 0.0).sum(1)
        p_rest = (1.0 - p.sum(1)).clamp(min=0.0)
        loss = loss + torch.where(p_rest > 0, p_rest * (torch.log(p_rest) - torch.log(rest / total[:, 0])), 0.0)
    loss = torch.where(some, loss, 0.0) * soft * temperature ** 2
    if state["labels"] is not None:
        labels = state["labels"].long()
        known = labels >= 0
        y = labels.clamp(min=0)[:, None]
        e1 = torch.exp(z - most)
        total1 = e1.sum(1, keepdim=True)
        loss = loss + hard * torch.where(known, (torch.log(total1) + most - z.gather(1, y))[:, 0], 0.0)
    loss = loss * weight
    if not grad:
        return {"loss": loss}
    d = e / total
    if state["lse"] is not None:
        d = d - torch.where(outside, e * (p_rest / rest)[:, None], 0.0)
    d.scatter_add_(1, at, -p)
    d = torch.where(some[:, None], d, 0.0) * (soft * temperature)
    if state["labels"] is not None:
        d1 = e1 / total1
        d1.scatter_add_(1, y, torch.full_like(total1, -1.0))
        d = d + hard * torch.where(known[:, None], d1, 0.0)
    return {"loss": loss, "grad": (d * weight[:, None]).to(state["logits"].dtype)}


# ---- the definitions in 64 bits --------------------------------------------------------------------------
def _round64(x):
    """The 4-bit form of x along its rows in 64 bits: the step between neighbours is 1/2, 1 or 2 times the scale."""
    rows, cols = x.shape
    out = torch.zeros(rows, -(-cols // 32) * 32, dtype=torch.float64, device=x.device)
    out[:, :cols] = x.double()
    out = out.reshape(-1, 32)
    most = out.abs().max(1, keepdim=True).values
    powers = torch.tensor([2.0 ** k for k in range(-125, 129)], dtype=torch.float64, device=x.device)
    scale = powers[(torch.searchsorted(powers, most, right=True) - 1).clamp(min=0)] / 4
    out = out / scale
    size = out.abs()
    step = 0.5 + 0.5 * (size >= 2) + 1.0 * (size >= 4)
    out = (torch.round(out / step) * step).clamp(-6.0, 6.0) * scale
    return out.reshape(rows, -1)[:, :cols]


def exact(case, seed):
    state = _exact_inputs(case, seed)
    op = case["op"]
    if op == "quantize":
        out = {"values": _round64(state["x"])}
        if case["both"]:
            out["values_t"] = _round64(state["x"].t())
        return out
    if op == "linear":
        return {"y": _round64(state["x"]) @ state["w"].double().t()}
    if op == "train":
        x, w, dy = state["x"], state["w"], state["dy"]
        return {"y": _round64(x) @ _round64(w).t(), "dx": _round64(dy) @ _round64(w.t()).t(),
                "dw": _round64(dy.t()) @ _round64(x.t()).t()}
    return _exact_distill(state, op == "distill_grad")


def _exact_inputs(case, seed):
    global own
    kept, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = kept


def _exact_distill(state, grad):
    """The loss as written, its gradient term by term, one row group at a time."""
    case = state["case"]
    temp = case["temperature"]
    soft, hard = (_SOFT, _HARD) if case["labels"] else (1.0, 0.0)
    losses, grads = [], []
    for first in range(0, case["rows"], 1024):
        part = slice(first, first + 1024)
        z = state["logits"][part].double()
        n = z.shape[0]
        log_q, log_q1 = torch.log_softmax(z / temp, 1), torch.log_softmax(z, 1)
        # The teacher's probabilities laid out over the vocabulary; a spare last column takes the missing entries.
        index = state["index"][part].long()
        missing = index < 0
        index = torch.where(missing, case["vocab"], index)
        t = (state["teacher"][part].double() / temp).masked_fill(missing, -math.inf)
        norm = torch.logsumexp(t, 1) if state["lse"] is None else state["lse"][part].double()
        any_ = (~missing).any(1)
        p = torch.zeros(n, case["vocab"] + 1, dtype=torch.float64, device=z.device)
        p.scatter_(1, index, torch.exp(t - norm[:, None]).nan_to_num(0.0))
        p = p[:, :-1]
        inside = torch.zeros(n, case["vocab"] + 1, dtype=torch.bool, device=z.device)
        inside.scatter_(1, index, True)
        inside = inside[:, :-1]
        loss = (torch.special.xlogy(p, p) - p * log_q).sum(1)
        q = torch.exp(log_q)
        d = q - p
        if state["lse"] is not None:
            p_rest = 1.0 - p.sum(1)
            q_rest = q.masked_fill(inside, 0.0).sum(1)
            loss = loss + p_rest * torch.log(p_rest / q_rest)
            d = d - (q * (p_rest / q_rest)[:, None]).masked_fill(inside, 0.0)
        loss = soft * temp ** 2 * loss.masked_fill(~any_, 0.0)
        d = soft * temp * d.masked_fill(~any_[:, None], 0.0)
        if state["labels"] is not None:
            y = state["labels"][part].long()
            at = torch.arange(n, device=z.device)[y >= 0]
            loss[at] -= hard * log_q1[at, y[at]]
            d[at] += hard * torch.exp(log_q1[at])
            d[at, y[at]] -= hard
        weight = state["weight"][part].double()
        losses.append(loss * weight)
        if grad:
            grads.append(d * weight[:, None])
    out = {"loss": torch.cat(losses)}
    if grad:
        out["grad"] = torch.cat(grads)
    return out
