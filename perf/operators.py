"""The measured operators of language models: activations and weights held in microscaled 8- or 4-bit numbers, their
products, the root-mean-square norm that feeds them, and the log probabilities at the end.

A pass of a "pair" case quantises a matrix and reads it back (the cache of a linear layer: by rows for the forward
product, by columns too for the gradient of the weights).  A "product" case is a linear layer at inference, its weights
quantised once, its tokens at every call.  A "linear" case is the forward and backward pass of a linear layer whose three
products take quantised operands.  "norm" adds the residual, normalises and hands on 8-bit numbers; "norm_step" is the
training form with its gradients.  "logprobs" looks up given tokens, with entropies and the top alternatives;
"logprobs_step" adds the gradient of the logits.

The format: blocks of 32 neighbours along a row share a scale, the smallest power of two with which the block's largest
magnitude does not pass the largest number of the format (e4m3: 448, e2m1: 6), between 2^-127 and 2^127; values are
divided by it and rounded to nearest, ties to even.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
LARGEST = {"e4m3": 448.0, "e2m1": 6.0}
CODE_BYTES = {"e4m3": 1 + 1 / 32, "e2m1": 0.5 + 1 / 32}
EPS = 1e-5


def listed():
    return [
        # the tokens of one short request, to 8 bits and back: what the calls cost
        dict(name="pair_small", kind="pair", rows=64, cols=768, x="bf16", fmt="e4m3", both=False),
        # activations of a long batch, by rows and by columns from one reading: the cache of a training step
        dict(name="pair_large", kind="pair", rows=8192, cols=8192, x="bf16", fmt="e4m3", both=True),
        # one token through a square layer with 4-bit weights: the weights' bytes count
        dict(name="product_token", kind="product", rows=1, cols=4096, outs=4096, x="bf16", fmt="e2m1"),
        # a handful of ragged requests, sizes that end inside tiles
        dict(name="product_ragged", kind="product", rows=777, cols=2720, outs=5000, x="f16", fmt="e2m1"),
        # a long prompt through a wide layer, 4 bits
        dict(name="product_prompt", kind="product", rows=8192, cols=4096, outs=8192, x="bf16", fmt="e2m1"),
        # a training step of a linear layer in 8 bits: three products, four operands quantised, two of them twice
        dict(name="linear_step", kind="linear", rows=8192, cols=4096, outs=4096, x="bf16", fmt="e4m3"),
        # one token of a few sequences between two layers
        dict(name="norm_token", kind="norm", rows=4, cols=4096, x="bf16", fmt="e4m3", residual=True),
        # a prompt, odd number of rows, the last block of a row cut short
        dict(name="norm_prompt", kind="norm", rows=4099, cols=5000, x="f16", fmt="e4m3", residual=True),
        # the training form, with the gradients of input, residual and weight
        dict(name="norm_step", kind="norm_step", rows=16384, cols=4096, x="bf16", residual=True),
        # the next token of one sequence: one row over a large vocabulary, in full precision
        dict(name="logprobs_token", kind="logprobs", rows=1, vocab=131072, x="f32", top=20, masked=True),
        # scoring a prompt, odd vocabulary
        dict(name="logprobs_prompt", kind="logprobs", rows=2000, vocab=49157, x="bf16", top=5, masked=True),
        # the loss of a training step with its gradient
        dict(name="logprobs_step", kind="logprobs_step", rows=8192, vocab=65536, x="bf16", masked=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("pair", "product", "product", "linear", "norm", "norm_step", "logprobs", "logprobs_step"))
    x = rng.choice(("bf16", "bf16", "f16") if kind in ("product", "linear") else ("bf16", "bf16", "f16", "f32"))
    fmt = rng.choice(("e4m3", "e2m1"))
    if kind == "pair":
        rows = _log_uniform(rng, 1, 8192)
        return dict(kind=kind, rows=rows, cols=_log_uniform(rng, 32, 8192), x=x, fmt=fmt, both=rng.random() < 0.5)
    if kind == "product":
        return dict(kind=kind, rows=_log_uniform(rng, 1, 8192), cols=_log_uniform(rng, 64, 4096), outs=_log_uniform(rng, 64, 8192), x=x, fmt=fmt)
    if kind == "linear":
        return dict(kind=kind, rows=_log_uniform(rng, 16, 8192), cols=_log_uniform(rng, 64, 4096), outs=_log_uniform(rng, 64, 4096), x=x, fmt=fmt)
    if kind == "norm":
        return dict(kind=kind, rows=_log_uniform(rng, 1, 4096), cols=_log_uniform(rng, 64, 8192), x=x, fmt="e4m3", residual=rng.random() < 0.7)
    if kind == "norm_step":
        return dict(kind=kind, rows=_log_uniform(rng, 8, 8192), cols=_log_uniform(rng, 64, 8192), x=x, residual=rng.random() < 0.7)
    rows, vocab = _log_uniform(rng, 1, 4096), _log_uniform(rng, 100, 131072)
    rows = max(1, min(rows, 200_000_000 // vocab))
    if kind == "logprobs":
        return dict(kind=kind, rows=rows, vocab=vocab, x=x, top=rng.randint(0, 20), masked=rng.random() < 0.5)
    return dict(kind=kind, rows=rows, vocab=vocab, x=x, masked=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------
def _tokens(g, rows, cols, dtype):
    """Activations: a scale per token and a few channels that stand out."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    x *= 1 + 7 * (torch.rand(1, cols, generator=g, device="cuda") < 0.01)
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    kind, dtype = case["kind"], TYPES[case["x"]]
    state = {"case": dict(case)}
    if kind in ("pair", "product", "linear", "norm", "norm_step"):
        rows, cols = case["rows"], case["cols"]
        state["x"] = _tokens(g, rows, cols, dtype)
        if kind in ("product", "linear"):
            w = torch.randn(case["outs"], cols, generator=g, device="cuda").mul_(cols ** -0.5).to(dtype)
            if kind == "linear":
                state["w"] = w
                state["dy"] = _tokens(g, rows, case["outs"], dtype) * 0.01
            else:
                state["w"] = _lm().mx_quantize(w, case["fmt"]) if own else _values(w, case["fmt"])      # laid out once
        if kind in ("norm", "norm_step"):
            state["w"] = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(dtype)
            state["residual"] = _tokens(g, rows, cols, dtype) if case["residual"] else None
        if kind == "norm_step":
            state["dy"] = torch.randn(rows, cols, generator=g, device="cuda").to(dtype)
            state["dh"] = torch.randn(rows, cols, generator=g, device="cuda").to(dtype) if case["residual"] else None
    else:
        rows, vocab = case["rows"], case["vocab"]
        x = torch.randn(rows, vocab, generator=g, device="cuda")
        x *= 1 + 2 * torch.rand(rows, 1, generator=g, device="cuda")
        if case["masked"]:                                      # a constrained vocabulary
            x.masked_fill_(torch.rand(rows, vocab, generator=g, device="cuda") < 0.2, -math.inf)
        state["x"] = x.to(dtype)
        del x
        state["targets"] = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        if case["masked"]:                                      # given tokens are allowed ones
            state["x"].scatter_(1, state["targets"][:, None], torch.randn(rows, 1, generator=g, device="cuda").to(dtype))
        if kind == "logprobs_step":
            state["dlogprobs"] = -torch.rand(rows, generator=g, device="cuda") / rows
            state["dentropy"] = 0.01 * torch.randn(rows, generator=g, device="cuda") / rows
    return state


# ------------------------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------------------------
def _values(x, fmt):
    """The numbers that the quantised rows of x stand for, in 32 bits."""
    rows, cols = x.shape
    pad = -cols % 32
    v = torch.nn.functional.pad(x.float(), (0, pad)).view(rows, -1, 32)
    mantissa, exponent = torch.frexp(v.abs().amax(2, keepdim=True) / LARGEST[fmt])
    exponent = (exponent - (mantissa == 0.5).int()).clamp(-127, 127)
    one = torch.ones_like(mantissa)
    v = v * torch.ldexp(one, -exponent)
    if fmt == "e4m3":
        v = v.to(torch.float8_e4m3fn).float()
    else:
        a = v.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        v = torch.copysign(torch.round(a / step) * step, v)
    return (v * torch.ldexp(one, exponent)).view(rows, cols + pad)[:, :cols]


def _norm(x, w, residual):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    f = h.float()
    rstd = torch.rsqrt(f.square().mean(1, keepdim=True) + EPS)
    return h, f * rstd, rstd


def _plain(s):
    case, kind, x = s["case"], s["case"]["kind"], s["x"]
    if kind == "pair":
        out = [_values(x, case["fmt"]).to(torch.bfloat16)]
        if case["both"]:
            out.append(_values(x.t(), case["fmt"]).to(torch.bfloat16))
        return out
    if kind == "product":
        return (_values(x, case["fmt"]) @ s["w"].t()).to(x.dtype)
    if kind == "linear":
        w, dy, fmt = s["w"], s["dy"], case["fmt"]
        y = _values(x, fmt) @ _values(w, fmt).t()
        dx = _values(dy, fmt) @ _values(w.t(), fmt).t()
        dw = _values(dy.t(), fmt) @ _values(x.t(), fmt).t()
        return y.to(x.dtype), dx.to(x.dtype), dw.to(w.dtype)
    if kind == "norm":
        h, n, _ = _norm(x, s["w"], s["residual"])
        return _values(n * s["w"].float(), case["fmt"]).to(torch.bfloat16), h
    if kind == "norm_step":
        h, n, rstd = _norm(x, s["w"], s["residual"])
        y = n * s["w"].float()
        dy = s["dy"].float()
        dn = dy * s["w"].float()
        dx = rstd * (dn - n * (dn * n).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return y.to(x.dtype), h, dx.to(x.dtype), (dy * n).sum(0).to(s["w"].dtype)
    f, t = x.float(), s["targets"][:, None]
    f = f - f.amax(1, keepdim=True)
    lse = torch.log(torch.exp(f).sum(1, keepdim=True))
    logp = f - lse
    p = torch.exp(logp)
    plogp = torch.where(p > 0, p * logp, 0.0)
    entropy = -plogp.sum(1)
    logprobs = logp.gather(1, t)[:, 0]
    if kind == "logprobs":
        order = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :case["top"]]
        return logprobs, entropy, logp.gather(1, order), order
    d = -p * s["dlogprobs"][:, None] - s["dentropy"][:, None] * (plogp + p * entropy[:, None])
    d.scatter_add_(1, t, s["dlogprobs"][:, None])
    return logprobs, entropy, d.to(x.dtype)


# ------------------------------------------------------------------------------------------------------------
# the framework's operators
# ------------------------------------------------------------------------------------------------------------
def _lm():
    from paper_2208_04187_b200 import language
    return language


def _own(s):
    lm = _lm()
    case, kind, x = s["case"], s["case"]["kind"], s["x"]
    if kind == "pair":
        got = lm.mx_quantize_both(x, case["fmt"]) if case["both"] else (lm.mx_quantize(x, case["fmt"]),)
        return [q.dequantize(torch.bfloat16) for q in got]
    if kind == "product":
        return lm.mx_matmul(lm.mx_quantize(x, case["fmt"]), s["w"], x.dtype)
    if kind == "linear":
        x, w = x.detach().requires_grad_(), s["w"].detach().requires_grad_()
        y = lm.mx_linear(x, w, fmt=case["fmt"])
        return (y, *torch.autograd.grad(y, (x, w), s["dy"]))
    if kind == "norm":
        q, h = lm.rms_norm_mx(x, s["w"], s["residual"], eps=EPS, fmt=case["fmt"])
        return q.dequantize(torch.bfloat16), h
    if kind == "norm_step":
        x, w = x.detach().requires_grad_(), s["w"].detach().requires_grad_()
        y, h = lm.rms_norm(x, w, s["residual"], eps=EPS)
        if s["dh"] is None:
            return (y, h, *torch.autograd.grad(y, (x, w), s["dy"]))
        return (y, h, *torch.autograd.grad((y, h), (x, w), (s["dy"], s["dh"])))
    if kind == "logprobs":
        return tuple(lm.token_logprobs(x, s["targets"], top=case["top"]))
    x = x.detach().requires_grad_()
    logprobs, entropy = lm.token_logprobs(x, s["targets"])[:2]
    return logprobs, entropy, torch.autograd.grad((logprobs, entropy), x, (s["dlogprobs"], s["dentropy"]))[0]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------------------
# the least work
# ------------------------------------------------------------------------------------------------------------
def work(case):
    kind, b = case["kind"], BYTES[case["x"]]
    if kind in ("logprobs", "logprobs_step"):
        n = case["rows"] * case["vocab"]
        if kind == "logprobs":
            return {"bytes": n * b + case["rows"] * (16 + 12 * case["top"]), "flops": 5 * n}
        return {"bytes": 3 * n * b + 24 * case["rows"], "flops": 11 * n}      # the gradient needs the whole row's sum first: read twice
    rows, cols = case["rows"], case["cols"]
    n = rows * cols
    if kind == "pair":
        times = 2 if case["both"] else 1
        return {"bytes": n * b + times * n * (2 * CODE_BYTES[case["fmt"]] + 2), "flops": 6 * n * times}
    if kind in ("product", "linear"):
        outs, c = case["outs"], CODE_BYTES[case["fmt"]]
        if kind == "product":
            return {"bytes": n * b + outs * cols * c + rows * outs * b, "flops": 2 * n * outs}
        # x, w and dy read, y, dx and dw written; the columns' codes of x, w and dy outlive the pass that makes them
        return {"bytes": 2 * b * (n + outs * cols + rows * outs) + 2 * c * n, "flops": 6 * n * outs}
    if kind == "norm":
        return {"bytes": n * b * (3 if case["residual"] else 1) + n * (2 * CODE_BYTES[case["fmt"]] + 2), "flops": 10 * n}
    # forward: x, residual, y, h; backward: dy, dh, h, dx
    return {"bytes": n * b * (8 if case["residual"] else 5), "flops": 14 * n}


# ------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------------------
def _values64(x, fmt):
    rows, cols = x.shape
    x = x.double()
    blocks = torch.zeros(rows, -(-cols // 32) * 32, dtype=torch.float64, device=x.device)
    blocks[:, :cols] = x
    blocks = blocks.unflatten(1, (-1, 32))
    largest = blocks.abs().max(dim=2, keepdim=True).values
    scale = torch.exp2(torch.ceil(torch.log2(largest / LARGEST[fmt])).clamp(-127, 127))
    scale = torch.where(largest > scale * LARGEST[fmt], scale * 2, scale)             # (a logarithm that came out a little low or high)
    scale = torch.where((largest <= scale / 2 * LARGEST[fmt]) & (scale > 2.0 ** -127), scale / 2, scale)
    v = blocks / scale
    bits, lowest = (3, -6) if fmt == "e4m3" else (1, 0)
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** lowest))) - bits)
    return (torch.round(v / step) * step * scale).flatten(1)[:, :cols]


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    kind, x = case["kind"], s["x"].double()
    if kind == "pair":
        out = [_values64(x, case["fmt"])]
        if case["both"]:
            out.append(_values64(x.t(), case["fmt"]))
        return out
    if kind == "product":
        return _values64(x, case["fmt"]) @ s["w"].double().t()      # (the weights' plain form is exact)
    if kind == "linear":
        w, dy, fmt = s["w"].double(), s["dy"].double(), case["fmt"]
        return (_values64(x, fmt) @ _values64(w, fmt).t(), _values64(dy, fmt) @ _values64(w.t(), fmt).t(),
                _values64(dy.t(), fmt) @ _values64(x.t(), fmt).t())
    if kind in ("norm", "norm_step"):
        w = s["w"].double()
        whole = x if s["residual"] is None else x + s["residual"].double()
        h = whole.to(s["x"].dtype).double()                          # what is handed on is what is normalised
        rms = torch.sqrt((h * h).sum(1) / h.shape[1] + EPS)[:, None]
        if kind == "norm":
            return _values64(h / rms * w, case["fmt"]), whole
        g = s["dy"].double() * w
        dx = g / rms - h * ((g * h).sum(1, keepdim=True) / (h.shape[1] * rms ** 3))
        if s["dh"] is not None:
            dx += s["dh"].double()
        return h / rms * w, whole, dx, (s["dy"].double() * h / rms).sum(0)
    lse = torch.logsumexp(x, 1)
    logp = x - lse[:, None]
    p = torch.exp(logp)
    terms = torch.xlogy(p, p)
    entropy = -terms.sum(1)
    target = logp[torch.arange(len(x), device=x.device), s["targets"]]
    if kind == "logprobs":
        return target, entropy, torch.sort(logp, dim=1, descending=True)[0][:, :case["top"]], None
    d = -(p * s["dlogprobs"].double()[:, None]) - s["dentropy"].double()[:, None] * (terms + p * entropy[:, None])
    d[torch.arange(len(x), device=x.device), s["targets"]] += s["dlogprobs"].double()
    return target, entropy, d
