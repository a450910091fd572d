"""Plain NumPy statement, in 64 bits, of the operators of language models: microscaled quantisation, the root-mean-square
norm with its gradients, log probabilities with entropies, alternatives and gradient.  Written from their definitions; shares
nothing with the library."""
import numpy as np

LARGEST = {"e4m3": 448.0, "e2m1": 6.0}


def round_to(x, dtype):
    """Round float64 values to the nearest number of a dtype name (ties to even), as float64."""
    x = np.asarray(x, np.float64)
    if dtype == "f64":
        return x
    if dtype == "f32":
        return x.astype(np.float32).astype(np.float64)
    if dtype == "f16":
        return x.astype(np.float16).astype(np.float64)
    bits, lowest, largest = 7, -126, 3.3895313892515355e38          # bf16
    out = _round_bits(x, bits, lowest)
    return np.where(np.abs(out) > largest, np.copysign(np.inf, out), out)


def _round_bits(v, bits, lowest):
    """To `bits` bits of fraction, exponents from `lowest` up (below: steps of the smallest one)."""
    with np.errstate(all="ignore"):
        _, e = np.frexp(v)                                   # |v| in [2^(e-1), 2^e)
        step = np.ldexp(1.0, np.maximum(e - 1, lowest) - bits)
        out = np.rint(v / step) * step
    return np.where(np.isfinite(v) & (v != 0), out, v)


def mx_blocks(x, fmt):
    """(codes' values, scales) of x by rows: arrays rows x blocks x 32 and rows x blocks; NaN scale where a block is not finite."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    v = np.zeros((rows, -(-cols // 32) * 32))
    v[:, :cols] = x
    v = v.reshape(rows, -1, 32)
    big = np.abs(v).max(axis=2)
    finite = np.isfinite(big)
    with np.errstate(all="ignore"):
        fraction, e = np.frexp(np.where(finite, big, 1.0) / LARGEST[fmt])       # ratio = fraction * 2^e, fraction in [0.5, 1)
    e = np.where(fraction == 0.5, e - 1, e)                  # smallest power of two that the ratio does not pass
    e = np.where(big == 0, -127, np.clip(e, -127, 127))
    scale = np.ldexp(1.0, e)
    t = np.where(finite[..., None], v / scale[..., None], 0.0)
    codes = _round_bits(t, 3, -6) if fmt == "e4m3" else _round_bits(t, 1, 0)
    return codes, np.where(finite, scale, np.nan)


def mx_values(x, fmt):
    """The numbers that the quantised rows of x stand for."""
    codes, scale = mx_blocks(x, fmt)
    rows, cols = np.shape(x)
    return (codes * scale[..., None]).reshape(rows, -1)[:, :cols]


def rms_norm(x, residual, weight, eps, dtype):
    """(y, h, rstd): h is rounded to dtype, y is not rounded."""
    x = np.asarray(x, np.float64)
    h = x if residual is None else round_to(x + np.asarray(residual, np.float64), dtype)
    rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    return h * rstd[:, None] * np.asarray(weight, np.float64), h, rstd


def rms_norm_backward(dy, dh, h, weight, rstd):
    """(dx, dweight), unrounded."""
    dy, h, weight = (np.asarray(a, np.float64) for a in (dy, h, weight))
    n = h * rstd[:, None]
    g = dy * weight
    dx = rstd[:, None] * (g - n * (g * n).mean(axis=1, keepdims=True))
    if dh is not None:
        dx = dx + np.asarray(dh, np.float64)
    return dx, (dy * n).sum(axis=0)


def token_logprobs(logits, targets, top):
    """(logprobs, entropy, top log probabilities, top indices); rows of nothing but -inf as documented."""
    x = np.asarray(logits, np.float64)
    rows, vocab = x.shape
    with np.errstate(all="ignore"):
        m = x.max(axis=1)
        empty = np.isneginf(m)
        base = np.where(empty, 0.0, m)
        e = np.exp(x - base[:, None])
        s = e.sum(axis=1)
        logp = (x - base[:, None]) - np.log(np.where(empty, 1.0, s))[:, None]
        p = np.exp(logp)
        entropy = -np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, logp)).sum(axis=1)
    entropy = np.where(empty, 0.0, entropy)
    logp = np.where(empty[:, None], -np.inf, logp)
    lp = np.zeros(rows)
    for i, t in enumerate(np.asarray(targets)):
        lp[i] = 0.0 if t < 0 else np.nan if t >= vocab else logp[i, t]
    # a NaN above all, then by value, equal ones by index
    order = np.argsort(np.where(np.isnan(x), -np.inf, -x) - 0.0, axis=1, kind="stable")
    nan_first = np.argsort(~np.take_along_axis(np.isnan(x), order, 1), axis=1, kind="stable")
    order = np.take_along_axis(order, nan_first, 1)[:, :top]
    return lp, entropy, np.take_along_axis(logp, order, 1), order


def token_logprobs_backward(logits, targets, dlogprobs, dentropy):
    """dlogits, unrounded."""
    x = np.asarray(logits, np.float64)
    rows, vocab = x.shape
    out = np.zeros_like(x)
    for i in range(rows):
        t = int(targets[i])
        if not np.isneginf(x[i]).all():
            with np.errstate(all="ignore"):
                a = x[i] - x[i].max()
                logp = a - np.log(np.exp(a).sum())
                p = np.exp(logp)
                terms = np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, logp))
            h = -terms.sum()
            dl = 0.0 if t < 0 else np.nan if t >= vocab else dlogprobs[i]
            out[i] = -p * dl - dentropy[i] * (terms + p * h)
            if 0 <= t < vocab:
                out[i, t] += dl
    return out
