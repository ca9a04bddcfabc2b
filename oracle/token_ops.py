"""Definitions of the operators of a token model's output side in numpy float64: the RMS norm with the residual's addition, its 8-bit
output and its gradient; the log probabilities of given tokens with entropy, top alternatives and gradient; the AdamW step with states
in 32 bits or in 8.  Shares no code with the GPU path; test infrastructure only."""
import numpy as np


# ---- small floating-point formats ----

def grid_step(x, mantissa, least):
    """The distance of neighbours around x of a format with `mantissa` bits whose least normal exponent is `least`."""
    e = np.frexp(np.abs(x))[1] - 1
    return np.exp2(np.maximum(e, least).astype(np.float64) - mantissa)


def round_to(x, mantissa, least):
    """Nearest value of the format, ties to even (np.rint), no upper limit."""
    x = np.asarray(x, dtype=np.float64)
    step = grid_step(x, mantissa, least)
    return np.rint(x / step) * step


def e4m3(x):
    """Values of e4m3 (largest 448, least 2^-9); the caller keeps |x| at most 448 but for rounding."""
    return round_to(x, 3, -6)


def bf16(x):
    return round_to(np.asarray(x, dtype=np.float64), 7, -126)


def dither21(index, seed):
    """21 bits for element `index` of a tensor: two rounds of shift and odd product modulo 2^32 (the golden ratio's and root two's bits)."""
    m = (1 << 32) - 1
    u = [(int(i) + seed * 0x9E3779B1 + 0x7F4A7C15) & m for i in np.ravel(index)]
    u = [((v ^ (v >> 16)) * 0x9E3779B1) & m for v in u]
    u = [((v ^ (v >> 15)) * 0x6A09E667) & m for v in u]
    return np.array([v >> 11 for v in u], dtype=np.float64).reshape(np.shape(index))


def e5m2_dithered(x, bits):
    """x >= 0 on the grid of e5m2: up where the dropped part of a step and the dither, bits / 2^21, come to one; never from above zero to zero."""
    step = grid_step(x, 2, -14)
    q = np.floor(x / step + bits / 2.0 ** 21) * step
    return np.where(x > 0, np.maximum(q, 2.0 ** -16), 0.0)


def power_scale(amax, most):
    """The smallest power of two s >= 2^-126 with amax / s <= most; 1 for amax = 0."""
    if amax == 0:
        return 1.0
    f, e = np.frexp(amax / most)
    return float(2.0 ** max(-126, e - 1 if f == 0.5 else e))


# ---- RMS norm ----

def rmsnorm(x, residual, gamma, eps, store=lambda v: v):
    """(total, rstd, y) with y unrounded; `store` is the rounding total goes through."""
    h = np.asarray(x, np.float64) if residual is None else store(np.asarray(x, np.float64) + np.asarray(residual, np.float64))
    rstd = 1.0 / np.sqrt(np.mean(h * h, axis=1) + eps)
    return h, rstd, h * rstd[:, None] * np.asarray(gamma, np.float64)


def quantise_rows(y, group):
    """(values of the codes, scales): scale = max(amax/448, 2^-126) for each group of columns."""
    rows, c = y.shape
    w = group or c
    q, scales = np.zeros_like(y), np.zeros((rows, -(-c // w)))
    for j, at in enumerate(range(0, c, w)):
        part = y[:, at:at + w]
        scales[:, j] = np.maximum(np.max(np.abs(part), axis=1) / 448.0, 2.0 ** -126)
        q[:, at:at + w] = e4m3(part / scales[:, j:j + 1])
    return q, scales


def rmsnorm_bwd(h, rstd, gamma, dy, dtotal=None):
    h, dy = np.asarray(h, np.float64), np.asarray(dy, np.float64)
    n = h * rstd[:, None]
    a = dy * gamma
    dx = rstd[:, None] * (a - n * np.mean(a * n, axis=1, keepdims=True))
    return dx if dtotal is None else dx + dtotal, np.sum(dy * n, axis=0)


# ---- log probabilities of given tokens ----

def token_logprob(z, tokens, top=0):
    """(logprob, entropy, lse, top tokens, top log probabilities); masked logits are -inf, a token outside the vocabulary does not count."""
    z = np.asarray(z, np.float64)
    rows, k = z.shape
    m = z.max(axis=1)
    empty = m == -np.inf
    from_ = np.where(empty, 0.0, m)
    e = np.exp(z - from_[:, None])
    with np.errstate(divide="ignore", invalid="ignore"):
        log_s = np.log(e.sum(axis=1))
        logp = np.where(empty[:, None], -np.inf, z - from_[:, None] - log_s[:, None])
    p = np.where(empty[:, None], 0.0, np.exp(logp))
    entropy = -np.sum(p * np.where(p > 0, logp, 0.0), axis=1)
    lse = np.where(empty, -np.inf, from_ + log_s)
    counts = (tokens >= 0) & (tokens < k)
    logprob = np.where(counts, logp[np.arange(rows), np.clip(tokens, 0, k - 1)], 0.0)
    order = np.argsort(-z, axis=1, kind="stable")[:, :top]
    ids, lp = np.full((rows, top), -1, np.int64), np.full((rows, top), -np.inf)
    n = order.shape[1]
    there = np.take_along_axis(z, order, 1) > -np.inf
    ids[:, :n] = np.where(there, order, -1)
    lp[:, :n] = np.where(there, np.take_along_axis(logp, order, 1), -np.inf)
    return logprob, entropy, lse, ids, lp


def token_logprob_bwd(z, tokens, dlogprob, dentropy):
    z = np.asarray(z, np.float64)
    rows, k = z.shape
    _, entropy, lse, _, _ = token_logprob(z, tokens)
    empty = lse == -np.inf
    logp = z - np.where(empty, 0.0, lse)[:, None]
    p = np.exp(logp)
    hot = np.zeros_like(z)
    counts = (tokens >= 0) & (tokens < k)
    hot[np.arange(rows)[counts], tokens[counts]] = 1.0
    a = np.where(counts, dlogprob, 0.0)[:, None]
    dz = a * (hot - p) - dentropy[:, None] * p * (np.where(p > 0, logp, 0.0) + entropy[:, None])
    return np.where(empty[:, None], 0.0, dz)


# ---- AdamW ----

def adamw(w, g, m, v, lr, beta1, beta2, eps, decay, step, scale=1.0):
    """(w, m, v) after one step, float64."""
    w, g, m, v = (np.asarray(a, np.float64) for a in (w, g, m, v))
    g = g * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    update = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return w - lr * decay * w - lr * update, m, v


def adam_states_as_rounded(g, m, v, beta1, beta2, scale=1.0):
    """m and v with every product and sum rounded to fp32 by itself, as the step defines them."""
    f = np.float32
    g, m, v = (np.asarray(a, f) for a in (g, m, v))
    x = g * f(scale)
    return f(beta1) * m + f(1 - beta1) * x, f(beta2) * v + f(1 - beta2) * (x * x)


def states_in_8_bits(m, v, seed, block=256):
    """((values of m's codes, scales), (values of v's codes, scales)) of one tensor."""
    m, v = np.asarray(m, np.float64), np.asarray(v, np.float64)
    out = []
    bits = dither21(np.arange(m.size), seed)
    for x, most, code in ((m, 448.0, lambda x, b: e4m3(x)), (v, 57344.0, e5m2_dithered)):
        scales = np.array([power_scale(np.max(np.abs(x[i:i + block])), most) for i in range(0, x.size, block)])
        wide = np.repeat(scales, block)[:x.size]
        out.append((code(x / wide, bits), scales))
    return out
