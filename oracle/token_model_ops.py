"""Definitions of the operators of a token model's input side and inner layers in numpy float64: the layer norm with the residual's addition and its gradient, the lookup of
embeddings and the gradient of their table, the Newton-Schulz steps that orthogonalise a matrix and the optimizer's step around them.  Shares no code with the GPU
path; test infrastructure only."""
import numpy as np


# ---- layer norm ----

def layernorm(x, residual, gamma, beta, eps, store=lambda v: v):
    """(total, mean, rstd, n, y) with y unrounded; `store` is the rounding total goes through."""
    h = np.asarray(x, np.float64) if residual is None else store(np.asarray(x, np.float64) + np.asarray(residual, np.float64))
    mean = np.mean(h, axis=1)
    d = h - mean[:, None]
    rstd = 1.0 / np.sqrt(np.mean(d * d, axis=1) + eps)
    n = d * rstd[:, None]
    return h, mean, rstd, n, n * np.asarray(gamma, np.float64) + (0.0 if beta is None else np.asarray(beta, np.float64))


def layernorm_bwd(h, mean, rstd, gamma, dy, dtotal=None):
    """(dx, dgamma, dbeta) for the mean and rstd given."""
    h, dy = np.asarray(h, np.float64), np.asarray(dy, np.float64)
    n = (h - mean[:, None]) * rstd[:, None]
    a = dy * gamma
    dx = rstd[:, None] * (a - np.mean(a, axis=1, keepdims=True) - n * np.mean(a * n, axis=1, keepdims=True))
    return dx if dtotal is None else dx + dtotal, np.sum(dy * n, axis=0), np.sum(dy, axis=0)


# ---- embeddings ----

def embedding(table, tokens, scale):
    """scale * the tokens' rows; zeros for a token outside the table."""
    table = np.asarray(table, np.float64)
    there = (tokens >= 0) & (tokens < len(table))
    return np.where(there[:, None], scale * table[np.clip(tokens, 0, len(table) - 1)], 0.0)


def embedding_bwd(vocab, tokens, dout, scale, before=None):
    """(gradient of the table, the same of magnitudes, tokens' counts)."""
    dout = np.asarray(dout, np.float64)
    sums = [np.zeros((vocab, dout.shape[1])) if before is None else np.array(before, np.float64), np.zeros((vocab, dout.shape[1]))]
    there = (tokens >= 0) & (tokens < vocab)
    np.add.at(sums[0], tokens[there], scale * dout[there])
    np.add.at(sums[1], tokens[there], abs(scale) * np.abs(dout[there]))
    return sums[0], sums[1], np.bincount(tokens[there], minlength=vocab)


# ---- Newton-Schulz steps ----

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def newton_schulz(x, iterations=5, eps=1e-7):
    """A matrix divided by its norm (and eps), its singular values then taken through the polynomial `iterations` times."""
    x = np.asarray(x, np.float64)
    x = x / (np.sqrt(np.sum(x * x)) + eps) if np.any(x) else x
    a, b, c = COEFFICIENTS
    u, s, vt = np.linalg.svd(x, full_matrices=False)
    for _ in range(iterations):
        s = a * s + b * s ** 3 + c * s ** 5
    return (u * s) @ vt


def muon(w, g, m, lr, momentum, decay, nesterov=True, iterations=5, eps=1e-7, grad_scale=1.0, scale=None):
    """(w, m) after one step of a matrix."""
    w, g, m = (np.asarray(v, np.float64) for v in (w, g, m))
    g = g * grad_scale
    m = momentum * m + g
    rows, cols = w.shape
    factor = np.sqrt(max(1.0, rows / cols)) if scale is None else scale
    return w - lr * decay * w - lr * factor * newton_schulz(g + momentum * m if nesterov else m, iterations, eps), m
