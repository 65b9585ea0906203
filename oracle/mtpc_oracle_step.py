"""fp64 CPU oracle of what a training step does beside the head: byte embeddings, the residual norm, the gradients' norm. TEST
INFRASTRUCTURE, not a product path: plain numpy from the definitions in include/mtpc.h, sharing no code with the CUDA library.

Pins (tests/test_oracle_step.py): every gradient equals central finite differences of the forward functions; e4m3 values equal a table of all
of them; a clipped list has norm max_norm.
"""
from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0


def embed(tokens, table, scale):
    """Rows of the table; negative: zeros; no such row: NaN."""
    v, d = table.shape
    out = np.zeros((len(tokens), d))
    for t, b in enumerate(tokens):
        if b >= v:
            out[t] = np.nan
        elif b >= 0:
            out[t] = np.float64(scale) * table[b].astype(np.float64)
    return out


def embed_grad(tokens, d_out, scale, v, start=None):
    """(gradient, sum of the terms' magnitudes) per element."""
    d_out = d_out.astype(np.float64)
    grad, size = np.zeros((v, d_out.shape[1])), np.zeros((v, d_out.shape[1]))
    keep = (tokens >= 0) & (tokens < v)
    np.add.at(grad, tokens[keep], d_out[keep])
    np.add.at(size, tokens[keep], np.abs(d_out[keep]))
    grad, size = grad * scale, size * abs(scale)
    if start is not None:
        grad, size = grad + start, size + np.abs(start)
    return grad, size


def rmsnorm(x, residual, weight, eps):
    """(s, out)"""
    s = x.astype(np.float64) + (0.0 if residual is None else residual.astype(np.float64))
    rstd = 1.0 / np.sqrt((s * s).mean(1, keepdims=True) + np.float64(eps))
    return s, s * rstd * (1.0 if weight is None else weight.astype(np.float64))


def rmsnorm_grad(s, weight, eps, d_out, d_sum=None):
    """(d_s, d_weight, magnitudes of d_s's terms, magnitudes of d_weight's terms)"""
    s, dy = s.astype(np.float64), d_out.astype(np.float64)
    w = np.ones(s.shape[1]) if weight is None else weight.astype(np.float64)
    d = s.shape[1]
    rstd = 1.0 / np.sqrt((s * s).mean(1, keepdims=True) + np.float64(eps))
    unit, up = s * rstd, dy * w
    dx = rstd * (up - unit * (up * unit).sum(1, keepdims=True) / d)
    size = rstd * (np.abs(up) + np.abs(unit) * np.abs(up * unit).sum(1, keepdims=True) / d)
    if d_sum is not None:
        dx = dx + d_sum
        size = size + np.abs(d_sum)
    return dx, (dy * unit).sum(0), size, np.abs(dy * unit).sum(0)


def e4m3(x):
    """Nearest value of four exponent and three mantissa bits (ties to even, steps of 2^-9 below 2^-6), at most 448 in magnitude."""
    x = np.asarray(x, dtype=np.float64)
    _, exponent = np.frexp(x)
    step = np.exp2(np.maximum(exponent - 1, -6) - 3.0)
    return np.clip(np.rint(x / step) * step, -E4M3_MAX, E4M3_MAX)


def in_groups(y, group):
    """[T, d] -> [T, groups, columns], zeros behind a short last group; group 0: the row."""
    group = group or y.shape[1]
    return np.pad(y, ((0, 0), (0, -y.shape[1] % group))).reshape(y.shape[0], -1, group)


def code_scales(y, group):
    largest = np.abs(in_groups(y, group)).max(2)
    return np.where(largest == 0, 1.0, largest / E4M3_MAX)


def clip(grads, max_norm):
    """(norm, scaled gradients)"""
    norm = np.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads))
    by = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return norm, [g.astype(np.float64) * by for g in grads]
