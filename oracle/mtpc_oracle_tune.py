"""fp64 CPU oracle of what fits a model to tasks beside its head: adaptors beside a projection, dropout, and the policy and preference losses. TEST INFRASTRUCTURE, not a
product path: plain numpy from the definitions in include/mtpc.h, position by position, sharing no code with the CUDA library.

Pins (tests/test_oracle_tune.py): Philox4x32-10 equals the published known answers; every gradient equals central finite differences of its loss.
"""
from __future__ import annotations

import math

import numpy as np

MASK32 = 0xFFFFFFFF


def philox4x32(counter, key, rounds=10):
    """Salmon et al. 2011: four 32-bit words of a counter of four under a key of two."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & MASK32, (a >> 32) ^ c[3] ^ k[1], a & MASK32]
        k = [(k[0] + 0x9E3779B9) & MASK32, (k[1] + 0xBB67AE85) & MASK32]
    return c


def dropout_cut(p):
    return min(65535, int(math.floor(float(np.float32(p)) * 65536 + 0.5)))


def dropout_kept(T, d, p, seed, step):
    """Which elements of a [T, d] matrix are kept."""
    draws = []
    for block in range(-(-T * d // 8)):
        words = philox4x32([block & MASK32, block >> 32, step & MASK32, (step >> 32) & MASK32], [seed & MASK32, (seed >> 32) & MASK32])
        draws += [part for w in words for part in (w & 0xFFFF, w >> 16)]
    return (np.array(draws[:T * d]) >= dropout_cut(p)).reshape(T, d)


def dropout(x, p, seed, step, residual=None):
    kept = dropout_kept(*x.shape, p, seed, step)
    y = np.where(kept, x.astype(np.float64) * (65536.0 / (65536 - dropout_cut(p))), 0.0)
    return y if residual is None else y + residual.astype(np.float64)


def policy_loss(logp, old, ref, advantage, offsets, clip_low, clip_high, beta, mask=None, by_sequence=False, by_position=False):
    """(loss, stats [3], gradient [T] with NaN outside of the sequences, sum of the weighted terms' magnitudes)"""
    S = len(offsets) - 1
    valid = np.ones(len(logp), bool) if mask is None else np.asarray(mask) != 0
    grad, stats, size = np.full(len(logp), np.nan), np.zeros(3), 0.0
    total = sum(int(valid[offsets[s]:offsets[s + 1]].sum()) for s in range(S))
    for s in range(S):
        here = int(valid[offsets[s]:offsets[s + 1]].sum())
        for t in range(offsets[s], offsets[s + 1]):
            grad[t] = 0.0
            if not valid[t]:
                continue
            w = 1.0 / (S * here) if by_sequence else 1.0 / total
            a = float(advantage[t] if by_position else advantage[s])
            r = math.exp(float(logp[t]) - float(old[t]))
            held = min(max(r, 1.0 - clip_low), 1.0 + clip_high)
            first = -min(r * a, held * a)
            clipped = held * a < r * a
            q = float(ref[t]) - float(logp[t]) if beta else 0.0
            kl = math.expm1(q) - q if q < math.inf else q
            stats += w * np.array([first, kl, float(clipped)])
            size += w * (abs(first) + beta * kl)
            grad[t] = w * ((0.0 if clipped else -r * a) - beta * math.expm1(q))
    return stats[0] + beta * stats[1], stats, grad, size


def preference_loss(logp, ref, offsets, beta, smoothing=0.0, mask=None):
    """(loss, h [S / 2], gradient [T] with NaN outside of the sequences)"""
    valid = np.ones(len(logp), bool) if mask is None else np.asarray(mask) != 0
    S = len(offsets) - 1
    ratio = []
    for s in range(S):
        at = [t for t in range(offsets[s], offsets[s + 1]) if valid[t]]
        ratio.append(math.fsum([float(logp[t]) for t in at] + [-float(ref[t]) for t in at]))
    grad, hs, loss = np.full(len(logp), np.nan), [], 0.0
    log_sigmoid = lambda x: -math.log1p(math.exp(-x)) if x > -30 else x - math.log1p(math.exp(x))  # noqa: E731
    of = lambda share, x: share * x if share else 0.0  # noqa: E731  (a factor of zero takes its term away, also one without a bound)
    for p in range(S // 2):
        h = of(beta, ratio[2 * p] - ratio[2 * p + 1])
        hs.append(h)
        loss -= (of(1 - smoothing, log_sigmoid(h)) + of(smoothing, log_sigmoid(-h))) / (S // 2)
        slope = beta * (smoothing - math.exp(log_sigmoid(-h))) / (S // 2)
        for s, sign in ((2 * p, 1), (2 * p + 1, -1)):
            for t in range(offsets[s], offsets[s + 1]):
                grad[t] = sign * slope if valid[t] else 0.0
    return loss, np.array(hs), grad


def adapted_projection(x, W, A, B, scale, which, x_low=None):
    """(out, low, sums of the magnitudes of out's terms [T, m], of low's [T, k]); which None: adaptor 0, negative: none, >= S: NaN"""
    f = lambda a: np.asarray(a, dtype=np.float64)  # noqa: E731
    x, W, A, B = f(x), f(W), f(A), f(B)
    x_low = x if x_low is None else f(x_low)
    S, _, k = A.shape
    out, size = x @ W.T, np.abs(x) @ np.abs(W).T
    low, low_size = np.zeros((len(x), k)), np.zeros((len(x), k))
    for t in range(len(x)):
        i = 0 if which is None else int(which[t])
        if i >= S:
            out[t], low[t] = np.nan, np.nan
        elif i >= 0:
            s = 1.0 if scale is None else float(scale[i])
            low[t], low_size[t] = s * (B[i] @ x_low[t]), abs(s) * (np.abs(B[i]) @ np.abs(x_low[t]))
            out[t] += A[i] @ low[t]
            size[t] += np.abs(A[i]) @ low_size[t]
    return out, low, size, low_size


def adapted_projection_grad(x_low, W, A, B, scale, which, low, d_out):
    """dict of d_x, d_x_low (its adaptors' part), dA, dB and, by the same names with _size, the sums of their terms' magnitudes"""
    f = lambda a: np.asarray(a, dtype=np.float64)  # noqa: E731
    x_low, W, A, B, low, g = f(x_low), f(W), f(A), f(B), f(low), f(d_out)
    S = len(A)
    base, base_size = g @ W, np.abs(g) @ np.abs(W)
    part, part_size = np.zeros_like(base), np.zeros_like(base)
    r = {key: np.zeros_like(v) for key, v in (("dA", A), ("dA_size", A), ("dB", B), ("dB_size", B))}
    for t in range(len(g)):
        i = 0 if which is None else int(which[t])
        if i >= S:
            base[t], part[t] = np.nan, np.nan
        elif i >= 0:
            s = 1.0 if scale is None else float(scale[i])
            v, v_size = s * (A[i].T @ g[t]), abs(s) * (np.abs(A[i]).T @ np.abs(g[t]))
            part[t], part_size[t] = B[i].T @ v, np.abs(B[i]).T @ v_size
            r["dA"][i] += np.outer(g[t], low[t])
            r["dA_size"][i] += np.abs(np.outer(g[t], low[t]))
            r["dB"][i] += np.outer(v, x_low[t])
            r["dB_size"][i] += np.outer(v_size, np.abs(x_low[t]))
    return dict(r, d_x=base + part, d_x_size=base_size + part_size, d_x_base=base, d_x_base_size=base_size, d_x_low=part, d_x_low_size=part_size)
