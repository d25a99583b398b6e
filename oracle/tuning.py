"""Fine-tuning operators in fp64 numpy, from their definitions (include/nmd.h).

Rows with a target below zero take no part: nothing of theirs is read.
"""
from __future__ import annotations

import numpy as np


def _lse(z):
    """log sum exp of each row; -inf entries add nothing."""
    m = z.max(axis=1, keepdims=True)
    return (m + np.log(np.exp(z - m).sum(axis=1, keepdims=True)))[:, 0]


def token_logprobs(x, y, temperature=1.0):
    """(T,) log-probability of column y[t] of row t; 0 where y[t] < 0."""
    y = np.asarray(y)
    lp = np.zeros(len(y))
    live = np.flatnonzero(y >= 0)
    if len(live):
        z = np.asarray(x, np.float64)[live] / temperature
        lp[live] = z[np.arange(len(live)), y[live]] - _lse(z)
    return lp


def factor_logprobs(A, B, y, temperature=1.0):
    y = np.asarray(y)
    live = y >= 0
    A = np.where(live[:, None], np.asarray(A, np.float64), 0.0)
    return token_logprobs(A @ np.asarray(B, np.float64).T, y, temperature)


def logits_gradient(x, y, g, temperature=1.0):
    """d[t, v] = g_t (1[v = y_t] - p_tv) / temperature, zero rows where y[t] < 0 or g_t = 0."""
    d = np.zeros(np.shape(x))
    live = np.flatnonzero((np.asarray(y) >= 0) & (np.asarray(g) != 0))
    if len(live):
        z = np.asarray(x, np.float64)[live] / temperature
        p = np.exp(z - _lse(z)[:, None])
        p = -p
        p[np.arange(len(live)), np.asarray(y)[live]] += 1.0
        d[live] = p * (np.asarray(g, np.float64)[live] / temperature)[:, None]
    return d


def _log_sigmoid(h):
    return np.minimum(h, 0.0) - np.log1p(np.exp(-np.abs(h)))


def preference_loss(x, y, offsets, reference, beta=0.1, smoothing=0.0, average=False, temperature=1.0):
    """dict of loss, logps, ratios, margins, coef (g_t) and grad."""
    y = np.asarray(y)
    lp = token_logprobs(x, y, temperature)
    K = len(offsets) - 1
    ratios, share = np.zeros(K), np.ones(K)
    for k in range(K):
        rows = np.arange(offsets[k], offsets[k + 1])
        rows = rows[y[rows] >= 0]
        ratios[k] = np.sum(lp[rows] - np.asarray(reference, np.float64)[rows])
        if average and len(rows):
            share[k] = 1.0 / len(rows)
            ratios[k] *= share[k]
    h = beta * (ratios[0::2] - ratios[1::2])
    P = K // 2
    loss = np.mean(-(1.0 - smoothing) * _log_sigmoid(h) - smoothing * _log_sigmoid(-h))
    slope = beta * (smoothing - np.exp(_log_sigmoid(-h))) / P
    coef = np.zeros(len(y))
    for k in range(K):
        coef[offsets[k]:offsets[k + 1]] = (slope[k // 2] if k % 2 == 0 else -slope[k // 2]) * share[k]
    coef[y < 0] = 0.0
    return {"loss": loss, "logps": lp, "ratios": ratios, "margins": h, "coef": coef,
            "grad": logits_gradient(x, y, coef, temperature)}


def policy_weights(y, offsets=None):
    y = np.asarray(y)
    live = y >= 0
    if offsets is None:
        return live / max(1, live.sum())
    w = np.zeros(len(y))
    S = len(offsets) - 1
    for k in range(S):
        rows = np.arange(offsets[k], offsets[k + 1])
        rows = rows[live[rows]]
        if len(rows):
            w[rows] = 1.0 / (S * len(rows))
    return w


def policy_loss(x, y, old, reference, advantages, offsets=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0,
                temperature=1.0):
    """dict of loss, logps, kl, clipped, coef (g_t) and grad."""
    y = np.asarray(y)
    lp = token_logprobs(x, y, temperature)
    w = policy_weights(y, offsets)
    coef, loss, kl_sum, cut_sum = np.zeros(len(y)), 0.0, 0.0, 0.0
    for t in np.flatnonzero(w):                         # neither left out nor outside every sequence
        rho, A = np.exp(lp[t] - np.float64(old[t])), np.float64(advantages[t])
        cut = (A > 0 and rho > 1.0 + clip_high) or (A < 0 and rho < 1.0 - clip_low)
        term = -min(rho * A, min(max(rho, 1.0 - clip_low), 1.0 + clip_high) * A)
        g = 0.0 if cut else -rho * A
        k = 0.0
        if reference is not None:
            gap = np.float64(reference[t]) - lp[t]
            k = np.expm1(gap) - gap
            g -= kl_coef * np.expm1(gap)
        loss += w[t] * (term + kl_coef * k)
        kl_sum += w[t] * k
        cut_sum += w[t] * cut
        coef[t] = w[t] * g
    return {"loss": loss, "logps": lp, "kl": kl_sum, "clipped": cut_sum, "coef": coef,
            "grad": logits_gradient(x, y, coef, temperature)}


def clip_grad_norm(grads, max_norm):
    """(norm, scaled gradients)."""
    flat = [np.asarray(g, np.float64) for g in grads]
    top = max([np.abs(g).max() for g in flat if g.size] + [0.0])
    norm = top * np.sqrt(sum(np.sum((g / top) ** 2) for g in flat)) if 0.0 < top < np.inf else \
        np.sqrt(sum(np.sum(g ** 2) for g in flat))
    scale = 1.0 if norm <= max_norm else max_norm / norm
    return norm, [g * scale for g in flat]


def beam_select(x, scores, width, finished=None, end=None, temperature=1.0):
    """(scores, parents, tokens, finished), each (B, width): the largest of scores[b, k] + log softmax(x / temperature),
    of equal ones the lowest (k, column); -inf, 0, -1 and False where nothing finite is left."""
    scores = np.asarray(scores, np.float64)
    B, K = scores.shape
    V = np.shape(x)[1]
    finished = None if finished is None else np.asarray(finished)
    value = np.full((B, K, V), -np.inf)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for b in range(B):
            for k in range(K):
                if not np.isfinite(scores[b, k]):
                    continue
                if finished is not None and finished[b, k]:
                    value[b, k, end] = scores[b, k]
                    continue
                z = np.asarray(x[b * K + k], np.float64)
                z = (z - z.max()) / temperature   # (huge values would swallow the logarithm of the sum)
                value[b, k] = scores[b, k] + (z - np.log(np.exp(z).sum()))
    value[~np.isfinite(value)] = -np.inf
    value = value.reshape(B, K * V)
    value = np.concatenate([value, np.full((B, max(0, width - K * V)), -np.inf)], axis=1)
    order = np.argsort(-value, axis=1, kind="stable")[:, :width]
    best = np.take_along_axis(value, order, 1)
    some = best > -np.inf
    tokens = np.where(some, order % V, -1)
    return best, np.where(some, order // V, 0), tokens, some & (tokens == (-2 if end is None else end))


def beam_reorder(x, parents, dim=0, out=None):
    """Along ``dim``, row b K + k of what parents (B, width) take; a parent outside [0, K) leaves the row of ``out``."""
    B, w = np.shape(parents)
    K = np.shape(x)[dim] // B if B else 0
    y = np.moveaxis(np.array(x if out is None else out), dim, 0)
    x = np.moveaxis(np.array(x), dim, 0)
    for b in range(B):
        for k in range(w):
            if 0 <= parents[b, k] < K:
                y[b * w + k] = x[b * K + parents[b, k]]
    return np.moveaxis(y, 0, dim)


def orthogonalize(G, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    """U f(S) V^T of the update's singular value decomposition, f the map of the steps on S / (|G|_F + eps)."""
    G = np.asarray(G, np.float64)
    a, b, c = coefficients
    if G.size == 0:
        return G.copy()
    U, s, Vt = np.linalg.svd(G / (np.linalg.norm(G) + eps), full_matrices=False)
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return (U * s) @ Vt


def muon_step(W, G, M, lr, beta=0.95, nesterov=True, weight_decay=0.0, scale=None, round_momentum=lambda m: m, **kw):
    """(weights, momentum) after one step; ``round_momentum`` rounds the momentum to its type."""
    W, G, M = (np.asarray(v, np.float64) for v in (W, G, M))
    M = round_momentum(beta * M + (1 - beta) * G)
    U = beta * M + (1 - beta) * G if nesterov else M
    if scale is None:
        scale = max(1.0, W.shape[0] / max(1, W.shape[1])) ** 0.5
    return (1 - lr * weight_decay) * W - lr * scale * orthogonalize(U, **kw), M
