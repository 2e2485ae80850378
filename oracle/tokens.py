"""CPU oracle of the operators at the two ends of a step on tokens, and of layer norm: embedding lookup and its gradient, layer
norm and its backward pass, log probabilities of given tokens with entropy and top alternatives, distillation from a
teacher's top scores.

NumPy only; test infrastructure.  Everything is computed in fp64 from the definitions, row by row where that is plainer."""
from __future__ import annotations

import math

import numpy as np

MASKED = -(2.0 ** 126)          # a row without a score above this has nothing left


def embedding(tokens, table, scale=1.0):
    out = np.zeros((len(tokens), table.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < len(table):
            out[i] = scale * table[t]
    return out


def embedding_backward(dy, tokens, vocab, scale=1.0, dtable=None):
    """(the gradient, the sum of the terms' magnitudes, the number of terms of each row)."""
    total = np.zeros((vocab, dy.shape[1])) if dtable is None else dtable.astype(np.float64).copy()
    size, count = np.abs(total), np.zeros(vocab, dtype=np.int64)
    for i, t in enumerate(tokens):
        if 0 <= t < vocab:
            total[t] += scale * dy[i]
            size[t] += np.abs(scale * dy[i])
            count[t] += 1
    return total, size, count


def layernorm(x, r, w, b, eps):
    """(h, y, mean, rstd)"""
    h = x if r is None else x + r
    mean = h.mean(axis=1)
    c = h - mean[:, None]
    with np.errstate(divide="ignore"):
        rstd = 1.0 / np.sqrt(np.mean(c * c, axis=1) + eps)
    y = c * rstd[:, None]
    y = y if w is None else y * w
    return h, (y if b is None else y + b), mean, rstd


def layernorm_backward(dy, h, w, mean, rstd, dres=None):
    """(dx, dw, db)"""
    xh = (h - mean[:, None]) * rstd[:, None]
    q = dy if w is None else dy * w
    dx = rstd[:, None] * (q - q.mean(axis=1, keepdims=True) - xh * np.mean(q * xh, axis=1, keepdims=True))
    return (dx if dres is None else dx + dres), np.sum(dy * xh, axis=0), dy.sum(axis=0)


def log_softmax(x, scale):
    """(log p, lse) of one row; a row with nothing left: -inf everywhere, one with NaN or +inf: NaN."""
    if np.isnan(x).any() or np.isposinf(x).any():
        return np.full(len(x), math.nan), math.nan
    top = x.max()
    if top <= MASKED:
        return np.full(len(x), -math.inf), -math.inf
    d = scale * (x - top)
    total = math.log(np.exp(d).sum())
    return d - total, scale * top + total


def top_places(x, k):
    """The k best places: by score, a NaN above all, of equal ones the lowest place first."""
    key = np.where(np.isnan(x), 0, 1), -np.where(np.isnan(x), 0.0, x)
    return np.lexsort((np.arange(len(x)), key[1], key[0]))[:k]


def logprobs(x, tokens, scale=1.0, top=0):
    """(logp, lse, entropy, top values, top index) of every row"""
    n = len(x)
    logp, lse, entropy = np.zeros(n), np.zeros(n), np.zeros(n)
    values, index = np.zeros((n, top)), np.zeros((n, top), dtype=np.int64)
    for i in range(n):
        lp, lse[i] = log_softmax(x[i], scale)
        if tokens is not None and 0 <= tokens[i] < x.shape[1]:
            logp[i] = lp[tokens[i]]
        if math.isnan(lse[i]):
            entropy[i] = math.nan
        elif lse[i] > -math.inf:
            some = lp > -math.inf
            entropy[i] = -np.sum(np.exp(lp[some]) * lp[some])
        index[i] = top_places(x[i], top)
        values[i] = lp[index[i]]
    return logp, lse, entropy, values, index


def logprobs_backward(x, tokens, lse, scale=1.0, dlogp=None, dlse=None, dentropy=None, entropy=None):
    """(dx, the magnitude of each element's terms) with p = exp(scale x - lse)"""
    dx, size = np.zeros(x.shape), np.zeros(x.shape)
    for i in range(len(x)):
        t = -1 if tokens is None or dlogp is None or not 0 <= tokens[i] < x.shape[1] else tokens[i]
        up = dlogp[i] if t >= 0 else 0.0
        z, h = (0.0 if dlse is None else dlse[i]), (0.0 if dentropy is None else dentropy[i])
        if lse[i] == -math.inf or (up == 0 and z == 0 and h == 0):
            continue
        lp = scale * x[i] - lse[i]
        p = np.exp(lp)
        lp = np.where(p == 0, 0.0, lp)
        e = 0.0 if h == 0 else entropy[i]
        dx[i] = p * (z - up - h * (lp + e))
        size[i] = p * (abs(z) + abs(up) + abs(h) * (np.abs(lp) + abs(e)))
        if t >= 0:
            dx[i, t] += up
            size[i, t] += abs(up)
    return scale * dx, scale * size


def teacher(index, values, vocab, scale, normalize):
    """(q, log q) of one row; empty entries have q = 0, whatever the others hold"""
    live = (index >= 0) & (index < vocab)
    v = np.where(live, scale * values, -math.inf)
    if normalize and v.max() != -math.inf:
        v = v - v.max()
        v = np.where(live, v - np.log(np.exp(v).sum()), -math.inf)
    return np.exp(v), v


def distill(x, index, values, scale=1.0, normalize=True):
    """(loss, lse, the sum of the magnitudes of the loss's terms)"""
    n = len(x)
    loss, lse, size = np.zeros(n), np.zeros(n), np.zeros(n)
    for i in range(n):
        lp, lse[i] = log_softmax(x[i], scale)
        q, log_q = teacher(index[i], values[i], x.shape[1], scale, normalize)
        for j, a, b in zip(index[i], q, log_q):
            if a != 0:
                loss[i] += a * (b - lp[j])
                size[i] += a * (abs(b) + abs(lp[j]))
    return loss, lse, size


def distill_backward(x, index, values, lse, dloss, scale=1.0, normalize=True):
    """(dx, the magnitude of each element's terms)"""
    dx, size = np.zeros(x.shape), np.zeros(x.shape)
    for i in range(len(x)):
        q, _ = teacher(index[i], values[i], x.shape[1], scale, normalize)
        if lse[i] == -math.inf or dloss[i] == 0 or not q.any():
            continue
        dx[i] = q.sum() * np.exp(scale * x[i] - lse[i])
        size[i] = dx[i]
        for j, a in zip(index[i], q):
            if a != 0:
                dx[i, j] -= a
                size[i, j] += a
        dx[i] *= scale * dloss[i]
        size[i] *= scale * abs(dloss[i])
    return dx, size
