"""Routing by scores, in numpy from the definitions: selection with a balancing bias within the best groups of experts, the
gates and their gradient in float64, and the step of the bias."""
from __future__ import annotations

import numpy as np

SOFTMAX, SIGMOID = 0, 1


def scores(logits, score):
    """s [T, E] in float64, 0 where the logit is -inf or NaN, and where it is neither."""
    x = np.asarray(logits, dtype=np.float64)
    taken = x > -np.inf
    with np.errstate(all="ignore"):
        if score == SIGMOID:
            s = 1 / (1 + np.exp(-x))
        else:
            top = np.where(taken, x, -np.inf).max(1, keepdims=True)
            e = np.where(taken, np.where(x == top, 1.0, np.exp(x - top)), 0.0)
            s = e / e.sum(1, keepdims=True)
    return np.where(taken, s, 0.0), taken


def _first(keys, n):
    """Places of the n largest of every row, the lower place first among equal ones."""
    return np.argsort(-keys, axis=1, kind="stable")[:, :n]


def select(logits, K, score, bias=None, groups=1, topk_groups=1, group_best=2, renormalize=True, scale=1.0):
    """topk_idx [T, K] (-1: none left) and topk_gate [T, K] in float64."""
    s, taken = scores(logits, score)
    T, E = s.shape
    with np.errstate(all="ignore"):
        key = s.astype(np.float32)
        if bias is not None:
            key = key + np.asarray(bias, dtype=np.float32)
        low = np.finfo(np.float32).min
        key = np.where(taken & (key > low), key, -np.inf).astype(np.float32)
        if groups > 1:
            g = key.reshape(T, groups, E // groups)
            best = -np.sort(-g, axis=2)[:, :, :group_best]
            value = best[:, :, 0].copy()
            if best.shape[2] > 1:
                value = np.where(best[:, :, 1] > -np.inf, np.maximum(value + best[:, :, 1], low), value)
            keep = np.zeros((T, groups), dtype=bool)
            np.put_along_axis(keep, _first(value, topk_groups), True, 1)
            key = np.where(keep[:, :, None], g, -np.inf).reshape(T, E)
    idx = _first(key, K)
    has = np.take_along_axis(key, idx, 1) > -np.inf
    g = np.where(has, np.take_along_axis(s, idx, 1), 0.0)
    if renormalize:
        total = g.sum(1, keepdims=True)
        g = np.divide(g, total, out=np.zeros_like(g), where=total > 0)
    return np.where(has, idx, -1).astype(np.int32), g * scale


def select_backward(logits, idx, dgate, score, renormalize=True, scale=1.0):
    """dlogits [T, E] in float64, and the size of what is added up in every element of it."""
    s, taken = scores(logits, score)
    T, E = s.shape
    out, size = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        slots = [k for k in range(idx.shape[1]) if 0 <= idx[t, k] < E and taken[t, idx[t, k]]]
        if not slots:
            continue
        e = idx[t, slots]
        d, r = dgate[t, slots].astype(np.float64) * scale, s[t, e]
        a = abs(d)
        if renormalize:
            if r.sum() == 0:
                continue
            r = r / r.sum()
            a, d = a + (abs(d) * r).sum(), d - (d * r).sum()
        c, a = r * d, r * a
        if score == SIGMOID:
            rest = 1 / (1 + np.exp(logits[t, e].astype(np.float64)))
            np.add.at(out[t], e, c * rest)
            np.add.at(size[t], e, a * rest)
        else:
            np.add.at(out[t], e, c)
            np.add.at(size[t], e, a)
            out[t] -= s[t] * c.sum()
            size[t] += s[t] * a.sum()
    return out, size


def bias_update(counts, rate, bias):
    n = np.asarray(counts, dtype=np.int64).reshape(-1, len(bias)).sum(0)
    return np.asarray(bias, dtype=np.float32) + np.float32(rate) * np.sign(n.sum() - n * len(n)).astype(np.float32)
