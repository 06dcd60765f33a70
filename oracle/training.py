"""What follows the layer's gradients in a training step, in float64 numpy from the definitions: the router's balance loss
and its gradient, the norm of a list of gradients, the AdamW step and the 8-bit form of its states."""
from __future__ import annotations

import numpy as np

BLOCK = 32           # elements of an 8-bit state that share a scale


def _tokens(T, mask, offsets):
    """Sequence of every token that counts, -1 for the others."""
    offsets = np.array([0, T]) if offsets is None else np.asarray(offsets)
    seq = np.full(T, -1)
    for s in range(len(offsets) - 1):
        seq[offsets[s]:offsets[s + 1]] = s
    if mask is not None:
        seq[np.asarray(mask) == 0] = -1
    return seq, len(offsets) - 1


def softmax(logits):
    """p and log-sum-exp of one token's logits; zeros where all of them are -inf."""
    x = np.asarray(logits, dtype=np.float64)
    top = x.max()
    if top == -np.inf:
        return np.zeros_like(x), 0.0
    e = np.exp(x - top)
    return e / e.sum(), top + np.log(e.sum())


def balance_loss(logits, idx, balance_coef, z_coef, mask=None, offsets=None):
    """counts, prob_sums, seq_tokens (n_s, then n) and the two losses."""
    T, E = logits.shape
    K = idx.shape[1]
    seq, S = _tokens(T, mask, offsets)
    counts, sums, n, z = np.zeros((S, E), dtype=np.int64), np.zeros((S, E)), np.zeros(S, dtype=np.int64), 0.0
    for t in np.nonzero(seq >= 0)[0]:
        p, lse = softmax(logits[t])
        sums[seq[t]] += p
        n[seq[t]] += 1
        z += lse ** 2
        for e in idx[t]:
            if 0 <= e < E:
                counts[seq[t], e] += 1
    total = n.sum()
    losses = np.zeros(2)
    if total:
        losses[0] = balance_coef * E / (K * total) * sum((counts[s] * sums[s]).sum() / n[s] for s in range(S) if n[s])
        losses[1] = z_coef / total * z
    return counts, sums, np.append(n, total), losses


def balance_loss_backward(logits, counts, seq_tokens, dlosses, K, balance_coef, z_coef, mask=None, offsets=None):
    """Gradient of dlosses . losses in the logits, and the size of what is added up in every element of it."""
    T, E = logits.shape
    seq, _ = _tokens(T, mask, offsets)
    d, size, n = np.zeros((T, E)), np.zeros((T, E)), max(int(seq_tokens[-1]), 1)
    for t in np.nonzero(seq >= 0)[0]:
        p, lse = softmax(logits[t])
        g = dlosses[0] * balance_coef * E / (K * n * seq_tokens[seq[t]]) * counts[seq[t]]
        az = dlosses[1] * 2 * z_coef / n
        d[t] = p * (g - (p * g).sum() + az * lse)
        size[t] = p * (abs(g) + (p * abs(g)).sum() + abs(az * lse))
    return d, size


def grad_norm(grads, max_norm=0.0, multiplier=1.0):
    norm = abs(multiplier) * np.sqrt(sum((np.asarray(g, dtype=np.float64) ** 2).sum() for g in grads))
    if not np.isfinite(norm):
        return norm, np.nan
    return norm, multiplier * (min(1.0, max_norm / (norm + 1e-6)) if max_norm > 0 else 1.0)


def adamw(p, g, m, v, lr, beta1, beta2, eps, step, decay):
    """p, m and v after a step, in float64."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g ** 2
    return adamw_weight(p, m, v, lr, beta1, beta2, eps, step, decay), m, v


def adamw_weight(p, m, v, lr, beta1, beta2, eps, step, decay):
    """p after a step whose new moments are m and v, in float64."""
    p, m, v = (np.asarray(a, dtype=np.float64) for a in (p, m, v))
    denom = np.sqrt(v) / np.sqrt(1 - beta2 ** step) + eps
    return p * (1 - lr * decay) - lr / (1 - beta1 ** step) * m / denom


def moments32(g, m, v, beta1, beta2):
    """The two moments with every operation rounded to fp32, as the interface says."""
    g, m, v = (np.asarray(a, dtype=np.float32) for a in (g, m, v))
    b1, c1, b2, c2 = (np.float32(x) for x in (beta1, 1 - beta1, beta2, 1 - beta2))
    return m * b1 + g * c1, v * b2 + (g * g) * c2


def _mix(x):
    x = x ^ (x >> np.uint32(16))
    x = x * np.uint32(0x7feb352d)
    x = x ^ (x >> np.uint32(15))
    x = x * np.uint32(0x846ca68b)
    return x ^ (x >> np.uint32(16))


def random_bits(seed, tensor, j):
    """32 bits of the elements j (int64 array) of a tensor."""
    j = np.asarray(j, dtype=np.uint64)
    high = (j >> np.uint64(32)).astype(np.uint32)
    with np.errstate(over="ignore"):
        first = np.uint32((seed + 0x9e3779b9 * (tensor + 1)) & 0xffffffff)
        return _mix((j & np.uint64(0xffffffff)).astype(np.uint32) ^ _mix(first + np.uint32(0x85ebca6b) * high))


def e4m3_values():
    """Value of every code (OCP E4M3: bias 7, no infinities, 0x7f and 0xff NaN)."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * 2.0 ** (e - 7.0))
    v[(c & 0x7f) == 0x7f] = np.nan
    return np.where(c & 0x80, -v, v)


def mxfp8_values(codes, scales):
    """What codes and scales stand for."""
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return e4m3_values()[codes] * np.repeat(s, BLOCK)[:len(codes)]


def mxfp8(x, random16, keep_positive):
    """Codes and scales of x: each magnitude goes to the value below it or, where the part cut off is at least
    1 - (u + 1/2) / 65536 of the step between them, to the one above; ``keep_positive``: what is above 0 stays there."""
    x = np.asarray(x, dtype=np.float64)
    grid = e4m3_values()[:127]
    codes = np.zeros(len(x), dtype=np.uint8)
    scales = np.zeros((len(x) + BLOCK - 1) // BLOCK, dtype=np.uint8)
    for b in range(len(scales)):
        at = slice(b * BLOCK, min((b + 1) * BLOCK, len(x)))
        if not np.isfinite(x[at]).all():
            scales[b], codes[at] = 255, 0x7f
            continue
        top, k = np.abs(x[at]).max(), -126
        if top > 448 * 2.0 ** k:
            k = int(np.ceil(np.log2(top / 448)))
            while top > 448 * 2.0 ** k:
                k += 1
            while k > -126 and top <= 448 * 2.0 ** (k - 1):
                k -= 1
        scales[b] = k + 127
        y = np.abs(x[at]) / 2.0 ** k
        low = np.searchsorted(grid, y, side="right") - 1
        step = np.append(np.diff(grid), 32.0)[low]
        c = low + ((y - grid[low]) / step >= 1 - (random16[at] + 0.5) / 65536)
        if keep_positive:
            c = np.where((c == 0) & (y > 0), 1, c)
        codes[at] = c | np.where(np.signbit(x[at]), 0x80, 0)
    return codes, scales


def bf16_stochastic(p, bits):
    """Bit patterns of fp32 values rounded to bf16: up where the part cut off is at least 1 - u / 65536 of the step."""
    u = (bits.astype(np.uint64) * 0x9e3779b1 & 0xffffffff) >> 16
    return ((np.asarray(p, dtype=np.float32).view(np.uint32).astype(np.uint64) + u) >> 16).astype(np.uint16)
