"""Plain 64-bit implementations of the steps of decoding between and behind the products, from their definitions (test infrastructure only).

Heads, their rotation and their form in a cache of microscaled 4 bits, attention over it, the draw of a token; see include/esparse.h.  Everything is numpy on
the CPU; floats are float64.
"""
import numpy as np

from . import operators_oracle as mx


def row_of(D):
    return 64 if D <= 64 else 128 if D <= 128 else 256


def rotate(x, weight, eps, positions, frequencies, paired):
    """Heads x[T, H, D] normalised (with a weight) and rotated."""
    y = x.astype(np.float64)
    if weight is not None:
        with np.errstate(all="ignore"):
            y = y * weight.astype(np.float64) / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
    half = 0 if frequencies is None else len(frequencies)
    out = y.copy()
    for i in range(half):
        t = (positions.astype(np.float64) * float(frequencies[i]))[:, None]
        a, b = (2 * i, 2 * i + 1) if paired else (i, i + half)
        with np.errstate(invalid="ignore"):
            out[..., a] = y[..., a] * np.cos(t) - y[..., b] * np.sin(t)
            out[..., b] = y[..., b] * np.cos(t) + y[..., a] * np.sin(t)
    return out


def cache_rows(x):
    """Bytes uint8 [T, H, row / 2] and scales [T, H, row / 32] of heads x[T, H, D]."""
    T, H, D = x.shape
    row = row_of(D)
    wide = np.zeros((T * H, row))
    wide[:, :D] = x.reshape(T * H, D)
    code, E = mx.mx_quantize(wide, mx.FP4)   # (padded to 128 channels: the first `row` are ours)
    return mx.mx_data(code[:, :row], mx.FP4).reshape(T, H, row // 2), E[:, : row // 32].reshape(T, H, row // 32)


def cache_values(data, scales, D):
    """float64 [..., D] that bytes [..., row / 2] and scales [..., row / 32] stand for."""
    code = np.stack((data & 15, data >> 4), -1).reshape(-1, 2 * data.shape[-1])
    return mx.mx_values(code, scales.reshape(code.shape[0], -1), mx.FP4).reshape(data.shape[:-1] + (2 * data.shape[-1],))[..., :D]


def attend(q, k, v, scale, last):
    """(out [m, D], ln sum exp [m], sum p |v| [m, D], sum |v| [m, D], the largest error that fp32 sums of the scores may have [m]) of one head's queries q[m, D] over tokens
    k, v[n, D]; row i sees tokens 0 .. last[i]."""
    m, n = len(q), len(k)
    out, lse, spread, mass, off = np.zeros(q.shape), np.full(m, -np.inf), np.zeros(q.shape), np.zeros(q.shape), np.zeros(m)
    for i in range(m):
        c = min(int(last[i]) + 1, n)
        if c <= 0:
            continue
        with np.errstate(invalid="ignore"):
            x = k[:c] @ q[i] * scale
            p = np.exp(x - x.max())
            out[i] = p @ v[:c] / p.sum()
            lse[i] = x.max() + np.log(p.sum())
            spread[i] = p @ np.abs(v[:c]) / p.sum()
            mass[i] = np.abs(v[:c]).sum(0) / p.sum()
            off[i] = (np.abs(k[:c]) @ np.abs(q[i]) * abs(scale)).max() * q.shape[1] * 2.0 ** -23 + np.abs(x).max() * 2.0 ** -21
    return out, lse, spread, mass, off


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, indices kept) of one row of logits."""
    x = x.astype(np.float64)
    if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any() or not 0 <= temperature < np.inf:
        return -1, np.nan, []
    if temperature == 0:
        return int(np.argmax(x)), 0.0, [int(np.argmax(x))]
    w = np.exp((x - x.max()) / float(temperature))
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        upto = np.cumsum(w[order])
        order = order[: max(1, int((upto - w[order] < float(top_p) * upto[-1]).sum()))]
    if min_p > 0:
        order = order[w[order] >= min(float(min_p), 1.0)]
    kept = np.sort(order)
    upto = np.cumsum(w[kept])
    u = 0.0 if not u > 0 else min(float(u), 1 - 2.0 ** -24)
    token = kept[min(int(np.searchsorted(upto, u * upto[-1], side="right")), len(kept) - 1)]
    return int(token), float((x[token] - x.max()) / float(temperature) - np.log(upto[-1])), kept
