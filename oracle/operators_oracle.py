"""Plain 64-bit implementations of the operators around a 4-bit linear layer, from their definitions (test infrastructure only).

MX numbers: 32 channels share 2^(E - 127); see include/esparse.h.  Everything is numpy on the CPU; floats are float64.
"""
import numpy as np

FP4, FP8 = 0, 1
GRID = {FP4: np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6.0]),
        FP8: np.array([k * 2.0 ** -9 for k in range(8)] + [(8 + k) * 2.0 ** (p - 3) for p in range(-6, 9) for k in range(8)][:-1])}
EMAX = {FP4: 2, FP8: 8}


def mx_quantize(x, fmt):
    """Codes uint8 [R, Kp] (one per byte) and scale bytes [R, Kp / 32] of x[R, K]."""
    R, K = x.shape
    p = np.zeros((R, -(-K // 128) * 128))
    p[:, :K] = x
    b = p.reshape(R, -1, 32)
    bad = ~np.isfinite(b).all(2)
    b = np.where(bad[:, :, None], 0.0, b)
    top = np.abs(b).max(2)
    with np.errstate(divide="ignore"):
        e = np.where(top > 0, np.frexp(top)[1] - 1 - EMAX[fmt], -127)
    E = np.maximum(e, -127) + 127
    a = np.abs(b) / np.ldexp(1.0, E - 127)[:, :, None]
    g = GRID[fmt]
    hi = np.clip(np.searchsorted(g, a), 0, len(g) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = g[hi] - a, a - g[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo) + np.where(np.signbit(b), len(g) if fmt == FP4 else 128, 0)
    code[bad] = 0
    return code.reshape(R, -1).astype(np.uint8), np.where(bad, 255, E).astype(np.uint8)


def mx_values(code, E, fmt):
    """float64 [R, Kp] that codes and scale bytes stand for."""
    g = GRID[fmt]
    half = 8 if fmt == FP4 else 128
    mag = code.astype(int) % half
    v = np.where(code >= half, -1.0, 1.0) * np.where(mag < len(g), g[np.minimum(mag, len(g) - 1)], np.nan)
    s = np.where(E == 255, np.nan, np.ldexp(1.0, E.astype(int) - 127))
    return (v.reshape(v.shape[0], -1, 32) * s[:, :, None]).reshape(v.shape)


def mx_data(code, fmt):
    """The bytes of the library's data tensor."""
    return code if fmt == FP8 else code[:, 0::2] | code[:, 1::2] << 4


def mx_scales(E):
    """The library's scales [Kp / 128, R, 4]."""
    return np.ascontiguousarray(E.reshape(E.shape[0], -1, 4).transpose(1, 0, 2))


def mx_pack(code, E):
    """Values and scale words of packed 4-bit weights, as one run of bytes."""
    N, Kp = code.shape
    Np, steps = -(-N // 64) * 64, Kp // 128
    c = np.zeros((Np, Kp), np.uint8)
    c[:N] = code
    s = np.zeros((Np, Kp // 32), np.uint8)
    s[:N] = E
    units = mx_data(c, FP4).reshape(Np // 16, 16, steps, 4, 16).transpose(0, 2, 3, 1, 4)  # [row tile, step, block, row, byte]
    words = s.reshape(Np // 64, 4, 16, steps, 4).transpose(0, 3, 4, 2, 1)                 # [64 rows, step, block, row, byte]
    return np.concatenate([np.ascontiguousarray(units).reshape(-1), np.ascontiguousarray(words).reshape(-1)])


def rms_norm(h, weight, eps):
    return h * weight / np.sqrt((h * h).mean(1, keepdims=True) + eps)


def token_logprobs(x, tokens, top):
    """logprob [R], entropy [R], ids [R, top], their log probabilities [R, top] of logits x[R, V]."""
    R, V = x.shape
    lp, ent = np.empty(R), np.empty(R)
    ids, tops = np.empty((R, top), np.int64), np.empty((R, top))
    for r in range(R):
        row = x[r]
        if np.isnan(row).any() or (row == np.inf).any():
            logp, ent[r], ids[r] = np.full(V, np.nan), np.nan, -1
        elif (row == -np.inf).all():
            logp, ent[r], ids[r] = np.full(V, -np.inf), 0.0, np.arange(top)
        else:
            d = row - row.max()
            logp = d - np.log(np.exp(d).sum())
            p = np.exp(logp)
            ent[r] = -(p[p > 0] * logp[p > 0]).sum()
            ids[r] = np.argsort(-row, kind="stable")[:top]
        tops[r] = logp[ids[r]]
        t = tokens[r]
        lp[r] = 0.0 if t < 0 else (np.nan if t >= V else logp[t])
    return lp, ent, ids, tops
