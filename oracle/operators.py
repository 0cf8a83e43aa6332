"""Oracle of the operators beside the paged attention: rotary positions, attention over whole prompts, accumulated attention
weights, eviction.  TEST INFRASTRUCTURE ONLY; shares no code with the CUDA library.

Each function is the definition written out in fp64, token by token and head by head; angles are formed in extended precision.
"""
from __future__ import annotations

import numpy as np


def rotate(x, positions, pair_axis, inv_freq, adjacent=False, amplitude=1.0):
    """x [n][H][D] real, positions int [axes][n], pair_axis / inv_freq [rotary / 2]
    -> (rotated [n][H][D] fp64, |a| + |b| of the pair each element belongs to [n][H][D])"""
    x = np.asarray(x, dtype=np.float64)
    out, size = x.copy(), np.zeros_like(x)
    half = len(pair_axis)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, half + i)
        angle = np.asarray(positions[pair_axis[i]], dtype=np.longdouble) * np.longdouble(inv_freq[i])
        angle = np.fmod(angle, 2 * np.longdouble("3.14159265358979323846264338327950288"))
        c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
        out[:, :, a] = amplitude * (x[:, :, a] * c - x[:, :, b] * s)
        out[:, :, b] = amplitude * (x[:, :, b] * c + x[:, :, a] * s)
        size[:, :, a] = size[:, :, b] = amplitude * (np.abs(x[:, :, a]) + np.abs(x[:, :, b]))
    return out, size


def attend(q, k, v, scale):
    """One query row over tokens k, v [t][D] -> (out [D], weights [t], sum_t weight |v| [D])"""
    s = scale * (k @ q)
    p = np.exp(s - s.max())
    p = p / p.sum()
    return p @ v, p, p @ np.abs(v)


def prompt_attention(q, k, v, offsets, scale):
    """q [n][Hq][D], k, v [n][Hkv][D] real -> (out [n][Hq][D], sum of weight |v| [n][Hq][D]); token i of a sequence sees the
    sequence's tokens up to itself."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    out, size = np.zeros_like(q), np.zeros_like(q)
    group = q.shape[1] // k.shape[1]
    for s in range(len(offsets) - 1):
        o, e = int(offsets[s]), int(offsets[s + 1])
        for i in range(o, e):
            for h in range(q.shape[1]):
                out[i, h], _, size[i, h] = attend(q[i, h], k[o:i + 1, h // group], v[o:i + 1, h // group], scale)
    return out, size


def attention_weights(q, k, scale):
    """q [Hq][D], k [t][Hkv][D] real: one sequence's decode step -> per KV head and token the weights its group gave [Hkv][t]"""
    hq, hkv = q.shape[0], k.shape[1]
    w = np.zeros((hkv, k.shape[0]))
    for h in range(hq):
        if k.shape[0]:
            w[h // (hq // hkv)] += attend(q[h], k[:, h // (hq // hkv)], np.zeros_like(k[:, 0]), scale)[1]
    return w


def keep(weights, ctx, budget, recent):
    """Positions that one KV head keeps, ascending: all of at most `budget`; else the newest `recent` and, of the others, the
    budget - recent with the largest weights (equal ones: the lower position; NaN the smallest)."""
    if ctx <= budget:
        return list(range(ctx))
    old = sorted(range(ctx - recent), key=lambda t: (not np.isnan(weights[t]), 0.0 if np.isnan(weights[t]) else weights[t], -t), reverse=True)
    return sorted(old[:budget - recent]) + list(range(ctx - recent, ctx))
