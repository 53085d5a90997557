"""Definitions in 64 bits of the operators beside the cache: rotary positions, the values a cache held in 8 bits keeps, and
attention over rows of different lengths.  Test infrastructure; numpy only, and nothing of the library."""
import math

import numpy as np


def rotary_frequencies(P, base=10000.0, scaling="plain", factor=1.0, original_length=0.0, beta_fast=32.0, beta_slow=1.0):
    """Frequencies of one axis of P channels."""
    w = []
    for i in range(P // 2):
        if scaling == "base":
            w.append((base * factor ** (P / (P - 2.0))) ** (-2.0 * i / P))
            continue
        f = base ** (-2.0 * i / P)
        if scaling == "linear":
            f /= factor
        elif scaling == "parts":
            ends = [P * math.log(original_length / (2 * math.pi * b)) / (2 * math.log(base)) for b in (beta_fast, beta_slow)]
            lo = min(max(math.floor(ends[0]), 0), P - 1)
            hi = min(max(math.ceil(ends[1]), 0), P - 1)
            g = min(max((i - lo) / ((hi - lo) if hi > lo else 0.001), 0.0), 1.0)
            f = f * (1 - g) + f / factor * g
        w.append(f)
    return np.array(w)


def rotary_angles(positions, rotary_dim, **spec):
    """positions [n, axes] -> angles [n, rotary_dim / 2], axis by axis."""
    axes = positions.shape[1]
    w = rotary_frequencies(rotary_dim // axes, **spec)
    return np.concatenate([positions[:, a:a + 1].astype(np.float64) * w for a in range(axes)], 1)


def rotary_pairs(rotary_dim, axes, interleaved):
    """Channels (first, second) of every column of the table."""
    P = rotary_dim // axes
    out = []
    for a in range(axes):
        for i in range(P // 2):
            out.append((a * P + 2 * i, a * P + 2 * i + 1) if interleaved else (a * P + i, a * P + i + P // 2))
    return np.array(out)


def rotate(x, angles, axes, interleaved=False, amplitude=1.0, transposed=False):
    """x [..., T, D], angles [..., T, rotary_dim / 2] (NaN: a token without a position)."""
    pairs = rotary_pairs(2 * angles.shape[-1], axes, interleaved)
    idle = np.isnan(angles)
    c = np.where(idle, 1.0, amplitude * np.cos(angles))
    s = np.where(idle, 0.0, amplitude * np.sin(angles)) * (-1.0 if transposed else 1.0)
    y = x.astype(np.float64).copy()
    u, w = y[..., pairs[:, 0]], y[..., pairs[:, 1]]
    y[..., pairs[:, 0]], y[..., pairs[:, 1]] = u * c - w * s, w * c + u * s
    return y


def held_exponents(x):
    """Powers of two of the blocks of 16 tokens: x [..., T, D] -> [..., ceil(T / 16)] integers."""
    T = x.shape[-2]
    out = []
    for b in range(0, T, 16):
        top = np.abs(x[..., b:b + 16, :]).max((-2, -1))
        e = np.zeros(top.shape, dtype=np.int64)
        for i in np.ndindex(top.shape):
            if top[i] > 0:
                e[i] = -100
                while top[i] > 448.0 * 2.0 ** e[i]:
                    e[i] += 1
        out.append(e)
    return np.stack(out, -1)


def round_e4m3(y):
    """To the nearest number of 4 significant bits, in steps of 2^-9 below 2^-6; ties to even."""
    size = np.maximum(np.abs(y), 2.0 ** -6)
    step = np.exp2(np.floor(np.log2(size)) - 3)
    step = np.where(size < step * 8, step / 2, np.where(size >= step * 16, step * 2, step))   # (log2 may be off by a rounding)
    return np.round(y / step) * step


def held_values(x):
    """What a cache of 8 bits gives back for x [..., T, D]."""
    e = np.repeat(held_exponents(x), 16, -1)[..., :x.shape[-2], None].astype(np.float64)
    return round_e4m3(x * np.exp2(-e)) * np.exp2(e)


def attention(q, k, v, scale):
    """[..., T, D] over [..., S, D]: the outputs, and the same sums with |v| (what roundings of the probabilities are measured by)."""
    if k.shape[-2] == 0:
        return np.zeros(q.shape), np.zeros(q.shape)
    s = scale * (q @ np.swapaxes(k, -1, -2))
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return p @ v, p @ np.abs(v)
