"""fp64 statement of the operators around the expert layer: residual + root-mean-square norm, rows in e4m3 with scales, and
attention of one new token over a paged cache.  Test infrastructure only; shares nothing with the library."""
from __future__ import annotations

import numpy as np

E4M3_MAX, MIN_SCALE = 448.0, 2.0 ** -126


def add_norm(x, residual, weight, eps):
    """(s, n): s = x + residual, n = s / sqrt(mean(s^2) + eps) * weight, row by row."""
    s = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    return s, s / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps) * np.asarray(weight, np.float64)


def e4m3(r):
    """The nearest value with a sign, four exponent bits (smallest normal 2^-6) and three bits after the point; ties to even."""
    r = np.asarray(r, np.float64)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(r), 2.0 ** -20))), -6) - 3)
    return np.clip(np.round(r / step) * step, -E4M3_MAX, E4M3_MAX)


def e4m3_scale(rows):
    """One scale for each last axis."""
    return np.maximum(np.abs(rows).max(axis=-1) / E4M3_MAX, MIN_SCALE)


def attention(q, k, v, scale):
    """One query head over its tokens: q [dim], k and v [n, dim] -> (out [dim], lse, weights [n])."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    if len(k) == 0:
        return np.zeros(v.shape[1]), -np.inf, np.zeros(0)
    logits = scale * (k @ q)
    lse = logits.max() + np.log(np.exp(logits - logits.max()).sum())
    p = np.exp(logits - lse)
    return p @ v, lse, p


def paged_rows(pages, scales, table, first, end):
    """Rows [heads, end - first, dim] of one sequence's tokens in float64."""
    page_size = pages.shape[2]
    at = np.arange(first, end)
    rows = pages[table[at // page_size], :, at % page_size].astype(np.float64)             # [n, heads, dim]
    if scales is not None:
        rows = rows * scales[table[at // page_size], :, at % page_size].astype(np.float64)[..., None]
    return rows.transpose(1, 0, 2)


def scored(x, distance, cap=0.0, slope=0.0, bias=None, back=0, ahead=0):
    """Logits of the scores x of keys at these distances (query's place less the key's): capped, less slope * |distance|, plus the bias of the distance."""
    x, distance = np.asarray(x, np.float64), np.asarray(distance, np.int64)
    if cap:
        x = cap * np.tanh(x / cap)
    x = x - slope * np.abs(distance)
    return x if bias is None else x + np.asarray(bias, np.float64)[np.clip(distance, -ahead, back) + ahead]


def masked_attention(q, k, v, scale, place, first, end, window=0, **scores):
    """Query rows [n, dim] at their places over the keys [first, end) of each, in the window: (out [n, dim], lse [n], logits [n, keys], weights)."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    t = np.arange(len(k))
    place, first, end = (np.asarray(a, np.int64)[:, None] for a in (place, first, end))
    if window:
        first = np.maximum(first, place - window + 1)
    seen = (t >= first) & (t < end)
    logits = scored(scale * (q @ k.T), place - t, **scores)
    x = np.where(seen, logits, -np.inf)
    top = x.max(axis=1, initial=-np.inf, keepdims=True)
    w = np.exp(x - np.where(top == -np.inf, 0.0, top))
    total = w.sum(axis=1, keepdims=True)
    p = w / np.where(total == 0, 1.0, total)
    with np.errstate(divide="ignore"):
        lse = (top + np.log(total))[:, 0]
    return p @ v, lse, np.where(seen, logits, 0.0), p


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original=0, slow=1.0, fast=32.0):
    """Radians per position of each pair."""
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if scaling == "linear":
            f = f / factor
        if scaling == "base" and rot > 2:
            f = (base * factor ** (rot / (rot - 2))) ** (-2.0 * i / rot)
        if scaling == "parts":
            turns = original * f / (2 * np.pi)
            keep = min(max((turns - slow) / (fast - slow), 0.0), 1.0)
            f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return np.array(out)


def rotary(x, positions, freqs, rot, neighbours=False, amplitude=1.0):
    """Rows x [n, heads, dim]: the pairs of their first rot columns turned by position * frequency."""
    x = np.array(x, np.float64)
    angle = (np.asarray(positions, np.float64)[:, None] * np.asarray(freqs, np.float64))[:, None]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if neighbours else (slice(0, rot // 2), slice(rot // 2, rot))
    u, v = x[..., a].copy(), x[..., b].copy()
    x[..., a] = amplitude * (u * np.cos(angle) - v * np.sin(angle))
    x[..., b] = amplitude * (u * np.sin(angle) + v * np.cos(angle))
    return x
