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
