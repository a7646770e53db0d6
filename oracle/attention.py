"""The attention block around the linears -- oracle.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__``).  Plain NumPy in float64, one loop per
row and head, written from the formulas; nothing here is rounded.
"""
from __future__ import annotations

import numpy as np


def rope_frequencies(rotary_dim, theta, scaling="none", factor=1.0, original=None, fast=32.0, slow=1.0):
    """(radians a position of every pair, gain of cosine and sine)."""
    f, gain = [], 1.0
    for i in range(rotary_dim // 2):
        plain = theta ** (-2.0 * i / rotary_dim)
        if scaling == "linear":
            plain /= factor
        elif scaling == "ntk":
            plain = (theta * factor ** (rotary_dim / (rotary_dim - 2))) ** (-2.0 * i / rotary_dim)
        elif scaling == "yarn":
            # the pair that turns t times in `original` positions: original f / (2 pi) = t
            def pair(t):
                return rotary_dim * np.log(original / (t * 2 * np.pi)) / (2 * np.log(theta))
            lo, hi = max(np.floor(pair(fast)), 0), min(np.ceil(pair(slow)), rotary_dim - 1)
            g = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
            plain = plain / factor * g + plain * (1 - g)
            gain = 0.1 * np.log(factor) + 1.0
        f.append(plain)
    return np.array(f), gain


def norm_rotate(x, weight, eps, turn, interleaved):
    """One head x [D]: RMS norm where a weight is given, then the rotation of its first
    2 len(turn) dims by turn [(cos, sin)]."""
    y = np.asarray(x, np.float64).copy()
    if weight is not None:
        y = y / np.sqrt(np.mean(y * y) + eps) * weight
    half = len(turn)
    z = y.copy()
    for i, (c, s) in enumerate(turn):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        z[a] = y[a] * c - y[b] * s
        z[b] = y[b] * c + y[a] * s
    return z


def sees(i, j, mask_row):
    """Whether own token i of a request sees own token j."""
    if mask_row is None:
        return j <= i
    return j < len(mask_row) and bool(mask_row[j])


def tree_attention(q, keys, values, cached, scale, mask=None):
    """One request: q [n, Hq, D], keys / values [cached + n, Hk, D] (fewer: the rest is unseen) ->
    out [n, Hq, D], lse [n, Hq], and sum_j p_j |v_j| and max_j sum_d |q_d k_d| for error bounds."""
    n, Hq, D = q.shape
    Hk = keys.shape[1]
    out, spread = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    lse, size = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    for i in range(n):
        seen = [j for j in range(len(keys))
                if j < cached or sees(i, j - cached, None if mask is None else mask[i])]
        if not seen:
            continue
        for h in range(Hq):
            k, v = keys[seen, h // (Hq // Hk)], values[seen, h // (Hq // Hk)]
            s = scale * (k @ q[i, h])
            top = s.max()
            p = np.exp(s - top)
            out[i, h] = (p @ v) / p.sum()
            spread[i, h] = (p @ np.abs(v)) / p.sum()
            lse[i, h] = top + np.log(p.sum())
            size[i, h] = (np.abs(k) @ np.abs(q[i, h])).max()
    return out, lse, spread, size


def lora(x, Y, adapters, offsets, of):
    """adapters: [(A [r, K], B [N, r], scale)] -> (out, sum of the magnitudes that were added)."""
    out, size = Y.astype(np.float64).copy(), np.abs(Y).astype(np.float64)
    for s, a in enumerate(of):
        if not 0 <= a < len(adapters):
            continue
        A, B, scale = adapters[a]
        rows = slice(offsets[s], offsets[s + 1])
        out[rows] += scale * (x[rows] @ A.T) @ B.T
        size[rows] += abs(scale) * (np.abs(x[rows]) @ np.abs(A.T)) @ np.abs(B.T)
    return out, size
