"""The mixture-of-experts half of a layer -- oracle.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__``).  Plain NumPy in float64, one loop per row,
written from the formulas; nothing here is rounded.
"""
from __future__ import annotations

import numpy as np

from . import mxfp4


def _rms(v, w, eps, offset):
    return v / np.sqrt(np.mean(v * v) + eps) * (offset + w)


def block_norm(y, r, post=None, pre=None, gate=None, index=None, eps=1e-6, offset=0.0, a=1.0, b=1.0):
    """(r', h or None) of rows y, r (either may be None); index: gate row of each row."""
    lead = y if y is not None else r
    sums = np.zeros(lead.shape)
    h = None if pre is None else np.zeros(lead.shape)
    for m in range(len(lead)):
        u = np.zeros(lead.shape[1])
        if y is not None:
            u = _rms(y[m], post, eps, offset) if post is not None else y[m].copy()
            if gate is not None:
                g = int(index[m]) if index is not None else m if len(gate) > 1 else 0
                if 0 <= g < len(gate):
                    u = u * gate[g]
        sums[m] = b * u + (a * r[m] if r is not None else 0)
        if pre is not None:
            h[m] = _rms(sums[m], pre, eps, offset)
    return sums, h


def route(logits, k, sigmoid=False, bias=None, renormalize=True, scale=1.0):
    """(ids, weights) of logits [M, E]."""
    M, E = logits.shape
    ids, weights = np.zeros((M, k), np.int64), np.zeros((M, k))
    for m, l in enumerate(logits):
        with np.errstate(all="ignore"):
            s = 1 / (1 + np.exp(-l)) if sigmoid else np.exp(l - np.max(l)) / np.sum(np.exp(l - np.max(l)))
        key = (s + (0 if bias is None else bias)) if sigmoid else l
        order = sorted(range(E), key=lambda e: (bool(np.isnan(key[e])), -key[e] if not np.isnan(key[e]) else 0, e))
        ids[m] = order[:k]
        w = s[ids[m]]
        if renormalize:
            if not sigmoid:                       # of the chosen alone: others' infinities and NaN do not count
                c = l[ids[m]]
                w = np.exp(c - c[0])
            w = w / np.sum(w)
        weights[m] = w * scale
    return ids, weights


def dequantized(codes, scales):
    """[..., K] of packed codes [..., K / 2] and scales [..., K / 32]."""
    return mxfp4.mx_dequantize(mxfp4.unpack_codes(codes), scales)


def layer(x, ids, weights, gate_up, down, k_tail):
    """x [M, H], dequantized gate_up [E, 2 I, H] and down [E, N, I + k_tail] -> y [M, N] and, for error
    bounds, of what each y adds the magnitudes' sum and the root of the squares' sum, and how far y
    moves when every first sum moves by its own magnitudes' sum."""
    M, E, N = len(x), len(down), down.shape[1]
    I = down.shape[2] - k_tail
    y, size, square, reach = (np.zeros((M, N)) for _ in range(4))
    for m in range(M):
        for e, w in zip(ids[m], weights[m]):
            if not 0 <= e < E:
                continue
            g, u = gate_up[e, :I] @ x[m], gate_up[e, I:] @ x[m]
            with np.errstate(over="ignore"):
                sg = g / (1 + np.exp(-g))
            h = sg * u
            # SiLU's slope is below 1.1
            ag, au = np.abs(gate_up[e, :I]) @ np.abs(x[m]), np.abs(gate_up[e, I:]) @ np.abs(x[m])
            far = 1.1 * ag * np.abs(u) + np.abs(sg) * au
            h, far = (np.concatenate([v, v[I - k_tail:]]) for v in (h, far))
            y[m] += w * (down[e] @ h)
            size[m] += abs(w) * (np.abs(down[e]) @ np.abs(h))
            square[m] += w * w * (down[e] ** 2 @ h ** 2)
            reach[m] += abs(w) * (np.abs(down[e]) @ far)
    return y, size, np.sqrt(square), reach
