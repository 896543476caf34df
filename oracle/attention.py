"""CPU oracle -- TEST INFRASTRUCTURE ONLY: the operators of a cache-served attention layer in 64 bits, straight from their formulas.

Tensors are numpy arrays of float64 (values of the 16-bit types are exact in it).  `attention` and `dense_w4` also return what a bound of
the rounding errors needs: sums of magnitudes beside the sums.
"""
from __future__ import annotations

import math

import numpy as np


def rope_frequencies(rotary_dim, base, scaling="plain", factor=1.0, slow=1.0, fast=32.0, original_len=1.0):
    i = np.arange(rotary_dim // 2, dtype=np.float64)
    if scaling == "base":
        base = base * factor ** (rotary_dim / (rotary_dim - 2))
    f = base ** (-2.0 * i / rotary_dim)
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":
        turns = original_len * f / (2 * math.pi)
        g = np.clip((turns - slow) / (fast - slow), 0.0, 1.0)
        f = (1 - g) * f / factor + g * f
    return f


def rope(x, cos_sin, positions, style, inverse=False):
    """x [tokens, heads, dim]; cos_sin [rows, rd/2, 2]; style "half" or "interleaved"."""
    y = np.array(x, dtype=np.float64)
    rd = 2 * cos_sin.shape[1]
    for t, p in enumerate(positions):
        for i in range(rd // 2):
            a, b = (i, i + rd // 2) if style == "half" else (2 * i, 2 * i + 1)
            c, s = (float(v) for v in cos_sin[p, i]) if 0 <= p < len(cos_sin) else (math.nan, math.nan)
            if inverse:
                s = -s
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
    return y


def attention(q, k_cache, v_cache, page_table, q_starts, kv_lens, scale, causal=True, window=0):
    """q [tokens, Hq, D]; caches [pages, page_size, Hkv, D].  Returns (out, mag, spread, keys): mag = sum_j p_j |v_j| per element, spread = the
    largest sum_d |q_d k_d| * scale of a row's scores, keys = how many keys the row sees."""
    tokens, hq, dim = q.shape
    pages, ps, hkv, _ = k_cache.shape
    out, mag = np.zeros_like(q), np.zeros_like(q)
    spread, keys = np.zeros((tokens, hq)), np.zeros((tokens, hq))
    for b in range(len(kv_lens)):
        n0, n1, kv = int(q_starts[b]), int(q_starts[b + 1]), int(kv_lens[b])
        place = [(int(page_table[b, j // ps]), j % ps) for j in range(kv)]
        for t in range(n0, n1):
            p = kv - (n1 - n0) + (t - n0)
            seen = [j for j in range(kv) if (not causal or j <= p) and (not window or j > p - window) and 0 <= place[j][0] < pages]
            if not seen:
                continue
            pg, sl = np.array([place[j][0] for j in seen]), np.array([place[j][1] for j in seen])
            for h in range(hq):
                k, v = k_cache[pg, sl, h // (hq // hkv)], v_cache[pg, sl, h // (hq // hkv)]
                with np.errstate(all="ignore"):
                    s = (k * q[t, h]).sum(1) * scale
                    w = np.exp(s - s.max())
                    w = w / w.sum()
                    out[t, h] = (w[:, None] * v).sum(0)
                    mag[t, h] = (w[:, None] * np.abs(v)).sum(0)
                    spread[t, h] = (np.abs(k) * np.abs(q[t, h])).sum(1).max() * abs(scale)
                keys[t, h] = len(seen)
    return out, mag, spread, keys


def attention_tolerance(out, mag, spread, keys, vmax, dim, u, tiny):
    """Bound of |result - out| for scores, softmax and sums in fp32 and probabilities rounded to the output's type (unit roundoff u,
    smallest spacing `tiny`), from the errors of each step:
      a score's error e_s <= (dim + 4) 2^-24 spread (the products' sum and the scaling) moves its probability by a factor 1 + e_s, and so does
      the exponential's own 2^-21; the sums over the keys and their rescaling (keys + 64) 2^-23; the rounding of the probabilities u, or
      where they are small an absolute tiny/2 each beside a largest probability of 1; the result's own rounding u |out| + tiny/2."""
    e_s = (dim + 4) * 2.0 ** -24 * spread[..., None] + 2.0 ** -21
    rel = u + 2 * e_s + (keys[..., None] + 64) * 2.0 ** -23
    return rel * mag * 1.01 + u * np.abs(out) * 1.01 + keys[..., None] * tiny / 2 * vmax + tiny / 2


def dense_w4(x, codes, scales, zeros, group, bias=None, residual=None, relu=False):
    """x [m, k]; codes uint8 [n, k/2]; scales [n, groups]; zeros [n, groups] or None.  Returns (y, bound): the bound of fp32 sums,
    group by group with numbers 16 + code and 16 + zero, then over the groups and the tail."""
    m, k = x.shape
    n, groups = scales.shape
    c = np.empty((n, k))
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    y, err, size = np.zeros((m, n)), np.zeros((m, n)), np.zeros((m, n))
    for g in range(groups):
        i = slice(g * group, min(k, (g + 1) * group))
        z = np.full((n, 1), 8.0) if zeros is None else zeros[:, g:g + 1].astype(np.float64)
        part = (x[:, i] @ (c[:, i] - z).T) * scales[:, g]
        within = (np.abs(x[:, i]) @ (c[:, i] + z + 32.0).T) * np.abs(scales[:, g])
        y += part
        size += np.abs(part)
        err += (min(group, k) + 4) * 2.0 ** -24 * within
    if bias is not None:
        y, size = y + bias, size + np.abs(bias)
    if residual is not None:
        y, size = y + residual, size + np.abs(residual)
    if relu:
        y = np.maximum(y, 0)
    return y, err + (groups + 8) * 2.0 ** -24 * size
