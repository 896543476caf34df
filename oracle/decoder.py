"""CPU oracle -- TEST INFRASTRUCTURE ONLY: a decoder's operators beside its attention layer in 64 bits, straight from their formulas.

Tensors are numpy arrays of float64 (values of the 16-bit types are exact in it).  Beside its results each function returns what a test of
rounded results needs: a bound of the errors of 32-bit steps, formed step by step beside the values.
"""
from __future__ import annotations

import math

import numpy as np

from . import attention

E32 = 2.0 ** -24   # half a step of fp32, relative
DEPTH = 64         # additions that a term of a row's sum passes through at most: 32 of a thread, 6 of a wave, 16 of waves


def norm(v, dv, kind, eps, weight=None, bias=None):
    """v [tokens, channels] with absolute errors dv -> the normed rows and their errors; kind "rms" or "layer"."""
    w = np.ones(v.shape[1]) if weight is None else weight.astype(np.float64)
    z = np.zeros(v.shape[1]) if bias is None else bias.astype(np.float64)
    c, dc = v, dv
    if kind == "layer":
        m = v.mean(1, keepdims=True)
        dm = dv.mean(1, keepdims=True) + (DEPTH + 2) * E32 * (np.abs(v) + dv).mean(1, keepdims=True)
        c, dc = v - m, dv + dm + E32 * (np.abs(v - m) + dv + dm)
    q = (c * c).mean(1, keepdims=True)
    dq = (2 * np.abs(c) * dc + dc * dc).mean(1, keepdims=True)
    dq = dq + (DEPTH + 2) * E32 * (q + dq)
    k = 1 / np.sqrt(q + eps)
    dk = 1 / np.sqrt(np.maximum(q - dq, 0) + eps) - k    # (the side on which the root is steeper)
    dk = dk + 4 * E32 * (k + dk)
    out = c * k * w + z
    err = ((np.abs(c) + dc) * (k + dk) - np.abs(c) * k) * np.abs(w)
    return out, err + 3 * E32 * (np.abs(c * k * w) + err + np.abs(z))


def residual_norm(x, residual=None, gate=None, post=None, pre=None, branch_scale=1.0, residual_scale=1.0):
    """post, pre: None or (kind, eps, weight, bias).  Returns (s, ds, y, dy): the sum before its rounding and the normed sum."""
    v, dv = x, np.zeros_like(x)
    if post is not None:
        v, dv = norm(v, dv, *post)
    if gate is not None:
        v, dv = v * gate, dv * np.abs(gate) + E32 * (np.abs(v) + dv) * np.abs(gate)
    v, dv = v * branch_scale, (dv + E32 * (np.abs(v) + dv)) * abs(branch_scale)
    if residual is not None:
        v = v + residual * residual_scale
        dv = dv + E32 * (np.abs(v) + dv)
    y, dy = (None, None) if pre is None else norm(v, dv, *pre)
    return v, dv, y, dy


def route(x, w, top_k, score="softmax", bias=None, normalize=True, scale=1.0):
    """chosen and weights [tokens, top_k]."""
    l = x @ w.T
    if score == "softmax":
        s = np.exp(l - l.max(1, keepdims=True))
        s /= s.sum(1, keepdims=True)
    else:
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-l))
    by = s if bias is None else s + bias.astype(np.float64)
    chosen = np.argsort(-by, axis=1, kind="stable")[:, :top_k]
    weights = np.take_along_axis(s, chosen, 1)
    if normalize:
        total = weights.sum(1, keepdims=True)
        weights = np.where(total == 0, 0.0, weights / np.where(total == 0, 1.0, total))
    return chosen, weights * scale


def experts(x, chosen, weights, gate_up, down, inter, group, act="silu", residual=None, u=2.0 ** -11, tiny=2.0 ** -24):
    """gate_up, down: (codes, scales, zeros) of all experts' units one behind the other; u, tiny: half a step and the least step of the type that h is
    rounded to.  Returns y [tokens, channels] before its rounding and a bound of its error: of the sums of 32 bits (oracle.attention.dense_w4), through the activation
    (whose slope is 1.13 at most, its own functions off by 8 half-steps), the product and its rounding, through the second product, and times the weight (which is added
    up in one rounding with its part)."""
    tokens, channels = x.shape
    part = lambda w, first, n: tuple(None if a is None else a[first:first + n] for a in w)
    y, err = np.zeros((tokens, channels)), np.zeros((tokens, channels))
    size = np.zeros((tokens, channels))
    for e in sorted({int(c) for c in chosen.ravel() if 0 <= c < len(gate_up[0]) // (2 * inter)}):
        tok, slot = np.nonzero(chosen == e)
        (g, dg), (v, dv) = (attention.dense_w4(x[tok], *part(gate_up, (2 * e + i) * inter, inter), group) for i in (0, 1))
        with np.errstate(over="ignore"):
            a = g / (1 + np.exp(-g)) if act == "silu" else 0.5 * g * np.vectorize(math.erfc)(-g * math.sqrt(0.5))
        da = 1.13 * dg + 8 * E32 * (np.abs(a) + dg)
        h = a * v
        dh = (np.abs(a) + da) * (np.abs(v) + dv) - np.abs(h)
        dh = dh + E32 * (np.abs(h) + dh)
        dh = dh + u * (np.abs(h) + dh) + tiny
        wd = part(down, e * channels, channels)
        out, bound = attention.dense_w4(h, *wd, group)
        codes = np.empty((channels, inter))
        codes[:, 0::2], codes[:, 1::2] = wd[0] & 15, wd[0] >> 4
        which = np.arange(inter) // group
        mag = np.abs((codes - (8.0 if wd[2] is None else wd[2][:, which].astype(np.float64))) * wd[1][:, which])
        moved = dh @ mag.T
        w = weights[tok, slot][:, None]
        np.add.at(y, tok, w * out)
        np.add.at(err, tok, np.abs(w) * (1.02 * bound + moved))
        np.add.at(size, tok, np.abs(w) * (np.abs(out) + bound + moved))
    if residual is not None:
        y, size = y + residual, size + np.abs(residual)
    return y, err + (chosen.shape[1] + 2) * E32 * size


def sample(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, uniform=0.0):
    """One row: the token, its probability among the kept, and how many are kept."""
    l = np.where(np.isnan(logits), -np.inf, logits)
    if not (l > -np.inf).any():
        return -1, 0.0, 0
    order = np.argsort(-l, kind="stable")
    if math.isnan(temperature):
        temperature = 1.0
    if temperature <= 0:
        return int(order[0]), 1.0, 1
    d = np.where(l[order] == l[order[0]], 0.0, l[order] - (l[order[0]] if np.isfinite(l[order[0]]) else np.finfo(np.float64).max))
    with np.errstate(under="ignore"):
        w = np.where(np.isneginf(d), 0.0, np.exp(np.where(np.isneginf(d), 0.0, d / temperature)))
    n = len(w)
    if 0 < top_k < n:
        n = top_k
    if top_p < 1:
        mass = np.cumsum(w[:n])
        n = int(np.searchsorted(mass, top_p * mass[-1], side="left")) + 1 if top_p > 0 else 1
    if min_p > 0:
        n = max(1, min(n, int((w >= min_p).sum())))
    cum = np.cumsum(w[:n])
    u = 0.0 if math.isnan(uniform) else min(max(uniform, 0.0), 1 - 2.0 ** -24)
    at = int(np.searchsorted(cum, u * cum[-1], side="right"))
    return int(order[at]), float(w[at] / cum[-1]), n
