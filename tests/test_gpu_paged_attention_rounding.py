"""Attention of many rows: what the rounding of the probabilities does to a row's largest weight, it does to both sides of the quotient."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as O

from .test_gpu_paged_attention import B, TYPES, _case, _np, _run  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,kv,hq,workspace", [(40, 300, 2, False), (150, 400, 1, False), (40, 1500, 2, True)])
def test_a_weight_that_is_most_of_a_row(B, dtype, new, kv, hq, workspace):
    """Two keys count: one of the first tile, and a later one whose score is above by less than what makes the kernel take a new reference.  With weights w_j each
    off by a factor of 1 + d_j, |d_j| <= u (the rounding) + 2 e (its score's error) the quotient is off by sum w_j d_j (v_j - o) <= (u + 2 e) sum w_j |v_j - o|; the sums' own
    errors (kv + 64) 2^-23, and the result's rounding u |o|.  (Were the denominator's weights not rounded the error would be u |o| more.)"""
    c = _case(dtype, [(new, kv)], hq, 1, 64, 16)
    g = np.random.default_rng(5)
    tt, u, tiny = TYPES[dtype]
    late = kv - new - 3
    at = lambda j: (int(c["table"][0, j // 16]), j % 16)
    for j in range(kv):
        c["kc"][at(j)] = 0
    c["kc"][at(3)][0, 0], c["kc"][at(late)][0, 1] = 1, 1
    lag = g.uniform(4.5, 7.5, (new, hq))
    q = np.zeros((new, hq, 64))
    q[..., 1] = 30.0
    q[..., 0] = 30.0 - lag
    c["q"] = torch.from_numpy(q).to(tt)
    scale = math.log(2.0)     # (scores are powers of two)
    got, s = _run(B, c, True, 0, workspace, scale=scale)
    q, k, v = _np(c["q"]), np.nan_to_num(_np(c["kc"])), np.nan_to_num(_np(c["vc"]))
    pages = c["table"][0][np.arange(kv) // 16]
    k, v = k[pages, np.arange(kv) % 16, 0], v[pages, np.arange(kv) % 16, 0]
    worst = 0.0
    for t in range(new):
        sees = np.arange(kv) <= kv - new + t
        for h in range(hq):
            x = np.where(sees, (k @ q[t, h]) * float(np.float32(scale)), -np.inf)
            w = np.exp(x - x.max())
            w /= w.sum()
            o = w @ v
            e = (64 + 4) * 2.0 ** -24 * 30 * scale + 2.0 ** -21
            tol = (u + 2 * e) * (w[:, None] * np.abs(v - o)).sum(0) * 1.01 + (kv + 64) * 2.0 ** -23 * (w @ np.abs(v)) + u * np.abs(o) * 1.01 + tiny
            worst = max(worst, float((np.abs(_np(got[t, h]) - o) / tol).max()))
    assert worst <= 1, worst


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("new,off", [(1, 2.0 ** -6), (40, 2.0 ** -3)])
def test_many_small_weights_of_fp16(B, new, off, workspace):
    """One key ahead of 20000 others by 2^25.5: their weights together are 0.04 %, and each is below half of fp16's least number, 2^-24.  Taken 2^8 larger (many rows:
    2^4) a weight of 2^-25.5 is held to half of 2^-24 / 2^-17.5 (2^-21.5): 2^-7.5 and 2^-3.5 of it."""
    kv = 20000
    c = _case("f16", [(new, kv)], 2, 1, 64, 16)
    c["kc"].zero_()
    c["q"].zero_()
    c["q"][..., 0] = 25.5
    first = int(c["table"][0, 0])
    c["kc"][first, 5, 0, 0] = 1
    c["vc"].fill_(1000.0)
    c["vc"][first, 5] = 0
    got, _ = _run(B, c, True, 0, workspace, scale=math.log(2.0))
    seen = np.arange(kv - new, kv).astype(np.float64)           # others than the first that a token sees
    w = seen * 2.0 ** -25.5
    want = (1000.0 * w / (1 + w))[:, None, None]
    assert (np.abs(_np(got) - want) <= want * off + 2.0 ** -10).all()
