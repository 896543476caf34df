"""Dense with 4-bit weights where x holds infinities or numbers near the end of the type's range: each output is what the formula gives, whatever the number of
rows beside it."""
import numpy as np
import pytest
import torch

from oracle import attention as O

from .test_gpu_dense_w4 import B, DEV, TYPES, _case, _np  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


def _layer(B, dtype, m, n, k, group, zeros, seed=3):
    g = np.random.default_rng(seed)
    tt = TYPES[dtype][0]
    groups = (k + group - 1) // group
    codes = g.integers(0, 256, (n, k // 2)).astype(np.uint8)
    scales = torch.from_numpy(g.uniform(0.001, 0.01, (n, groups)).astype(np.float32)).to(tt)
    zp = g.integers(0, 16, (n, groups)).astype(np.uint8) if zeros else None
    x = torch.from_numpy(g.standard_normal((m, k)).astype(np.float32)).to(tt)
    c = np.empty((n, k))
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    of = np.arange(k) // group
    w = (c - (8.0 if zp is None else zp[:, of])) * _np(scales)[:, of]
    return x, w, codes, scales, zp


def _run(B, x, codes, scales, zp, group, y=None, residual=None):
    up = lambda a: None if a is None else (a if torch.is_tensor(a) else torch.from_numpy(a)).to(DEV)
    xd, zd, rd = up(x), up(zp), up(residual)
    y = torch.empty((x.shape[0], codes.shape[0]), dtype=x.dtype, device=DEV) if y is None else y
    d = B.qdense_w4_desc(xd, y, group, zd, None, rd)
    packed = torch.empty(B.relay_qdense_w4_packed_bytes(d), dtype=torch.uint8, device=DEV)
    B.relay_prepack_qdense_w4(d, up(codes), up(scales), zd, packed)
    B.relay_qdense_w4(d, xd, packed, None, rd, y)
    torch.cuda.synchronize()
    return y


def _products(x, w):
    """One row of x times the weights, product by product (an infinity times zero is a NaN, as are infinities of both signs)."""
    with np.errstate(invalid="ignore"):
        return (x[None, :] * w).sum(1)


SHAPES = [(1, 40, 264, 64), (1, 33, 1024, 128), (3, 50, 520, 96), (4, 64, 256, 32), (9, 75, 264, 64), (16, 5000, 256, 128), (40, 70, 520, 32), (200, 97, 1000, 128),
          (1100, 1500, 128 * 16, 128), (1100, 1501, 128 * 17 + 8, 32), (1100, 1500, 128 * 9, 64), (2100, 2500, 256, 128), (1020, 2050, 128 * 17 + 8, 64), (1020, 2050, 128 * 18 + 72, 128)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("m,n,k,group", SHAPES)
def test_an_infinity_in_x(B, dtype, zeros, m, n, k, group):
    x, w, codes, scales, zp = _layer(B, dtype, m, n, k, group, zeros)
    clean = _run(B, x, codes, scales, zp, group)
    bad, rows = x.clone(), sorted({m - 1, m // 2})
    for i, r in enumerate(rows):
        bad[r, (k - 1) if i else k // 3] = float("-inf") if i else float("inf")
    got = _run(B, bad, codes, scales, zp, group)
    others = [r for r in range(m) if r not in rows]
    assert torch.equal(got[others], clean[others])
    for r in rows:
        want, out = _products(_np(bad[r]), w), _np(got[r])
        assert not np.isfinite(want).any()
        assert np.array_equal(want, out, equal_nan=True), (want[:8], out[:8])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m,n,k,group", [(1, 40, 264, 64), (9, 75, 264, 64), (200, 97, 1000, 128), (1100, 1500, 2048, 128)])
def test_infinities_of_both_signs_and_a_nan(B, dtype, m, n, k, group):
    x, w, codes, scales, zp = _layer(B, dtype, m, n, k, group, True)
    x[m - 1, 1], x[m - 1, k - 2] = float("inf"), float("-inf")
    if m > 1:
        x[0, k // 2] = float("nan")
    got = _run(B, x, codes, scales, zp, group)
    assert np.array_equal(_products(_np(x[m - 1]), w), _np(got[m - 1]), equal_nan=True)
    assert m == 1 or torch.isnan(got[0]).all()


@pytest.mark.parametrize("m,n,k,group", [(1, 40, 264, 64), (9, 75, 264, 64), (200, 97, 1000, 128), (1100, 1500, 2048, 128), (1100, 1500, 2048, 32), (1020, 2050, 128 * 17 + 8, 64)])
def test_numbers_near_the_end_of_the_range(B, m, n, k, group):
    """bf16 reaches 3.4e38: 31 times as much does not, the weights' products with it do.  One such number to a row: the others, and the fp32 sums' errors,
    are 1e-30 beside it.  The rounding of the weight to fp32 and of the product 2^-23, of the result 2^-8."""
    x, w, codes, scales, zp = _layer(B, "bf16", m, n, k, group, True)
    rows = sorted({0, m - 1})
    for i, r in enumerate(rows):
        x[r, k // 2 + i] = 3e38 if i else -2.5e38
    residual = torch.ones((m, n), dtype=torch.bfloat16)
    y = residual.to(DEV)
    got = _run(B, x, codes, scales, zp, group, y, y)   # in place
    for r in rows:
        want, out = _np(x[r]) @ w.T, _np(got[r])
        assert np.isfinite(out).all()
        assert (np.abs(out - want - 1) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * np.abs(want) + 1.0).all()


def test_an_infinite_scale_stays_in_its_unit(B):
    x, w, codes, scales, zp = _layer(B, "f16", 5, 48, 256, 64, False)
    clean = _run(B, x, codes, scales, zp, 64)
    scales[7, 2] = float("inf")
    got = _run(B, x, codes, scales, zp, 64)
    others = [j for j in range(48) if j != 7]
    assert torch.equal(got[:, others], clean[:, others]) and not torch.isfinite(got[:, 7]).any()
