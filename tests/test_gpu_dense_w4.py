"""Dense with 4-bit weights against 64 bits: rows from one to many, odd units and reductions, every group size, zero points, the fused tail."""
import numpy as np
import pytest
import torch

from oracle import attention as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": (torch.float16, 2.0 ** -11, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -133)}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1904_08368_amd import binding
    return binding


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _case(B, dtype, m, n, k, group, zeros=False, bias=False, residual=False, relu=False, mean=0.0, xpad=0, ypad=0, seed=0):
    g = np.random.default_rng(seed + m + 3 * n + 7 * k)
    tt, u, tiny = TYPES[dtype]
    groups = (k + group - 1) // group
    codes = g.integers(0, 256, (n, k // 2)).astype(np.uint8)
    scales = torch.from_numpy((g.uniform(0.5, 2.0, (n, groups)) / np.sqrt(k) / 4).astype(np.float32)).to(tt)
    zp = g.integers(0, 16, (n, groups)).astype(np.uint8) if zeros else None
    x = torch.from_numpy((g.standard_normal((m, k + xpad)) + mean).astype(np.float32)).to(tt)
    res = torch.from_numpy(g.standard_normal((m, n + ypad)).astype(np.float32)).to(tt) if residual else None
    b = g.standard_normal(n).astype(np.float32) if bias else None
    up = lambda a: None if a is None else (a if torch.is_tensor(a) else torch.from_numpy(a)).to(DEV)
    xd, y = up(x)[:, :k], torch.full((m, n + ypad), 5.0, dtype=tt, device=DEV)
    rd = None if res is None else up(res)[:, :n]
    yv = y[:, :n]
    zd, bd = up(zp), up(b)
    d = B.qdense_w4_desc(xd, yv, group, zd, bd, rd, relu)
    packed = torch.full((B.relay_qdense_w4_packed_bytes(d),), 255, dtype=torch.uint8, device=DEV)
    B.relay_prepack_qdense_w4(d, up(codes), up(scales), zd, packed)
    B.relay_qdense_w4(d, xd, packed, bd, rd, yv)
    torch.cuda.synchronize()
    want, bound = O.dense_w4(_np(x)[:, :k], codes, _np(scales), zp, group, b, None if res is None else _np(res)[:, :n], relu)
    got = _np(yv)
    tol = bound + u * (np.abs(want) + bound) + tiny
    assert not np.isnan(got).any()
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
    assert (y[:, n:] == 5).all()
    return dict(d=d, x=xd, packed=packed, y=yv, bias=bd, res=rd)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m", [1, 2, 3, 7, 8, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 129, 200, 257])
@pytest.mark.parametrize("n,k,group", [(16, 128, 128), (40, 264, 64), (97, 1000, 32)])
def test_rows(B, dtype, m, n, k, group):
    _case(B, dtype, m, n, k, group, zeros=m % 2 == 1)


@pytest.mark.parametrize("n", [1, 15, 17, 31, 64, 127, 130, 1000])
@pytest.mark.parametrize("k,group", [(8, 32), (24, 64), (32, 32), (40, 32), (128, 32), (136, 128), (520, 96), (2048, 256), (4096, 4096), (5000, 64)])
@pytest.mark.parametrize("m", [1, 20])
def test_units_and_reductions(B, n, k, group, m):
    _case(B, "f16", m, n, k, group, zeros=True)
    _case(B, "bf16", m, n, k, group)


@pytest.mark.parametrize("m", [1, 5, 40, 150])
@pytest.mark.parametrize("zeros,bias,residual,relu", [(False, True, False, False), (True, False, True, False), (False, False, False, True), (True, True, True, True)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_tail(B, dtype, m, zeros, bias, residual, relu):
    _case(B, dtype, m, 75, 264, 32, zeros, bias, residual, relu)


@pytest.mark.parametrize("m", [1, 33, 130])
@pytest.mark.parametrize("xpad,ypad", [(8, 0), (24, 1), (0, 8)])
def test_strided_rows(B, m, xpad, ypad):
    _case(B, "f16", m, 70, 200, 64, True, True, True, xpad=xpad, ypad=ypad)


@pytest.mark.parametrize("m", [1, 9, 70])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_activations_with_a_mean(B, dtype, m):
    """Inputs of one sign, where the offset of the codes and its correction are largest."""
    _case(B, dtype, m, 64, 2048, 128, mean=4.0)


@pytest.mark.parametrize("m", [1, 2, 40])
def test_one_row_is_not_another(B, m):
    """An infinity or a NaN in one row of x stays in its row, and one unit's infinite scale in its unit."""
    s = _case(B, "f16", m + 1, 48, 256, 64)
    x = s["x"].clone()
    x[m, 3], x[m, 200] = float("inf"), float("nan")
    y = torch.empty_like(s["y"])
    B.relay_qdense_w4(s["d"], x, s["packed"], None, None, y)
    torch.cuda.synchronize()
    assert torch.equal(y[:m], s["y"][:m]) and torch.isnan(y[m]).all()


def test_residual_in_place(B):
    s = _case(B, "bf16", 3, 100, 136, 32, residual=True)
    y = s["res"].clone()
    B.relay_qdense_w4(s["d"], s["x"], s["packed"], None, y, y)
    torch.cuda.synchronize()
    assert torch.equal(y, s["y"])


def test_same_bits_on_every_call_and_stream(B):
    for m in (1, 20, 300):
        s = _case(B, "f16", m, 200, 1024, 128)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        y = torch.empty_like(s["y"])
        with torch.cuda.stream(side):
            B.relay_qdense_w4(s["d"], s["x"], s["packed"], None, None, y)
        side.synchronize()
        assert torch.equal(y, s["y"])


def test_no_rows(B):
    x, y = torch.empty((0, 64), dtype=torch.float16, device=DEV), torch.empty((0, 8), dtype=torch.float16, device=DEV)
    d = B.qdense_w4_desc(x, y, 32)
    packed = torch.zeros(B.relay_qdense_w4_packed_bytes(d), dtype=torch.uint8, device=DEV)
    B.relay_qdense_w4(d, x, packed, None, None, y)
