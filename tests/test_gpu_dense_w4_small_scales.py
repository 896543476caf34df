"""Dense with 4-bit weights whose scales are not normal numbers of fp16, or small ones of bf16: they count as what they are."""
import numpy as np
import pytest
import torch

from oracle import attention as O
from paper_1904_08368_amd.decoder import Dense4, quantize4

from .test_gpu_dense_w4 import B, DEV, TYPES, _np  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,std", [("f16", 2e-5), ("bf16", 1e-20)])
@pytest.mark.parametrize("m,n,k,group", [(1, 40, 264, 64), (3, 40, 256, 128), (9, 75, 520, 32), (200, 97, 1000, 128), (2100, 2500, 256, 128)])
def test_small_scales(B, dtype, std, m, n, k, group):
    tt, u, tiny = TYPES[dtype]
    g = np.random.default_rng(7)
    w = torch.from_numpy(g.standard_normal((n, k)) * std).to(tt)
    x = torch.from_numpy(g.standard_normal((m, k)) * (1.0 / std) ** 0.5).to(tt)
    codes, scales, zeros = quantize4(w, group)
    assert scales.double().max() < 2.0 ** -14
    y = torch.empty((m, n), dtype=tt, device=DEV)
    Dense4(codes.to(DEV), scales.to(DEV), zeros.to(DEV), group, k)(x.to(DEV), y)
    torch.cuda.synchronize()
    want, bound = O.dense_w4(_np(x), codes.numpy(), _np(scales), zeros.numpy(), group)
    assert (np.abs(_np(y) - want) <= bound + u * (np.abs(want) + bound) + tiny).all() and np.abs(want).max() > 0
