"""4-bit codes of weights of any size: none are lost to a least scale that is large beside them."""
import numpy as np
import pytest
import torch

from paper_1904_08368_amd.decoder import quantize4


@pytest.mark.parametrize("dtype,std", [(torch.float16, s) for s in (100.0, 1e-2, 1e-3, 1e-4, 2e-5, 1e-5)] +
                         [(torch.bfloat16, s) for s in (1e4, 1e-3, 1e-5, 1e-10, 1e-30)])
@pytest.mark.parametrize("n,k,group", [(5, 64, 32), (3, 72, 64)])
def test_small_and_large_weights_keep_their_codes(dtype, std, n, k, group):
    """Half a step for the code, half for the zero point's rounding, and 15 steps of the scale's own rounding: 2^-9 of it in bf16, 2^-12 in fp16, and there
    half of 2^-24 at most where it is not normal."""
    w = (torch.from_numpy(np.random.default_rng(1).standard_normal((n, k))) * std).to(dtype)
    codes, scales, zeros = quantize4(w, group)
    c, of = torch.stack((codes & 15, codes >> 4), 2).view(n, k).double(), torch.arange(k) // group
    s, z = scales.double()[:, of], zeros.double()[:, of]
    rounding = torch.maximum(s * 2.0 ** -9, torch.full_like(s, 2.0 ** -25 if dtype == torch.float16 else 0.0))
    assert ((c - z) * s - w.double()).abs().le(s * 1.001 + 15 * rounding).all()
    # the range of each group is 15 steps: most of the codes are in use
    assert scales.double().min() < 8 * std and (len(torch.unique(c)) > 12 or std <= 1e-5)
    assert ((c - z) * s - w.double()).norm() < 0.2 * w.double().norm()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_group_of_zeros(dtype):
    codes, scales, zeros = quantize4(torch.zeros(2, 64, dtype=dtype), 32)
    assert torch.isfinite(scales.float()).all() and (scales > 0).all()
    c = torch.stack((codes & 15, codes >> 4), 2).view(2, 2, 32)
    assert (c == zeros[..., None]).all()
