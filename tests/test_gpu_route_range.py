"""Router products past the range of 32 bits, which is bf16's own: they are exact in 64, for few tokens as for more."""
import numpy as np
import pytest
import torch

from .test_gpu_route import B, DEV, _check, scratch  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [1, 2, 4, 5, 20])
@pytest.mark.parametrize("power", [65, 100, 126])
@pytest.mark.parametrize("channels", [64, 4096])
def test_large_products(B, scratch, tokens, power, channels):
    """A logit is (m - n) 2^(2 power) from one product of m and one of -n: sums of whole multiples of one number, exact in 64 bits in any order, zero where m = n.  In 32 bits each
    product is an infinity, and their sum a NaN."""
    up = lambda a: torch.from_numpy(a).to(torch.bfloat16).to(DEV)   # (all numbers below have few bits)
    x, w = np.zeros((tokens, channels)), np.zeros((9, channels))
    a, b = 3, channels - 5
    x[:, a], x[:, b] = 2.0 ** power, 2.0 ** power
    m, n = np.array([1, 2, 3, 1, 1, 3, 2, 1, 2]), np.array([1, 1, 3, 2, 0, 1, 2, 3, 3])
    w[:, a], w[:, b] = m * 2.0 ** power, -n * 2.0 ** power
    for score in ("softmax", "sigmoid"):
        for top_k in (1, 4, 9):
            _, chosen, weights = _check(B, scratch, up(x), up(w), None, top_k, score, normalize=False)
            assert torch.isfinite(weights).all()
            if score == "sigmoid" and top_k == 9:   # m > n: 1; equal: a half; less: nothing
                assert chosen[0].tolist() == [1, 4, 5, 0, 2, 6, 3, 7, 8] and weights[0].tolist() == [1, 1, 1, 0.5, 0.5, 0.5, 0, 0, 0]
