"""An attention layer with its input added and without, in both types: the two differ by the input and the roundings of each."""
import pytest
import torch

from .test_gpu_decoder import D, DEV, DIM, HKV, TYPES, _np  # noqa: F401  (D is the fixture)
from .test_gpu_decoder_blocks import WIDTH, _model

pytestmark = pytest.mark.gpu
E32 = 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_with_and_without_the_input(D, dtype):
    """branch = round(v), with_input = round(v + n) of one sum v in 32 bits.  So |v - branch| <= u / (1 - u) |branch| + tiny =: d, and with_input is off branch + n by d and, of at most
    |branch + n| + d, half a step u of the type and one of 32 bits (the addition)."""
    decoder, _, _ = _model(D, dtype)
    _, u, tiny = TYPES[dtype]
    cache = D.PagedCache(2, 64, 16, HKV, DIM, TYPES[dtype][0])
    ids = [cache.open() for _ in range(3)]
    g = torch.Generator(device=DEV).manual_seed(6)
    for new in ([70, 5, 33], [1, 1, 1]):
        step = D.Step(cache, 3, sum(new), max(new), 200)
        step.extend(ids, new)
        n = torch.randn((step.tokens, WIDTH), generator=g, device=DEV).to(TYPES[dtype][0])
        for i, block in enumerate(decoder.blocks):
            branch, both = torch.empty_like(n), torch.empty_like(n)
            block.attention(n, i, step, branch, add=False)
            block.attention(n, i, step, both)
            want = _np(branch) + _np(n)
            d = u / (1 - u) * abs(_np(branch)) + tiny
            tol = d + (u + E32) * (abs(want) + d) + tiny
            off = abs(_np(both) - want)
            assert (off <= tol).all() and abs(_np(branch)).max() > 0.1, float((off / tol).max())
