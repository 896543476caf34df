"""Rows whose logits lie within 2^-90 of each other: bins have no width there, all tokens are in the first, and every one of them counts."""
import pytest
import torch

from .test_gpu_sample import B, DEV, TYPES, _check  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(1, 3), (2, 1000), (3, 1999), (2, 40000), (300, 77)])
@pytest.mark.parametrize("power", [-91, -100, -120])
def test_tiny_differences(B, dtype, rows, vocab, power):
    """k 2^power for k of 0 .. 127, in a mixed order: all weights are 1, and the order of the values names the token."""
    i = torch.arange(rows * vocab, device=DEV).view(rows, vocab)
    logits = ((i * 37 % 128).double() * 2.0 ** power).to(TYPES[dtype])
    for more in (dict(), dict(top_p=0.5), dict(top_k=2), dict(top_k=60), dict(top_k=600, top_p=0.9), dict(min_p=0.5)):
        for u in (0.0, 0.3, 0.99):
            _check(B, logits, uniform=u, **more)
            _check(B, -logits, uniform=u, **more)
        # min-p of 1 keeps the largest alone: exp of anything below zero is less than 1, which 64 bits of the weight itself (and so the oracle) do not tell; the kernels compare exponents.
        _, args = _check(B, logits, uniform=0.5, top_k=1)
        tokens, probs = args[6].clone(), args[7].clone()
        B.relay_sample(B.sample_desc(logits), logits, None, None, None, torch.ones(rows, device=DEV), torch.full((rows,), 0.0, device=DEV), tokens, probs, args[8])
        torch.cuda.synchronize()
        many = (logits == logits.amax(1, keepdim=True)).sum(1)
        assert torch.equal(tokens, args[6]) and (probs - 1 / many).abs().max() <= 2.0 ** -24
