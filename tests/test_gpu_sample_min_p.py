"""min-p at its upper end where several tokens share the maximum: at 1 all of them are kept, above it only the first."""
import pytest
import torch

from .test_gpu_sample import B, DEV, TYPES, _check  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(1, 9), (3, 1000), (2, 131073), (300, 1003)])
@pytest.mark.parametrize("more", [dict(), dict(top_k=4), dict(top_k=5000, temperature=0.7), dict(top_p=0.9), dict(temperature=3.0)])
def test_ties_at_the_maximum(B, dtype, rows, vocab, more):
    g = torch.Generator(device=DEV).manual_seed(vocab)
    logits = torch.randn((rows, vocab), generator=g, device=DEV).clamp_(max=1.0)
    for i in range(rows):
        logits[i, torch.tensor([i % 3 + 1, vocab // 2, vocab - 1], device=DEV)] = 4.0
    logits = logits.to(TYPES[dtype])
    for u in (0.1, 0.5, 0.9):
        for min_p, kept in ((1.0, 3), (1.0000001, 1), (7.0, 1), (float("inf"), 1)):
            _, args = _check(B, logits, uniform=u, min_p=min_p, **more)
            tokens, probs = args[6], args[7]
            if kept == 1:
                assert tokens.tolist() == [i % 3 + 1 for i in range(rows)] and (probs == 1).all()
            elif "top_p" not in more:   # (top-p may leave fewer of them)
                assert (probs == 1 / 3).all() and (u > 0.34) == (int(tokens[0]) != 1)
