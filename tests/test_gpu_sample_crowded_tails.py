"""Rows that crowd into one bin and do not end with a whole 16-byte piece: what lies behind the last one is looked through like the rest."""
import numpy as np
import pytest
import torch

from .test_gpu_sample import B, DEV, TYPES, _check  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("vocab", [2049, 2055, 4780, 9178, 20001, 46503, 60007])
@pytest.mark.parametrize("kind", ["near", "few values", "outliers in the tail"])
def test_crowded_rows(B, dtype, vocab, kind):
    g = np.random.default_rng(vocab)
    l = g.standard_normal((3, vocab)) * 0.01
    if kind == "few values":
        l = np.round(g.standard_normal((3, vocab))) / 64
    if kind == "outliers in the tail":   # (of the first bins, and of none at all)
        l[0, -1:], l[1, -2:], l[2, -1:] = 0.5, -30.0, -np.inf
    logits = torch.from_numpy(l.astype(np.float32)).to(TYPES[dtype]).to(DEV)
    for s in (dict(), dict(top_p=0.5), dict(top_p=0.95, temperature=0.7), dict(min_p=0.99), dict(top_k=vocab // 2), dict(top_k=vocab // 3, top_p=0.9), dict(temperature=3.0)):
        for u in (0.123, 0.456, 0.789):
            _check(B, logits, uniform=u, **s)
            _check(B, logits, uniform=u, with_workspace=False, **s)
