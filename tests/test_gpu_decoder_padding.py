"""Rows of padding in a step: a function of their input, whatever memory the layer's buffers were given."""
import pytest
import torch

from .test_gpu_decoder import D, DEV, DIM, HKV, _stack  # noqa: F401  (D is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_padding_rows_do_not_depend_on_old_memory(D, dtype, monkeypatch):
    tt = torch.float16 if dtype == "f16" else torch.bfloat16
    x = torch.randn((6, 192), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(tt)
    real, out = torch.empty, []
    for value in (float("nan"), 3.0):
        monkeypatch.setattr(torch, "empty", lambda *a, **k: (lambda t: t.fill_(value) if t.is_floating_point() else t)(real(*a, **k)))
        layers, _, _ = _stack(D, dtype, layers=1)
        monkeypatch.setattr(torch, "empty", real)
        cache = D.PagedCache(1, 8, 16, HKV, DIM, tt)
        step = D.Step(cache, 1, 6, 4, 64)
        step.extend([cache.open()], [4])          # (two rows of padding)
        out.append(layers[0](x, 0, step).clone())
    assert torch.isfinite(out[0].float()).all() and torch.equal(out[0], out[1])
