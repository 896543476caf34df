"""Dense with 4-bit weights: tensors that do not go with the packed weights are refused before any call of the library."""
import pytest
import torch

from paper_1904_08368_amd import binding as B
from paper_1904_08368_amd.decoder import Dense4, quantize4


@pytest.fixture
def layer(monkeypatch):
    """A layer of 40 units by 64 in groups of 32; packing and products are counted, not run."""
    calls = []
    monkeypatch.setattr(B, "_stream", lambda: None)
    real = B.lib()

    class Lib:
        def __getattr__(self, name):
            return (lambda *a: calls.append(name) or 0) if name in ("relay_prepack_qdense_w4", "relay_qdense_w4") else getattr(real, name)
    monkeypatch.setattr(B, "lib", lambda: Lib())
    codes, scales, zeros = quantize4(torch.randn(40, 64, dtype=torch.float16), 32)
    return Dense4(codes, scales, zeros, 32, 64, bias=torch.zeros(40)), calls


def _t(*shape, dtype=torch.float16):
    return torch.zeros(shape, dtype=dtype)


def test_a_layer_takes_what_it_was_made_for(layer):
    dense, calls = layer
    dense(_t(3, 64), _t(3, 40), _t(3, 40))
    assert calls == ["relay_prepack_qdense_w4", "relay_qdense_w4"]


@pytest.mark.parametrize("x,y", [(_t(3, 72), _t(3, 40)), (_t(3, 56), _t(3, 40)), (_t(3, 64), _t(3, 48)), (_t(3, 64), _t(3, 32)),
                                 (_t(3, 64, dtype=torch.bfloat16), _t(3, 40, dtype=torch.bfloat16)), (_t(3, 64), _t(2, 40)),
                                 (_t(3, 64), _t(3, 40, dtype=torch.bfloat16))])
def test_a_layer_refuses_other_widths_and_types(layer, x, y):
    dense, calls = layer
    with pytest.raises((ValueError, B.RelayError)):
        dense(x, y)
    assert calls == ["relay_prepack_qdense_w4"]


@pytest.mark.parametrize("residual", [_t(3, 40, dtype=torch.bfloat16), _t(3, 40, dtype=torch.float32), _t(3, 48)])
def test_a_layer_refuses_other_residuals(layer, residual):
    with pytest.raises(B.RelayError):
        layer[0](_t(3, 64), _t(3, 40), residual)


@pytest.mark.parametrize("bias", [_t(40), _t(39, dtype=torch.float32), _t(80, dtype=torch.float32)[::2]])
def test_other_biases_are_refused(layer, bias):
    with pytest.raises(B.RelayError):
        B.qdense_w4_desc(_t(3, 64), _t(3, 40), 32, None, bias)


def test_packing_refuses_other_operands(layer):
    d = B.qdense_w4_desc(_t(0, 64), _t(0, 40), 32, _t(1))
    good = [_t(40, 32, dtype=torch.uint8), _t(40, 2), _t(40, 2, dtype=torch.uint8)]
    packed = _t(d.packed_bytes, dtype=torch.uint8)
    B.relay_prepack_qdense_w4(d, *good, packed)
    for i, bad in [(0, _t(40, 64, dtype=torch.uint8)), (0, _t(39, 32, dtype=torch.uint8)), (0, _t(40, 32)), (0, _t(40, 64, dtype=torch.uint8)[:, ::2]),
                   (1, _t(40, 1)), (1, _t(40, 2, dtype=torch.bfloat16)), (1, _t(2, 40).t()), (2, _t(40, 2)), (2, _t(40, 3, dtype=torch.uint8))]:
        with pytest.raises(B.RelayError):
            B.relay_prepack_qdense_w4(d, *[bad if j == i else t for j, t in enumerate(good)], packed)


def test_packed_weights_of_another_layer_are_refused(layer):
    dense, calls = layer
    for x, y in ((_t(3, 256), _t(3, 40)), (_t(3, 64), _t(3, 64))):
        with pytest.raises(B.RelayError):
            B.relay_qdense_w4(B.qdense_w4_desc(x, y, 32, dense.zeros), x, dense.packed, None, None, y)
    assert "relay_qdense_w4" not in calls
