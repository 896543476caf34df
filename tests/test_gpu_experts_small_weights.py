"""The experts' results where a router leaves small weights, as scores that are not normalised do: each part of y keeps its bits, however little it counts."""
import numpy as np
import pytest
import torch

from oracle import decoder as O

from .test_gpu_experts import B, DEV, TYPES, Layer, _np, _run, scratch  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


class Steep(Layer):
    """The second product's scales 2^11 times as large, so that parts with small weights are a result of ordinary size."""

    def __init__(self, B, dtype, channels, inter, experts, group, zeros=False):
        super().__init__(B, dtype, channels, inter, experts, group, zeros)
        codes, scales, zp = self.host[1]
        scales = torch.from_numpy(scales * 2048.0).to(TYPES[dtype][0])
        x, y = (torch.empty((0, e), dtype=TYPES[dtype][0], device=DEV) for e in (inter, experts * channels))
        zd = None if zp is None else torch.from_numpy(zp).to(DEV)
        B.relay_prepack_qdense_w4(B.qdense_w4_desc(x, y, group, zd), torch.from_numpy(codes).to(DEV), scales.to(DEV), zd, self.packed[1])
        self.host[1] = (codes, _np(scales), zp)


# Few pairs (their sums within the second launch), more by rows, many by tiles; one expert and several.
@pytest.mark.parametrize("experts,top_k,tokens", [(16, 4, 1), (1, 1, 1), (16, 4, 7), (2, 2, 5), (2, 1, 90), (64, 8, 60)])
@pytest.mark.parametrize("dtype,channels,inter,group", [("f16", 256, 128, 128), ("f16", 272, 176, 64), ("bf16", 256, 128, 32)])
def test_small_weights(B, scratch, dtype, channels, inter, group, experts, top_k, tokens):
    layer = Steep(B, dtype, channels, inter, experts, group, zeros=group == 64)
    s = layer.inputs(tokens, top_k, residual=False)
    s["x"] = (s["x"].float() * 0.05).to(s["x"].dtype)              # act and what stands beside it: some 0.03 each
    g = np.random.default_rng(tokens)
    for size in (2e-4, 1e-6, 300.0):
        s["weights"].copy_(torch.from_numpy((size * g.uniform(0.5, 2.0, (tokens, top_k))).astype(np.float32)))
        _, y = _run(B, scratch, layer, s)
        _, u, tiny = TYPES[dtype]
        want, err = O.experts(_np(s["x"]), s["chosen"].cpu().numpy(), _np(s["weights"]), *layer.host, inter, group, "silu", None, u, tiny)
        got, tol = _np(y), err + u * (np.abs(want) + err) + tiny
        # fp16 ends at 65504 = 2^16 - 2^5, half a step behind which, from 65520 on, the rounding gives an infinity: that is right where y may lie there
        # (the largest of the large weights' sums do).
        over = (np.abs(want) + err >= 65520) & (got == np.copysign(np.inf, want)) if dtype == "f16" else np.zeros(got.shape, bool)
        off = np.where(over, 0.0, np.abs(np.where(over, 0.0, got) - np.where(over, 0.0, want)))
        assert (off <= tol).all(), (size, float((off / tol).max()))


def test_weights_of_zero_and_below(B, scratch):
    """A weight of zero leaves the residual as it is; one below zero subtracts."""
    layer = Layer(B, "f16", 256, 128, 4, 128)
    for tokens in (1, 6, 80):
        s = layer.inputs(tokens, 2)
        s["weights"].zero_()
        _, y = _run(B, scratch, layer, s)
        assert torch.equal(y, s["residual"])
        s["weights"].fill_(1.0)
        zero = torch.zeros_like(s["residual"])
        _, plus = _run(B, scratch, layer, {**s, "residual": zero})
        s["weights"].fill_(-1.0)
        _, minus = _run(B, scratch, layer, {**s, "residual": zero})
        assert torch.equal(plus, -minus) and plus.any()
