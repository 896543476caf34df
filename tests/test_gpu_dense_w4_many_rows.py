"""Dense with 4-bit weights where it is a matrix product: 128 x 128 tiles whose reduction one or two parts of a workgroup walk, reductions that end anywhere in a
chunk, outputs stored four at a time and one at a time."""
import pytest
import torch

from .test_gpu_dense_w4 import B, _case  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128, 96, 256])
@pytest.mark.parametrize("m,n,k", [(1100, 1500, 128 * 16),        # few tiles, an even number of chunks
                                   (1100, 1501, 128 * 17),        # ... an odd one; odd units
                                   (1030, 1300, 128 * 17 + 8),    # ... a last chunk of one piece
                                   (1030, 1300, 128 * 16 + 72),   # ... of a half and a piece
                                   (1030, 1300, 128 * 15 + 120),
                                   (2100, 2500, 128 * 2 + 40)])   # more tiles than CUs
def test_reductions_of_tiles(B, dtype, group, m, n, k):
    _case(B, dtype, m, n, k, group, zeros=group != 64)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("ypad", [0, 2, 4])
@pytest.mark.parametrize("n", [1500, 1502, 1503])
def test_tail_of_tiles(B, dtype, ypad, n):
    _case(B, dtype, 1100, n, 2048, 128, zeros=True, bias=True, residual=True, relu=True, xpad=8, ypad=ypad)
    _case(B, dtype, 33, n, 512, 128, bias=True, residual=True, ypad=ypad)


@pytest.mark.parametrize("offset", [1, 2, 3, 4])
def test_outputs_and_bias_of_any_alignment(B, offset):
    """y, the residual and the bias start anywhere their type allows; the results are those of aligned ones."""
    s = _case(B, "f16", 40, 512, 256, 64, zeros=True, bias=True, residual=True)
    flat = torch.full((40 * 512 + 16,), 7.0, dtype=torch.float16, device="cuda")
    res = torch.empty_like(flat)
    y, r = flat[offset:offset + 40 * 512].view(40, 512), res[offset:offset + 40 * 512].view(40, 512)
    r.copy_(s["res"])
    bias = torch.empty(512 + 4, device="cuda")[offset - 1:offset - 1 + 512]
    bias.copy_(s["bias"])
    B.relay_qdense_w4(s["d"], s["x"], s["packed"], bias, r, y)
    torch.cuda.synchronize()
    assert torch.equal(y, s["y"]) and (flat[:offset] == 7).all() and (flat[offset + 40 * 512:] == 7).all()


def test_weights_with_a_large_mean_of_x(B):
    """Rows of x far from zero: the zero points' share of the sums is large against the result."""
    for dtype in ("f16", "bf16"):
        _case(B, dtype, 1100, 1500, 2048, 128, zeros=True, mean=8.0)
