"""Dense with 4-bit weights in tiles of 128 x 128 whose reduction two halves of a workgroup share: reductions of even and odd numbers of chunks that end anywhere in
one, every group size, the tail."""
import pytest

from .test_gpu_dense_w4 import B, _case  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("k,group,zeros", [(128 * 16, 128, True), (128 * 17, 32, True), (128 * 17 + 8, 64, False), (128 * 16 + 72, 96, True), (128 * 15 + 120, 256, True),
                                           (128 * 20 + 56, 128, False)])
def test_reductions_in_two_parts(B, dtype, k, group, zeros):
    _case(B, dtype, 1020, 2050, k, group, zeros)


@pytest.mark.parametrize("n,ypad", [(2048, 0), (2049, 3), (2052, 4)])
def test_tail_in_two_parts(B, n, ypad):
    for dtype in ("f16", "bf16"):
        _case(B, dtype, 1000, n, 128 * 16, 128, zeros=True, bias=True, residual=True, relu=True, xpad=8, ypad=ypad, mean=2.0)
