"""Dense with 4-bit weights with one scale to a unit: groups as long as the row or longer, rows that end anywhere in a chunk."""
import pytest

from .test_gpu_dense_w4 import B, _case  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("k,group", [(8, 32), (40, 64), (200, 224), (200, 4096), (1000, 1024), (1000, 1 << 30), (2184, 2208)])
@pytest.mark.parametrize("m", [1, 3, 9, 40, 200])
def test_one_scale_to_a_unit(B, dtype, m, k, group):
    _case(B, dtype, m, 75, k, group, zeros=m != 3)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1020, 2050, 2184), (2100, 2500, 296)])
def test_one_scale_to_a_unit_in_tiles(B, dtype, m, n, k):
    _case(B, dtype, m, n, k, k + 32 - k % 32, zeros=True)
