"""Windows far longer than any sequence mask nothing, also for a sequence with more new tokens than keys."""
import pytest
import torch

from .test_gpu_paged_attention import B, _both, _case, _run  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 9, 2 ** 30])
@pytest.mark.parametrize("lens", [[(20, 12)], [(3, 2), (1, 1), (2, 300)], [(300, 5), (200, 190)], [(9, 1), (1, 2000)]])
@pytest.mark.parametrize("causal", [True, False])
def test_windows_that_mask_nothing(B, lens, causal, window):
    c = _case("f16", lens, 4, 2, 64, 16)
    _both(B, c, causal, window)
    for workspace in (True, False):
        got, none = (_run(B, c, causal, w, workspace)[0] for w in (window, 0))
        assert torch.equal(got, none)
