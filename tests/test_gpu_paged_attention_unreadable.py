"""Attention over a paged cache where tokens lose keys to page numbers outside of the cache: such keys count as unseen, and a token that has no
other gets zeros."""
import numpy as np
import pytest
import torch

from .test_gpu_paged_attention import B, _both, _case, _run, _verify  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("dtype,ps,dim", [("f16", 16, 64), ("bf16", 10, 128)])
@pytest.mark.parametrize("new,kv", [(1, 100), (40, 100), (1, 3000), (40, 3000), (300, 310)])
@pytest.mark.parametrize("page", [-1, 1 << 30])
def test_every_page_outside(B, workspace, dtype, ps, dim, new, kv, page):
    c = _case(dtype, [(new, kv)], 4, 2, dim, ps)
    c["table"][:] = page
    got, _ = _run(B, c, workspace=workspace)
    assert (got == 0).all()


@pytest.mark.parametrize("causal,window", [(True, 5), (True, 40), (True, 0), (False, 3)])
@pytest.mark.parametrize("new,kv", [(4, 90), (70, 90), (4, 2000), (300, 2000)])
def test_some_rows_lose_all_their_keys(B, causal, window, new, kv):
    """Runs of pages outside, also the first and the last ones: rows with other keys beside rows with none."""
    c = _case("f16", [(new, kv), (2, 33)], 4, 2, 64, 16)
    for first in range(0, c["table"].shape[1], 3):
        c["table"][0, first:first + 2] = -1
    c["table"][0, -1], c["table"][0, (kv - 1) // 16] = 10 ** 6, -7
    _both(B, c, causal, window)


def test_the_two_of_a_workgroups_pieces(B):
    """Sequences in one line of units, of which some cannot be read at all."""
    c = _case("bf16", [(1, 500 + 90 * i) for i in range(20)], 4, 2, 64, 16)
    c["table"][3:12:2] = 1 << 20
    _both(B, c)
    got, _ = _run(B, c)
    assert (got[3:12:2] == 0).all() and (got[2:12:2] != 0).any(dim=-1).all()
