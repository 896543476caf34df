"""Attention over a paged cache whose sequences are longer than the page table or the stated bound: positions go by the true length, the keys beyond
are unseen."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as O

from .test_gpu_paged_attention import B, DEV, TYPES, _case, _np, _run  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


def _want(c, limit, scale, causal, window):
    """The oracle over a table that names no page from key `limit` on; pages that both sides of the limit share are given twice, key by key."""
    ps, pages = c["kc"].shape[1], c["kc"].shape[0]
    # one key to a page, so that the limit may lie anywhere
    kc, vc = (np.nan_to_num(_np(c[n])).reshape(pages * ps, 1, *c[n].shape[2:]) for n in ("kc", "vc"))
    longest = int(c["kv"].max())
    table = np.full((len(c["kv"]), longest), -1, dtype=np.int64)
    for b, kv in enumerate(c["kv"]):
        j = np.arange(min(int(kv), limit))
        table[b, :len(j)] = c["table"][b][j // ps].astype(np.int64) * ps + j % ps
    return O.attention(_np(c["q"]), kc, vc, table, c["starts"], c["kv"], scale, causal, window)


def _check(B, c, limit, causal, window, workspace):
    got, s = _run(B, c, causal, window, workspace)
    want, mag, spread, keys = _want(c, limit, s["scale"], causal, window)
    _, u, tiny = TYPES[c["dtype"]]
    tol = O.attention_tolerance(want, mag, spread, keys, np.nanmax(np.abs(_np(c["vc"]))), c["dim"], u, tiny)
    got = _np(got)
    assert (np.abs(got - want) <= tol).all(), float(np.nanmax(np.abs(got - want) / tol))
    assert (got[keys == 0] == 0).all()


MASKS = [(True, 0), (True, 4), (True, 50), (False, 0), (False, 9)]


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("causal,window", MASKS)
@pytest.mark.parametrize("lens", [[(1, 80)], [(4, 80), (2, 20)], [(60, 80), (3, 200)], [(3, 900)], [(60, 900)]])
@pytest.mark.parametrize("limit", [1, 64, 71])
def test_bound_below_the_lengths(B, lens, causal, window, workspace, limit):
    c = _case("f16", lens, 4, 2, 64, 16)
    c["max_kv"] = limit
    _check(B, c, limit, causal, window, workspace)


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("causal,window", MASKS)
@pytest.mark.parametrize("lens,pages", [([(20, 80)], 4), ([(1, 80)], 4), ([(3, 1500), (2, 30)], 50), ([(90, 1500), (7, 30)], 50)])
def test_table_too_short_for_the_lengths(B, lens, pages, causal, window, workspace):
    c = _case("bf16", lens, 4, 2, 128, 16)
    c["table"] = np.ascontiguousarray(c["table"][:, :pages])
    _check(B, c, pages * 16, causal, window, workspace)
