"""How attention over a paged cache is cut for the chip, as far as the workspace that it asks for tells: no GPU."""
import ctypes as C

import pytest

from paper_1904_08368_amd import binding as B


def _bytes(max_q_len, max_kv_len, window, batch=1, causal=1):
    d = B.PagedAttentionDesc(B.RELAY_F16, batch, batch * max_q_len, 8, 2, 64, 5000, 16, 5000, max_q_len, max_kv_len, causal, window, 0.125, 512, 512, 2048, 128, 64)
    return B.relay_paged_attention_workspace_bytes(d)


@pytest.mark.parametrize("max_q_len", [1, 3, 40, 700])
@pytest.mark.parametrize("max_kv_len,batch", [(300, 1), (3000, 2), (70000, 1), (5000, 9)])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 40, 2 ** 30, 80000])
def test_a_window_longer_than_the_keys_changes_nothing(max_q_len, max_kv_len, batch, window):
    """Keys are shared out as without a window.  (A sum of window and tokens past 2^31 once counted as no keys at all: one workgroup to a sequence.)"""
    want = _bytes(max_q_len, max_kv_len, 0, batch)
    assert _bytes(max_q_len, max_kv_len, window, batch) == want
    assert want > 0 or max_kv_len == 300 or max_q_len == 700
