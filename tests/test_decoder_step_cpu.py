"""What a step tells the kernels before it has been given tokens."""
from paper_1904_08368_amd.decoder import PagedCache, Step


def test_a_step_without_tokens_stores_nothing():
    cache = PagedCache(1, 4, 4, kv_heads=1, head_dim=8, device="cpu")
    step = Step(cache, batch=2, tokens=5, max_q_len=3, max_kv_len=9)
    assert step.slots.tolist() == [-1] * 5 and step.page_table.tolist() == [[-1] * 3] * 2
    assert step.q_starts.tolist() == [0, 0, 0] and step.kv_lens.tolist() == [0, 0]
