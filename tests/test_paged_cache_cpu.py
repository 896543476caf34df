"""Room in the cache: what would leave a sequence with other pages than its tokens need is refused, and nothing changes."""
import pytest

from paper_1904_08368_amd.decoder import PagedCache


@pytest.mark.parametrize("seqs,new", [([0, 0], [1, 1]), ([0], [1, 2]), ([0, 1], [1]), ([0], [-2]), ([0, 1], [2, -1])])
def test_what_extend_refuses(seqs, new):
    cache = PagedCache(1, 6, 4, kv_heads=1, head_dim=8, device="cpu")
    ids = [cache.open(), cache.open()]
    cache.extend(ids, [3, 4])
    with pytest.raises(ValueError):
        cache.extend([ids[s] for s in seqs], new)
    assert cache.length == {ids[0]: 3, ids[1]: 4} and [len(cache.pages[s]) for s in ids] == [1, 1] and len(cache.free) == 4


def test_a_sequence_that_is_not_open_changes_nothing():
    cache = PagedCache(1, 6, 4, kv_heads=1, head_dim=8, device="cpu")
    a = cache.open()
    with pytest.raises(KeyError):
        cache.extend([a, a + 1], [5, 5])
    assert cache.length == {a: 0} and not cache.pages[a] and len(cache.free) == 6
