"""Rotation, store and attention: tensors of types that do not go together, and index tensors that the kernels would misread, are refused before any call of
the library."""
import pytest
import torch

from paper_1904_08368_amd import binding as B


@pytest.fixture(autouse=True)
def calls(monkeypatch):
    """The three entry points are counted, not run."""
    seen, real = [], B.lib()

    class Lib:
        def __getattr__(self, name):
            return (lambda *a: seen.append(name) or 0) if name in ("relay_rope", "relay_rope_append", "relay_paged_attention") else getattr(real, name)
    monkeypatch.setattr(B, "lib", lambda: Lib())
    monkeypatch.setattr(B, "_stream", lambda: None)
    return seen


def _t(*shape, dtype=torch.float16):
    return torch.zeros(shape, dtype=dtype)


def _i(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype)


Q, K, CACHE, TABLE, PAGES = _t(4, 8, 64), _t(4, 2, 64), _t(3, 16, 2, 64), torch.zeros(10, 32, 2), _i(2, 5)
BF = torch.bfloat16
BAD_INDEX = [lambda n: _i(n, dtype=torch.int64), lambda n: _i(n - 1), lambda n: _i(2 * n)[::2], lambda n: torch.zeros(n), lambda n: None]


def test_what_goes_together_is_taken(calls):
    B.relay_rope(B.rope_desc(Q, TABLE, Q), Q, TABLE, _i(4), Q)
    B.relay_rope_append(B.rope_append_desc(Q, K, K, TABLE, Q, CACHE), Q, K, K, TABLE, _i(4), _i(9), Q, CACHE, CACHE.clone())
    B.relay_paged_attention(B.paged_attention_desc(Q, CACHE, PAGES, Q, 1, 5, 0.1), Q, CACHE, CACHE, PAGES, _i(3), _i(2), Q, _i(64))
    B.relay_paged_attention(B.paged_attention_desc(Q, CACHE, PAGES, Q, 1, 5, 0.1), Q, CACHE, CACHE, PAGES, _i(3), _i(2), Q)
    assert calls == ["relay_rope", "relay_rope_append", "relay_paged_attention", "relay_paged_attention"]


@pytest.mark.parametrize("table", [TABLE.double(), TABLE.half(), TABLE[:, ::2], TABLE[..., 0], torch.zeros(10, 32, 3)])
def test_other_tables_are_refused(table):
    with pytest.raises(B.RelayError):
        B.rope_desc(Q, table, Q)
    with pytest.raises(B.RelayError):
        B.rope_append_desc(Q, K, K, table, Q, CACHE)


@pytest.mark.parametrize("bad", range(5))
def test_descriptors_refuse_mixed_types(bad):
    q, k, v, out, cache = (t.to(BF) if i == bad else t for i, t in enumerate((Q, K, K, Q, CACHE)))
    with pytest.raises(B.RelayError):
        B.rope_append_desc(q, k, v, TABLE, out, cache)
    if bad in (0, 3, 4):
        with pytest.raises(B.RelayError):
            B.paged_attention_desc(q, cache, PAGES, out, 1, 5, 0.1)


def test_descriptors_refuse_other_extents_and_page_numbers():
    with pytest.raises(B.RelayError):
        B.rope_append_desc(Q, _t(3, 2, 64), _t(3, 2, 64), TABLE, Q, CACHE)
    with pytest.raises(B.RelayError):
        B.rope_append_desc(Q, _t(4, 2, 32), _t(4, 2, 32), TABLE, Q, _t(3, 16, 2, 32))
    with pytest.raises(B.RelayError):
        B.paged_attention_desc(Q, CACHE, PAGES.long(), Q, 1, 5, 0.1)


@pytest.mark.parametrize("bad", range(len(BAD_INDEX)))
def test_calls_refuse_other_index_tensors(calls, bad):
    make = BAD_INDEX[bad]
    rope, append = B.rope_desc(Q, TABLE, Q), B.rope_append_desc(Q, K, K, TABLE, Q, CACHE)
    attention = B.paged_attention_desc(Q, CACHE, PAGES, Q, 1, 5, 0.1)
    for call in (lambda: B.relay_rope(rope, Q, TABLE, make(4), Q),
                 lambda: B.relay_rope_append(append, Q, K, K, TABLE, make(4), _i(4), Q, CACHE, CACHE),
                 lambda: B.relay_rope_append(append, Q, K, K, TABLE, _i(4), make(4), Q, CACHE, CACHE),
                 lambda: B.relay_paged_attention(attention, Q, CACHE, CACHE, PAGES, make(3), _i(2), Q),
                 lambda: B.relay_paged_attention(attention, Q, CACHE, CACHE, PAGES, _i(3), make(2), Q)):
        with pytest.raises(B.RelayError):
            call()
    assert not calls


def test_calls_refuse_what_is_missing(calls):
    append, attention = B.rope_append_desc(Q, K, K, TABLE, Q, CACHE), B.paged_attention_desc(Q, CACHE, PAGES, Q, 1, 5, 0.1)
    for i in range(7):
        args = [Q, K, K, TABLE, Q, CACHE, CACHE]
        args[i] = None
        with pytest.raises(B.RelayError):
            B.relay_rope_append(append, *args[:4], _i(4), _i(4), *args[4:])
    for i in range(5):
        args = [Q, CACHE, CACHE, PAGES, Q]
        args[i] = None
        with pytest.raises(B.RelayError):
            B.relay_paged_attention(attention, *args[:4], _i(3), _i(2), args[4])
    assert not calls
