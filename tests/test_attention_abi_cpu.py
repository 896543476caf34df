"""The entry points of the attention layer's operators without a GPU: what they refuse, with which status, before any HIP call; sizes of
packed weights; calls that launch nothing."""
import ctypes as C

import pytest

from paper_1904_08368_amd import binding as B

FAKE = 0x7F0000001000            # a non-NULL, 4096-byte aligned address that is never dereferenced
at = lambda i: FAKE + (i << 24)


def _status(fn, *args):
    return getattr(B.lib(), fn)(*args)


def _with(d, **kw):
    for k, v in kw.items():
        setattr(d, k, v)
    return C.byref(d)


def _rope(**kw):
    return _with(B.RopeDesc(B.RELAY_F16, 4, 2, 64, 32, B.ROPE_HALF, 0, 100, 128, 64, 128, 64), **kw)


def _call_rope(d, x=at(0), table=at(1), pos=at(2), y=at(3)):
    return _status("relay_rope", d, x, table, pos, y, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=B.RELAY_I8), 3), (dict(dtype=9), 3), (dict(tokens=-1), 2), (dict(heads=0), 2), (dict(head_dim=0), 2), (dict(rotary_dim=0), 2),
    (dict(rotary_dim=31), 2), (dict(rotary_dim=66), 2), (dict(style=2), 4), (dict(inverse=2), 4), (dict(table_rows=0), 2),
    (dict(x_token_stride=-1), 2), (dict(y_token_stride=63), 2), (dict(y_head_stride=0), 2), (dict(tokens=1 << 30, heads=1 << 20), 2)])
def test_rope_refuses(kw, status):
    assert _call_rope(_rope(**kw)) == status and B.lib().relay_last_error()


def test_rope_pointers():
    assert _call_rope(None) == 1
    for i in range(4):
        args = [at(j) for j in range(4)]
        args[i] = None
        assert _call_rope(_rope(), *args) == 1
    assert _call_rope(_rope(), x=at(0) + 1) == 5 and _call_rope(_rope(), y=at(3) + 1) == 5
    assert _call_rope(_rope(), table=at(1) + 4) == 5 and _call_rope(_rope(), pos=at(2) + 2) == 5
    assert _call_rope(_rope(y_token_stride=256), y=at(0)) == 4          # in place with other strides
    assert _call_rope(_rope(tokens=0), None, None, None, None) == 0     # nothing to do: nothing is needed


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), 2), (dict(first=-1), 2), (dict(rotary_dim=3), 2), (dict(rotary_dim=0), 2), (dict(scaling=4), 4), (dict(base=0.0), 2),
    (dict(base=float("nan")), 2), (dict(magnitude=float("inf")), 2), (dict(scaling=1, factor=0.5), 2), (dict(scaling=1, factor=float("nan")), 2),
    (dict(scaling=2, rotary_dim=2, factor=2.0), 2), (dict(scaling=3, factor=2.0, slow=4.0, fast=4.0), 2),
    (dict(scaling=3, factor=2.0, original_len=0.0), 2), (dict(scaling=3, factor=2.0, slow=float("nan")), 2)])
def test_rope_table_refuses(kw, status):
    assert _status("relay_rope_table", _with(B.rope_table_desc(10, 8), **kw), at(0), None) == status


def test_rope_table_pointers():
    assert _status("relay_rope_table", None, at(0), None) == 1
    assert _status("relay_rope_table", C.byref(B.rope_table_desc(10, 8)), None, None) == 1
    assert _status("relay_rope_table", C.byref(B.rope_table_desc(10, 8)), at(0) + 4, None) == 5
    assert _status("relay_rope_table", C.byref(B.rope_table_desc(0, 8)), None, None) == 0


def _append(**kw):
    return _with(B.RopeAppendDesc(B.RELAY_BF16, 4, 8, 2, 64, 64, B.ROPE_HALF, 100, 10, 16, 768, 768, 768, 512, 2048, 128, 64), **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=B.RELAY_I16), 3), (dict(tokens=-2), 2), (dict(q_heads=0), 2), (dict(kv_heads=0), 2), (dict(num_pages=0), 2), (dict(page_size=0), 2),
    (dict(num_pages=1 << 20, page_size=1 << 12), 2), (dict(rotary_dim=128), 2), (dict(style=-1), 4), (dict(k_token_stride=-1), 2),
    (dict(q_out_token_stride=511), 2), (dict(page_stride=63), 2), (dict(slot_stride=0), 2), (dict(head_stride=8), 2)])
def test_append_refuses(kw, status):
    assert _status("relay_rope_append", _append(**kw), *[at(i) for i in range(9)], None) == status


def test_append_pointers():
    for i in range(9):
        args = [at(j) for j in range(9)]
        args[i] = None
        assert _status("relay_rope_append", _append(), *args, None) == 1
        args[i] = at(i) + 1
        assert _status("relay_rope_append", _append(), *args, None) == 5
    same = [at(j) for j in range(9)]
    same[8] = same[7]                                                  # one cache for keys and values
    assert _status("relay_rope_append", _append(), *same, None) == 4
    inplace = [at(j) for j in range(9)]
    inplace[6] = inplace[0]
    assert _status("relay_rope_append", _append(), *inplace, None) == 4  # q and q_out of different strides
    assert _status("relay_rope_append", _append(tokens=0), *[None] * 9, None) == 0


def _attn(**kw):
    return _with(B.PagedAttentionDesc(B.RELAY_F16, 2, 5, 8, 2, 64, 10, 16, 4, 4, 60, 1, 0, 0.125, 512, 512, 2048, 128, 64), **kw)


def _call_attn(d, args=None, ws=None, ws_bytes=0):
    return _status("relay_paged_attention", d, *(args or [at(i) for i in range(7)]), ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=B.RELAY_F32), 3), (dict(batch=-1), 2), (dict(tokens=-1), 2), (dict(q_heads=0), 2), (dict(kv_heads=0), 2), (dict(q_heads=7), 2),
    (dict(head_dim=0), 4), (dict(head_dim=60), 4), (dict(head_dim=264), 4), (dict(num_pages=0), 2), (dict(page_size=0), 2), (dict(pages_per_seq=0), 2),
    (dict(max_q_len=-1), 2), (dict(max_kv_len=-1), 2), (dict(causal=2), 4), (dict(window=-1), 2), (dict(scale=float("nan")), 2),
    (dict(scale=float("inf")), 2), (dict(q_token_stride=-8), 2), (dict(out_token_stride=504), 2), (dict(q_token_stride=516), 5), (dict(page_stride=-8), 2),
    (dict(slot_stride=4), 5), (dict(head_stride=65), 5), (dict(out_token_stride=513), 5)])
def test_attention_refuses(kw, status):
    b = C.c_size_t()
    assert _call_attn(_attn(**kw)) == status
    assert _status("relay_paged_attention_workspace_bytes", _attn(**kw), C.byref(b)) == status


def test_attention_pointers_and_workspace():
    assert _call_attn(None) == 1
    b = C.c_size_t()
    assert _status("relay_paged_attention_workspace_bytes", _attn(), None) == 1
    for i in range(7):
        args = [at(j) for j in range(7)]
        args[i] = None
        assert _call_attn(_attn(), args) == 1
        args[i] = at(i) + 2
        assert _call_attn(_attn(), args) == 5
    alias = [at(j) for j in range(7)]
    alias[6] = alias[0]
    assert _call_attn(_attn(), alias) == 4
    assert _call_attn(_attn(), ws=at(9) + 128, ws_bytes=1 << 30) == 5
    long = dict(batch=1, tokens=1, max_q_len=1, num_pages=10000, pages_per_seq=5000, max_kv_len=80000)
    assert _status("relay_paged_attention_workspace_bytes", _attn(**long), C.byref(b)) == 0
    if b.value:
        assert _call_attn(_attn(**long), ws=at(9), ws_bytes=b.value - 1) == 6
    for kw in (dict(tokens=0), dict(batch=0), dict(max_q_len=0)):
        assert _call_attn(_attn(**kw), [None] * 7) == 0


def _w4(**kw):
    return _with(B.QDenseW4Desc(B.RELAY_F16, 3, 40, 128, 64, 0, 0, 128, 40), **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=B.RELAY_F32), 3), (dict(m=-1), 2), (dict(n=0), 2), (dict(k=0), 2), (dict(k=100), 5), (dict(group=0), 2), (dict(group=48), 2),
    (dict(has_zeros=2), 4), (dict(flags=B.HAS_BN), 4), (dict(flags=64), 4), (dict(x_stride=-8), 2), (dict(x_stride=132), 5), (dict(y_stride=39), 2)])
def test_w4_refuses(kw, status):
    b = C.c_size_t()
    assert _status("relay_qdense_w4_packed_bytes", _w4(**kw), C.byref(b)) == status
    assert _status("relay_qdense_w4", _w4(**kw), at(0), at(1), None, None, at(2), None) == status
    assert _status("relay_prepack_qdense_w4", _w4(**kw), at(0), at(1), None, at(2), 1 << 30, None) == status


def test_w4_pointers():
    f = "relay_qdense_w4"
    assert _status(f, None, at(0), at(1), None, None, at(2), None) == 1
    assert _status(f, _w4(), None, at(1), None, None, at(2), None) == 1
    assert _status(f, _w4(), at(0), None, None, None, at(2), None) == 1
    assert _status(f, _w4(), at(0), at(1), None, None, None, None) == 1
    assert _status(f, _w4(), at(0), at(1), at(3), None, at(2), None) == 1                      # bias without its flag
    assert _status(f, _w4(flags=B.HAS_BIAS), at(0), at(1), None, None, at(2), None) == 1
    assert _status(f, _w4(flags=B.HAS_RESIDUAL), at(0), at(1), None, None, at(2), None) == 1
    assert _status(f, _w4(), at(0) + 2, at(1), None, None, at(2), None) == 5
    assert _status(f, _w4(), at(0), at(1) + 8, None, None, at(2), None) == 5
    assert _status(f, _w4(), at(0), at(1), None, None, at(2) + 1, None) == 5
    assert _status(f, _w4(), at(0), at(1), None, None, at(0), None) == 4
    assert _status(f, _w4(m=0), None, None, None, None, None, None) == 0
    p = "relay_prepack_qdense_w4"
    assert _status(p, _w4(), None, at(1), None, at(2), 1 << 30, None) == 1
    assert _status(p, _w4(), at(0), at(1), at(3), at(2), 1 << 30, None) == 1                   # zeros without has_zeros
    assert _status(p, _w4(has_zeros=1), at(0), at(1), None, at(2), 1 << 30, None) == 1
    assert _status(p, _w4(), at(0), at(1), None, at(2) + 8, 1 << 30, None) == 5
    assert _status(p, _w4(), at(0), at(1), None, at(0), 1 << 30, None) == 4
    assert _status(p, _w4(), at(0), at(1), None, at(2), 10, None) == 6


def test_w4_packed_bytes():
    """Tiles of 16 units, chunks of 128 of the reduction, 4 bits each; 2 bytes a scale, 1 a zero point."""
    size = lambda **kw: (lambda b: (_status("relay_qdense_w4_packed_bytes", _w4(**kw), C.byref(b)), b.value))(C.c_size_t())
    assert size() == (0, 3 * 1024 + 3 * 2 * 32)
    assert size(has_zeros=1) == (0, 3 * 1024 + 3 * 2 * 48)
    assert size(n=4096, k=4096, group=128, y_stride=4096) == (0, 256 * 32 * 1024 + 256 * 32 * 32)
    assert size(k=8, group=32) == size(k=8, group=4096) == (0, 3 * 1024 + 3 * 32)


def test_binding_refuses_tensors_it_cannot_describe():
    import torch
    q, k = torch.zeros(4, 8, 64, dtype=torch.float16), torch.zeros(4, 2, 64, dtype=torch.float16)
    cache = torch.zeros(3, 16, 2, 64, dtype=torch.float16)
    table = torch.zeros(10, 32, 2)
    B.rope_append_desc(q, k, k, table, q, cache)
    pages = torch.zeros(2, 5, dtype=torch.int32)
    B.paged_attention_desc(q, cache, pages, q, 1, 5, 0.1)
    for bad in (lambda: B.rope_desc(q, table, q[:, :4]), lambda: B.rope_append_desc(q.transpose(0, 1), k, k, table, q.transpose(0, 1), cache),
                lambda: B.rope_append_desc(q, k, k, table, q, cache[..., :32]), lambda: B.rope_desc(q.int(), table, q.int()),
                lambda: B.paged_attention_desc(q, cache, pages[:, ::2], q, 1, 5, 0.1), lambda: B.qdense_w4_desc(q[0], q[0].t(), 32)):
        with pytest.raises(B.RelayError):
            bad()
