"""Rotary positions against 64 bits: both layouts, parts of a head, odd sizes and strides, the gradient, the store into a paged cache,
tables stretched for long contexts."""
import numpy as np
import pytest
import torch

from oracle import attention as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": (torch.float16, 2.0 ** -11, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -133), "f32": (torch.float32, 2.0 ** -24, 2.0 ** -149)}
STYLE = {"half": 0, "interleaved": 1}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1904_08368_amd import binding
    return binding


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _rand(shape, dtype, seed):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)).to(TYPES[dtype][0])


def _table(rows, rd, first=0):
    a = (first + np.arange(rows))[:, None] * O.rope_frequencies(rd, 10000.0)
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def _check(got, want, x, dtype):
    """Two products and a sum in fp32: 2^-23 of the pair's magnitude, below |x|'s largest; then one rounding."""
    _, u, tiny = TYPES[dtype]
    tol = 2.0 ** -23 * 2 * np.abs(x).max(-1, keepdims=True) + u * np.abs(want) + tiny
    assert not np.isnan(got).any()
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("style", ["half", "interleaved"])
@pytest.mark.parametrize("tokens,heads,dim,rd", [(1, 1, 2, 2), (1, 8, 128, 128), (7, 3, 80, 32), (5, 2, 80, 80), (3, 5, 96, 48), (9, 1, 66, 34),
                                                 (2, 3, 33, 10), (130, 4, 64, 64), (4, 2, 256, 8), (600, 16, 128, 128)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_matches_the_formula(B, dtype, style, tokens, heads, dim, rd, inverse):
    x = _rand((tokens, heads, dim), dtype, tokens * 1000 + dim)
    table = _table(50, rd, 1000)
    pos = np.random.default_rng(3).integers(0, 50, tokens).astype(np.int32)
    xd, td, pd = x.to(DEV), torch.from_numpy(table).to(DEV), torch.from_numpy(pos).to(DEV)
    y = torch.full_like(xd, float("nan"))
    B.relay_rope(B.rope_desc(xd, td, y, STYLE[style], inverse), xd, td, pd, y)
    torch.cuda.synchronize()
    _check(_np(y), O.rope(_np(x), table, pos, style, inverse), _np(x), dtype)
    # in place
    B.relay_rope(B.rope_desc(xd, td, xd, STYLE[style], inverse), xd, td, pd, xd)
    assert torch.equal(xd, y)


@pytest.mark.parametrize("dtype,style", [("f16", "half"), ("bf16", "interleaved"), ("f32", "half")])
@pytest.mark.parametrize("offset", [0, 1])
def test_rope_on_views(B, dtype, style, offset):
    """A head-major view of a wider tensor, on 16-byte boundaries and off them; what lies between the rows stays as it was."""
    t, h, d, rd = 11, 3, 64, 32
    wide = _rand((h, t, d + 24), dtype, 5).to(DEV)
    out = torch.full_like(wide, 7.0)
    x, y = (w[:, :, 8 + offset:8 + offset + d].transpose(0, 1) for w in (wide, out))
    table, pos = _table(t, rd), np.arange(t, dtype=np.int32)[::-1].copy()
    td, pd = torch.from_numpy(table).to(DEV), torch.from_numpy(pos).to(DEV)
    B.relay_rope(B.rope_desc(x, td, y, STYLE[style]), x, td, pd, y)
    torch.cuda.synchronize()
    _check(_np(y), O.rope(_np(x), table, pos, style), _np(x), dtype)
    assert (out[:, :, :8 + offset] == 7).all() and (out[:, :, 8 + offset + d:] == 7).all()


def test_position_outside_the_table(B):
    x = _rand((4, 2, 16), "f16", 1).to(DEV)
    y, td = torch.zeros_like(x), torch.from_numpy(_table(3, 8)).to(DEV)
    pos = torch.tensor([0, -1, 3, 2], dtype=torch.int32, device=DEV)
    B.relay_rope(B.rope_desc(x, td, y), x, td, pos, y)
    torch.cuda.synchronize()
    bad = torch.isnan(y)
    assert bad[1:3, :, :8].all() and not bad[[0, 3]].any() and not bad[:, :, 8:].any()
    assert torch.equal(y[:, :, 8:], x[:, :, 8:])


@pytest.mark.parametrize("style", ["half", "interleaved"])
def test_gradient_against_differences(B, style):
    """The inverse call is the gradient: <g, rope(x + h d) - rope(x - h d)> / 2h equals <rope_inverse(g), d>.  The map is linear, so
    the difference is exact up to rounding; fp32 sums of 2 x 3 x 48 products of normal values: 288 x 2^-23 x 8, over h = 1."""
    t, h, d, rd = 2, 3, 48, 32
    table, pos = _table(20, rd), np.array([7, 19], dtype=np.int32)
    td, pd = torch.from_numpy(table).to(DEV), torch.from_numpy(pos).to(DEV)
    x, g, e = (_rand((t, h, d), "f32", s).to(DEV) for s in (1, 2, 3))

    def call(v, inverse=False):
        y = torch.empty_like(v)
        B.relay_rope(B.rope_desc(v, td, y, STYLE[style], inverse), v, td, pd, y)
        return y.double()
    diff = ((call(x + e) - call(x - e)) / 2 * g.double()).sum()
    grad = (call(g, True) * e.double()).sum()
    assert abs(float(diff - grad)) <= 288 * 2.0 ** -23 * 8


@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "by_parts"])
@pytest.mark.parametrize("first,rows,rd", [(0, 5, 2), (0, 300, 128), (999999, 17, 64)])
def test_table(B, scaling, first, rows, rd):
    if scaling == "base" and rd == 2:
        pytest.skip("refused: no exponent")
    code = {"plain": B.ROPE_PLAIN, "linear": B.ROPE_LINEAR, "base": B.ROPE_BASE, "by_parts": B.ROPE_BY_PARTS}[scaling]
    out = torch.full((rows, rd // 2, 2), float("nan"), device=DEV)
    B.relay_rope_table(B.rope_table_desc(rows, rd, 500000.0, first, code, 8.0, 1.0, 32.0, 4096.0, 1.25), out)
    torch.cuda.synchronize()
    a = (first + np.arange(rows, dtype=np.float64))[:, None] * O.rope_frequencies(rd, 500000.0, scaling, 8.0, 1.0, 32.0, 4096.0)
    want = 1.25 * np.stack([np.cos(a), np.sin(a)], -1)
    # angles of a million in 64 bits: 2^-52 x 2^20 x a few operations, far below the fp32 rounding of the result
    assert np.abs(_np(out) - want).max() <= 1.25 * 2.0 ** -24 + 1e-8


def _append(B, dtype, tokens, hq, hkv, dim, rd, style, ps, pages, slots, hnd=False, packed=True, offset=0):
    tt = TYPES[dtype][0]
    width = (hq + 2 * hkv) * dim
    if packed:
        qkv = _rand((tokens, width + offset), dtype, 11).to(DEV)[:, offset:]
        q, k, v = (qkv[:, a:b].unflatten(1, (-1, dim)) for a, b in ((0, hq * dim), (hq * dim, (hq + hkv) * dim), ((hq + hkv) * dim, width)))
    else:
        q, k, v = (_rand((tokens, h, dim), dtype, 12 + h).to(DEV) for h in (hq, hkv, hkv))
    shape = (pages, hkv, ps, dim) if hnd else (pages, ps, hkv, dim)
    kc, vc = (_rand(shape, dtype, s).to(DEV) for s in (21, 22))
    if hnd:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    pos = np.random.default_rng(4).integers(0, 40, tokens).astype(np.int32)
    table = _table(40, rd, 123)
    td, pd, sd = torch.from_numpy(table).to(DEV), torch.from_numpy(pos).to(DEV), torch.tensor(slots, dtype=torch.int32, device=DEV)
    qo = torch.full((tokens, hq, dim), float("nan"), dtype=tt, device=DEV)
    k0, v0 = _np(kc), _np(vc)
    B.relay_rope_append(B.rope_append_desc(q, k, v, td, qo, kc, STYLE[style]), q, k, v, td, pd, sd, qo, kc, vc)
    torch.cuda.synchronize()
    _check(_np(qo), O.rope(_np(q), table, pos, style), _np(q), dtype)
    kr, kn, vn, kg, vg = O.rope(_np(k), table, pos, style), _np(k), _np(v), _np(kc), _np(vc)
    wrote = np.zeros((pages, ps), dtype=bool)
    for t, s in enumerate(slots):
        if 0 <= s < pages * ps:
            wrote[s // ps, s % ps] = True
            _check(kg[s // ps, s % ps], kr[t], kn[t], dtype)
            assert np.array_equal(vg[s // ps, s % ps], vn[t])
    # every other slot is as it was
    assert np.array_equal(kg[~wrote], k0[~wrote]) and np.array_equal(vg[~wrote], v0[~wrote])


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("tokens,hq,hkv,dim,rd,style,ps", [(1, 8, 2, 128, 128, "half", 16), (1, 1, 1, 8, 8, "interleaved", 1), (37, 6, 2, 80, 32, "interleaved", 24),
                                                           (37, 6, 2, 80, 32, "half", 5), (21, 4, 4, 40, 20, "half", 16), (700, 24, 8, 96, 96, "half", 32)])
@pytest.mark.parametrize("hnd", [False, True])
def test_append(B, dtype, tokens, hq, hkv, dim, rd, style, ps, hnd):
    pages = (tokens + ps - 1) // ps + 2
    slots = np.random.default_rng(tokens).permutation(pages * ps)[:tokens].tolist()
    _append(B, dtype, tokens, hq, hkv, dim, rd, style, ps, pages, slots, hnd)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_append_skips_padding_tokens_and_slots_outside(B, dtype):
    _append(B, dtype, 6, 4, 2, 64, 64, "half", 4, 3, [2, -1, 12, 11, -2147483648, 2147483647])


@pytest.mark.parametrize("packed,offset", [(False, 0), (True, 1), (True, 8)])
def test_append_sources(B, packed, offset):
    _append(B, "bf16", 9, 4, 2, 64, 32, "half", 8, 3, list(range(3, 12)), packed=packed, offset=offset)


def test_append_beyond_32_bit_offsets(B):
    """A cache whose last page starts 2^32 + elements in: 5 GiB of address space per tensor, of which the test touches a few pages."""
    hkv, dim, ps, pages = 2, 64, 16, 3
    stride = (1 << 31) + 4096
    kc, vc = (torch.empty(2 * stride + ps * hkv * dim, dtype=torch.float16, device=DEV).as_strided((pages, ps, hkv, dim), (stride, hkv * dim, dim, 1))
              for _ in range(2))
    q, k, v = (_rand((3, h, dim), "f16", 30 + h).to(DEV) for h in (4, 2, 2))
    table = _table(8, dim)
    td = torch.from_numpy(table).to(DEV)
    pos, slots = torch.tensor([0, 3, 7], dtype=torch.int32, device=DEV), torch.tensor([5, 17, 47], dtype=torch.int32, device=DEV)
    qo = torch.empty_like(q)
    B.relay_rope_append(B.rope_append_desc(q, k, v, td, qo, kc), q, k, v, td, pos, slots, qo, kc, vc)
    torch.cuda.synchronize()
    want = O.rope(_np(k), table, [0, 3, 7], "half")
    for t, (p, s) in enumerate([(0, 5), (1, 1), (2, 15)]):
        _check(_np(kc[p, s]), want[t], _np(k[t]), "f16")
        assert torch.equal(vc[p, s], v[t])


def test_no_tokens(B):
    x = torch.empty((0, 2, 16), dtype=torch.float16, device=DEV)
    td = torch.zeros((3, 8, 2), device=DEV)
    B.relay_rope(B.rope_desc(x, td, x), x, td, torch.empty(0, dtype=torch.int32, device=DEV), x)
