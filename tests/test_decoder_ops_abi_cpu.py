"""The entry points of a decoder's operators beside its attention layer without a GPU: what they refuse, with which status, before any HIP call; calls
that launch nothing; tensors that a descriptor cannot describe."""
import ctypes as C

import pytest
import torch

from paper_1904_08368_amd import binding as B

FAKE = 0x7F0000001000            # a non-NULL, 4096-byte aligned address that is never dereferenced
at = lambda i: FAKE + (i << 24)


def _status(fn, *args):
    return getattr(B.lib(), fn)(*args)


def _with(d, **kw):
    for k, v in kw.items():
        setattr(d, k, v)
    return C.byref(d)


# ---------------------------------------------------------------------------------- norms
def _norm(**kw):
    return _with(B.ResidualNormDesc(B.RELAY_F16, 4, 64, B.NORM_RMS, B.NORM_LAYER, 1e-5, 1e-5, 1.0, 1.0, 64, 64, 0, 64, 64), **kw)


def _call_norm(d, **kw):
    names = ("x", "residual", "gate", "post_weight", "post_bias", "pre_weight", "pre_bias", "sum", "y")
    return _status("relay_residual_norm", d, *[kw.get(n, at(i)) for i, n in enumerate(names)], None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=B.RELAY_I8), 3), (dict(dtype=7), 3), (dict(tokens=-1), 2), (dict(channels=0), 2), (dict(channels=32769), 2),
    (dict(dtype=B.RELAY_F32, channels=16385), 2), (dict(post=3), 4), (dict(pre=-1), 4), (dict(post_eps=-1e-6), 2), (dict(pre_eps=NAN), 2),
    (dict(post_eps=INF), 2), (dict(branch_scale=INF), 2), (dict(residual_scale=NAN), 2), (dict(x_stride=-1), 2), (dict(residual_stride=-64), 2),
    (dict(gate_stride=-1), 2), (dict(sum_stride=63), 2), (dict(y_stride=0), 2)])
def test_norm_refuses(kw, status):
    assert _call_norm(_norm(**kw)) == status and B.lib().relay_last_error()


def test_norm_pointers():
    assert _call_norm(None) == 1
    assert _call_norm(_norm(), x=None) == 1
    assert _call_norm(_norm(), y=None) == 1                                                  # a norm without a place for it
    assert _call_norm(_norm(pre=B.NORM_NONE), pre_weight=None, pre_bias=None) == 1           # ... and a place without a norm
    assert _call_norm(_norm(pre=B.NORM_NONE), pre_weight=None, pre_bias=None, y=None, sum=None) == 1
    assert _call_norm(_norm(pre=B.NORM_NONE), pre_bias=None, y=None) == 4                    # a weight without its norm
    assert _call_norm(_norm(post=B.NORM_NONE)) == 4
    for name in ("x", "residual", "gate", "post_weight", "post_bias", "pre_weight", "pre_bias", "sum", "y"):
        assert _call_norm(_norm(), **{name: at(20) + 1}) == 5
    assert _call_norm(_norm(), post_weight=at(20) + 2) == 5
    assert _call_norm(_norm(), sum=at(8)) == 4                                               # one place for both outputs
    assert _call_norm(_norm(x_stride=128), sum=at(0)) == 4                                   # in place with other strides
    assert _call_norm(_norm(), y=at(2)) == 4                                                 # in place of a gate that all tokens share
    assert _call_norm(_norm(tokens=0), x=None, y=None, sum=None) == 0


def _f16(*shape):
    return torch.zeros(shape, dtype=torch.float16)


def test_norm_descriptors():
    x = _f16(4, 64)
    d = B.residual_norm_desc(x, x, _f16(1, 64), None, x)
    assert (d.gate_stride, d.x_stride, d.sum_stride) == (0, 64, 64)
    assert B.residual_norm_desc(x, None, _f16(4, 128)[:, :64], x, None).gate_stride == 128
    for bad in (lambda: B.residual_norm_desc(x.t(), None, None, None, x.t()), lambda: B.residual_norm_desc(x, x.float(), None, None, x),
                lambda: B.residual_norm_desc(x, _f16(4, 65), None, None, x), lambda: B.residual_norm_desc(x, None, None, _f16(3, 64), x),
                lambda: B.residual_norm_desc(x, None, None, None, _f16(64, 4).t()), lambda: B.residual_norm_desc(x.int(), None, None, None, x.int()),
                lambda: B.residual_norm_desc(x, None, _f16(2, 64), None, x), lambda: B.residual_norm_desc(x[0], None, None, None, x[0])):
        with pytest.raises((B.RelayError, RuntimeError)):
            bad()
    w = torch.ones(64)
    for bad in (w.double(), w[:63], torch.ones(128)[::2], w.half()):
        with pytest.raises(B.RelayError):
            B.relay_residual_norm(d, x, x, None, None, None, bad, None, None, x)


# ------------------------------------------------------------------------------- sampling
def _sample(**kw):
    return _with(B.SampleDesc(B.RELAY_BF16, 3, 100, 100), **kw)


def _call_sample(d, ws=None, ws_bytes=0, **kw):
    names = ("logits", "temperature", "top_k", "top_p", "min_p", "uniform", "tokens", "probs")
    return _status("relay_sample", d, *[kw.get(n, at(i)) for i, n in enumerate(names)], ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [(dict(dtype=B.RELAY_I8), 3), (dict(rows=-1), 2), (dict(vocab=0), 2), (dict(vocab=(1 << 20) + 1), 2), (dict(logits_stride=-1), 2)])
def test_sample_refuses(kw, status):
    b = C.c_size_t()
    assert _call_sample(_sample(**kw)) == status
    assert _status("relay_sample_workspace_bytes", _sample(**kw), C.byref(b)) == status


def test_sample_pointers():
    assert _call_sample(None) == 1 and _call_sample(_sample(), logits=None) == 1 and _call_sample(_sample(), tokens=None) == 1
    assert _status("relay_sample_workspace_bytes", _sample(), None) == 1
    for name in ("logits", "temperature", "top_k", "top_p", "min_p", "uniform", "tokens", "probs"):
        assert _call_sample(_sample(), **{name: at(20) + 1}) == 5
    assert _call_sample(_sample(), tokens=at(0)) == 4 and _call_sample(_sample(), probs=at(6)) == 4 and _call_sample(_sample(), probs=at(0)) == 4
    assert _call_sample(_sample(rows=0), logits=None, tokens=None) == 0


def test_sample_operands():
    l = torch.zeros(3, 100)
    d = B.sample_desc(l)
    assert (d.rows, d.vocab, d.logits_stride) == (3, 100, 100) and B.sample_desc(torch.zeros(3, 128)[:, :100]).logits_stride == 128
    for bad in (l.t(), l[0], l.int()):
        with pytest.raises(B.RelayError):
            B.sample_desc(bad)
    good = dict(temperature=torch.ones(3), top_k=torch.ones(3, dtype=torch.int32), top_p=torch.ones(3), min_p=torch.ones(3), uniform=torch.ones(3),
                tokens=torch.zeros(3, dtype=torch.int32), probs=torch.zeros(3))
    for name, bad in (("temperature", torch.ones(2)), ("top_k", torch.ones(3)), ("top_k", torch.ones(3, dtype=torch.int64)), ("top_p", torch.ones(3).half()),
                      ("min_p", torch.ones(6)[::2]), ("uniform", torch.ones(3).double()), ("tokens", torch.zeros(3, dtype=torch.int64)),
                      ("tokens", torch.zeros(2, dtype=torch.int32)), ("tokens", None), ("probs", torch.zeros(2))):
        with pytest.raises(B.RelayError):
            B.relay_sample(d, l, **{**good, name: bad})


# -------------------------------------------------------------------------------- routing
def _route(**kw):
    return _with(B.RouteDesc(B.RELAY_F16, 5, 64, 8, 2, B.SCORE_SOFTMAX, 1, 1.0, 64), **kw)


def _call_route(d, ws=at(9), ws_bytes=1 << 30, **kw):
    names = ("x", "w", "bias", "chosen", "weights")
    return _status("relay_route", d, *[kw.get(n, at(i)) for i, n in enumerate(names)], ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=B.RELAY_F32), 3), (dict(tokens=-1), 2), (dict(channels=0), 2), (dict(channels=60), 5), (dict(experts=0), 2), (dict(experts=1025), 2),
    (dict(channels=(1 << 24) + 8), 2), (dict(channels=0x7ffffff8), 2), (dict(top_k=0), 2), (dict(top_k=9), 2), (dict(experts=100, top_k=65), 2), (dict(score=2), 4), (dict(normalize=2), 4), (dict(scale=INF), 2), (dict(scale=NAN), 2),
    (dict(x_stride=-8), 2), (dict(x_stride=68), 5)])
def test_route_refuses(kw, status):
    b = C.c_size_t()
    assert _call_route(_route(**kw)) == status
    assert _status("relay_route_workspace_bytes", _route(**kw), C.byref(b)) == status


def test_route_pointers():
    b = C.c_size_t()
    assert _call_route(None) == 1 and _status("relay_route_workspace_bytes", _route(), None) == 1
    for name in ("x", "w", "chosen", "weights"):
        assert _call_route(_route(), **{name: None}) == 1
    for name, off in (("x", 8), ("w", 8), ("bias", 2), ("chosen", 2), ("weights", 2)):
        assert _call_route(_route(), **{name: at(20) + off}) == 5
    for name, other in (("chosen", 4), ("weights", 2), ("chosen", 0), ("weights", 1)):
        assert _call_route(_route(), **{name: at(other)}) == 4
    assert _status("relay_route_workspace_bytes", _route(), C.byref(b)) == 0 and b.value > 0
    assert _call_route(_route(), ws=None) == 6 and _call_route(_route(), ws_bytes=b.value - 1) == 6 and _call_route(_route(), ws=at(9) + 128) == 5
    assert _call_route(_route(tokens=0), ws=None, x=None, w=None, chosen=None, weights=None) == 0


def test_route_operands():
    x, w, chosen, weights = _f16(5, 64), _f16(8, 64), torch.zeros(5, 2, dtype=torch.int32), torch.zeros(5, 2)
    d = B.route_desc(x, w, chosen)
    assert (d.tokens, d.channels, d.experts, d.top_k, d.x_stride) == (5, 64, 8, 2, 64)
    for bad in (lambda: B.route_desc(x, w.float(), chosen), lambda: B.route_desc(x, _f16(8, 72), chosen), lambda: B.route_desc(x, _f16(64, 8).t(), chosen),
                lambda: B.route_desc(x, w, chosen[:4]), lambda: B.route_desc(_f16(64, 5).t(), w, chosen),
                lambda: B.relay_route(d, x, w, torch.zeros(7), chosen, weights, None), lambda: B.relay_route(d, x, w, None, chosen.long(), weights, None),
                lambda: B.relay_route(d, x, w, None, chosen, weights.half(), None), lambda: B.relay_route(d, x, w, None, chosen, weights[:4], None),
                lambda: B.relay_route(d, x, w, None, chosen, None, None), lambda: B.relay_route(d, x, w, None, None, weights, None)):
        with pytest.raises(B.RelayError):
            bad()


# -------------------------------------------------------------------------------- experts
def _experts(**kw):
    return _with(B.ExpertsW4Desc(B.RELAY_BF16, 5, 2, 64, 32, 8, 32, 0, B.ACT_SILU, 0, 64, 64), **kw)


def _call_experts(d, ws=at(9), ws_bytes=1 << 30, **kw):
    names = ("x", "chosen", "weights", "gate_up", "down", "residual", "y")
    return _status("relay_experts_w4", d, *[kw.get(n, None if n == "residual" else at(i)) for i, n in enumerate(names)], ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=B.RELAY_F32), 3), (dict(tokens=-1), 2), (dict(top_k=0), 2), (dict(top_k=65), 2), (dict(channels=0), 2), (dict(channels=72), 5), (dict(inter=0), 2),
    (dict(inter=40), 5), (dict(experts=0), 2), (dict(experts=1025), 2), (dict(experts=1000, inter=1 << 21), 2), (dict(experts=1, inter=(1 << 29) + 16), 2), (dict(experts=1000, channels=1 << 22, y_stride=1 << 22), 2),
    (dict(group=0), 2), (dict(group=48), 2), (dict(has_zeros=2), 4), (dict(act=2), 4), (dict(flags=B.RELU), 4), (dict(flags=64), 4), (dict(x_stride=-8), 2),
    (dict(x_stride=68), 5), (dict(y_stride=63), 2)])
def test_experts_refuse(kw, status):
    b = C.c_size_t()
    assert _call_experts(_experts(**kw)) == status
    assert _status("relay_experts_w4_workspace_bytes", _experts(**kw), C.byref(b)) == status


def test_experts_pointers():
    b = C.c_size_t()
    assert _call_experts(None) == 1 and _status("relay_experts_w4_workspace_bytes", _experts(), None) == 1
    for name in ("x", "chosen", "weights", "gate_up", "down", "y"):
        assert _call_experts(_experts(), **{name: None}) == 1
    assert _call_experts(_experts(), residual=at(5)) == 1 and _call_experts(_experts(flags=B.HAS_RESIDUAL)) == 1
    for name, off in (("x", 8), ("chosen", 2), ("weights", 1), ("gate_up", 8), ("down", 4), ("y", 1)):
        assert _call_experts(_experts(), **{name: at(20) + off}) == 5
    assert _call_experts(_experts(flags=B.HAS_RESIDUAL), residual=at(5) + 1) == 5
    for other in (0, 1, 2, 3, 4, 9):
        assert _call_experts(_experts(), y=at(other)) == 4
    assert _status("relay_experts_w4_workspace_bytes", _experts(), C.byref(b)) == 0 and b.value > 0
    assert _call_experts(_experts(), ws=None) == 6 and _call_experts(_experts(), ws_bytes=b.value - 1) == 6 and _call_experts(_experts(), ws=at(9) + 128) == 5
    assert _call_experts(_experts(tokens=0), ws=None, x=None, chosen=None, weights=None, gate_up=None, down=None, y=None) == 0


def test_experts_operands():
    x, y, chosen, weights = _f16(5, 64), _f16(5, 64), torch.zeros(5, 2, dtype=torch.int32), torch.zeros(5, 2)
    d = B.experts_w4_desc(x, chosen, y, 8, 32, 32)
    assert (d.tokens, d.top_k, d.channels, d.inter, d.experts, d.flags) == (5, 2, 64, 32, 8, 0)
    assert d.packed_bytes == (32 * 1024 + 32 * 2 * 32, 32 * 1024 + 32 * 32)
    up, down = (torch.zeros(n, dtype=torch.uint8) for n in d.packed_bytes)
    call = lambda **kw: B.relay_experts_w4(*[{**dict(d=d, x=x, chosen=chosen, weights=weights, gate_up=up, down=down, residual=None, y=y, workspace=None), **kw}[n] for n in
                                             ("d", "x", "chosen", "weights", "gate_up", "down", "residual", "y", "workspace")])
    for bad in (lambda: B.experts_w4_desc(x, chosen, y.bfloat16(), 8, 32, 32), lambda: B.experts_w4_desc(x, chosen, _f16(5, 80), 8, 32, 32),
                lambda: B.experts_w4_desc(x, chosen[:4], y, 8, 32, 32), lambda: B.experts_w4_desc(x, chosen, y, 8, 32, 32, residual=_f16(5, 80)[:, :64]),
                lambda: B.experts_w4_desc(_f16(64, 5).t(), chosen, y, 8, 32, 32), lambda: call(chosen=chosen.long()), lambda: call(chosen=None),
                lambda: call(weights=weights.half()), lambda: call(weights=weights[:4]), lambda: call(gate_up=up[1:]), lambda: call(down=down[:100])):
        with pytest.raises(B.RelayError):
            bad()
