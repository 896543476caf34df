"""Workspace sizes of a decoder's operators: what the largest call asks for serves every smaller one, so a program that sizes its scratch once for its largest batch is never refused."""
import ctypes as C

import pytest

from paper_1904_08368_amd import binding as B

from .test_decoder_ops_abi_cpu import _call_experts, _call_route, _call_sample, _experts, _route, _sample, at

COUNTS = sorted(set(range(1, 70)) | {16 * i + j for i in range(1, 40) for j in (0, 1, 15)} | {1000, 1023, 1024, 1025, 2048, 4095, 4096, 4097, 4500, 9000})


def _bytes(operator, d):
    b = C.c_size_t()
    assert getattr(B.lib(), f"relay_{operator}_workspace_bytes")(d, C.byref(b)) == 0
    return b.value


def _grows(operator, make, call):
    sizes = [_bytes(operator, make(n)) for n in COUNTS]
    assert sizes == sorted(sizes), [(n, a, b) for n, a, b in zip(COUNTS[1:], sizes, sizes[1:]) if a > b][:3]
    for n, size in zip(COUNTS, sizes):   # (6: a workspace that does not suffice; without a GPU a call that is accepted ends otherwise)
        assert call(make(n), ws=at(4000) if size else None, ws_bytes=size) != 6, n
    return sizes


@pytest.mark.parametrize("experts", [1, 8, 16, 17, 60, 64, 128, 256, 257, 1024])
@pytest.mark.parametrize("channels", [64, 512, 1024, 1536, 2048, 4096])
def test_router(experts, channels):
    _grows("route", lambda n: _route(tokens=n, channels=channels, x_stride=channels, experts=experts, top_k=1), lambda d, **kw: _call_route(d, **{k: at(200 * i) for i, k in enumerate(("x", "w", "bias", "chosen", "weights"))}, **kw))


@pytest.mark.parametrize("vocab", [100, 24000, 24774, 25000, 32000, 48000, 50257, 128000, 1 << 20])
def test_sampler(vocab):
    names = ("logits", "temperature", "top_k", "top_p", "min_p", "uniform", "tokens", "probs")
    sizes = _grows("sample", lambda n: _sample(rows=n, vocab=vocab, logits_stride=vocab), lambda d, **kw: _call_sample(d, **{k: at(10 * i + (8000 if i == 0 else 0)) for i, k in enumerate(names)}, **kw))
    assert (sizes[-1] > 0) == (vocab * 31 >= 24000 * 32)


@pytest.mark.parametrize("experts,top_k", [(1, 1), (8, 2), (64, 8), (128, 64)])
def test_experts(experts, top_k):
    names = ("x", "chosen", "weights", "gate_up", "down", "y")
    _grows("experts_w4", lambda n: _experts(tokens=n, experts=experts, top_k=top_k), lambda d, **kw: _call_experts(d, **{k: at(200 * i) for i, k in enumerate(names)}, **kw))
