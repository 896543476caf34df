"""Operands of a decoder's operators that overlap where one is written: refused on the host, before any HIP call."""
import ctypes as C
import os
import re

import pytest

from paper_1904_08368_amd import binding as B

from .test_decoder_ops_abi_cpu import _call_experts, _call_route, _call_sample, _experts, _route, _sample, _status, at

SETTINGS = {"temperature": 1, "top_k": 2, "top_p": 3, "min_p": 4, "uniform": 5}


@pytest.mark.parametrize("name", SETTINGS)
@pytest.mark.parametrize("output", ["tokens", "probs"])
@pytest.mark.parametrize("off", [0, 4, 8, -4, -8])
def test_sample_refuses_outputs_that_are_settings(name, output, off):
    assert _call_sample(_sample(), **{output: at(SETTINGS[name]) + off}) == 4 and b"setting" in B.lib().relay_last_error()


def test_sampling_reads_no_output():
    """The kernels only write tokens and probs: no load of a row's settings goes there in the place of one that is not given."""
    text = open(os.path.join(os.path.dirname(B.__file__), "csrc", "sample.hip")).read()
    uses = re.findall(r"a\.(?:tokens|probs)\b.*", text)
    assert uses and all(re.match(r"a\.(tokens|probs)(\[r\] = |\) a\.probs\[r\] = )", u) for u in uses), uses


def _need(operator, d):
    b = C.c_size_t()
    assert _status(f"relay_{operator}_workspace_bytes", d, C.byref(b)) == 0 and b.value > 0
    return b.value


OPERANDS = {"route": (_call_route, _route, dict(x=640, w=1024, bias=32, chosen=40, weights=40)),
            "experts_w4": (_call_experts, lambda: _experts(flags=B.HAS_RESIDUAL), dict(x=640, chosen=40, weights=40, gate_up=32 * 1024 + 32 * 2 * 32, down=32 * 1024 + 32 * 32, residual=640, y=640)),
            "sample": (_call_sample, lambda: _sample(vocab=200000, logits_stride=200000), dict(logits=1200000, temperature=12, top_k=12, top_p=12, min_p=12, uniform=12, tokens=12, probs=12))}


@pytest.mark.parametrize("operator,name", [(o, n) for o, v in OPERANDS.items() for n in v[2]])
def test_operands_in_the_workspace(operator, name):
    """At its start, its end, and around it; beside it they are no reason to refuse (without a GPU the call then ends with another status)."""
    call, desc, sizes = OPERANDS[operator]
    need, size = _need(operator, desc()), -(-sizes[name] // 256) * 256
    given = dict(ws=at(40), ws_bytes=need)
    if operator == "experts_w4":
        given["residual"] = at(5)
    for place, refused in ((at(40), True), (at(40) + (need - 1) // 256 * 256, True), (at(40) - size + 256, True), (at(40) - size, False), (at(40) + -(-need // 256) * 256, False)):
        status = call(desc(), **{**given, name: place})
        assert (status == 4 and b"workspace" in B.lib().relay_last_error()) == refused or (refused and name == "y" and place == at(40) and status == 4), (place - at(40), status)


def test_a_workspace_between_the_rows_of_an_operand():
    """Rows that are far apart may have it between them, not in one of them."""
    for operator, (call, desc, _) in OPERANDS.items():
        name, stride, es = ("logits", "logits_stride", 2) if operator == "sample" else ("x", "x_stride", 2)
        given = dict(ws=at(40), ws_bytes=_need(operator, desc()))
        if operator == "experts_w4":
            given["residual"] = at(5)
        far = lambda: _set(desc(), stride, (1 << 22) // es)
        assert call(far(), **{**given, name: at(40) - (1 << 21)}) != 4
        assert call(far(), **{**given, name: at(40) - (1 << 22)}) == 4 and b"workspace" in B.lib().relay_last_error()


def _set(d, field, value):
    setattr(d._obj, field, value)
    return d


def test_strides_at_the_end_of_their_type():
    """A call of one row may have any stride: it is not multiplied out as a signed number."""
    far = 2 ** 63 - 8
    for operator, (call, desc, _) in OPERANDS.items():
        d = _set(_set(desc(), "rows" if operator == "sample" else "tokens", 1), "logits_stride" if operator == "sample" else "x_stride", far)
        given = dict(ws=at(40), ws_bytes=_need(operator, d))
        if operator == "experts_w4":
            given["residual"] = at(5)
        assert call(d, **given) not in (2, 4, 6)
