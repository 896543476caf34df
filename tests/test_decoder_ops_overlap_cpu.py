"""Operands of a decoder's operators that overlap where one is written: refused on the host, before any HIP call."""
import os
import re

import pytest

from paper_1904_08368_amd import binding as B

from .test_decoder_ops_abi_cpu import _call_sample, _sample, at

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
