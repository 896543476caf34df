"""The sampler's gathering clears a number that all waves read behind its last barrier: between two gatherings of one workgroup there is a barrier on every way through the source."""
import os
import re

from paper_1904_08368_amd import binding as B

TEXT = open(os.path.join(os.path.dirname(B.__file__), "csrc", "sample.hip")).read()


def _body(head):
    at = TEXT.index("{", TEXT.index(head))
    depth = 0
    for i in range(at, len(TEXT)):
        depth += (TEXT[i] == "{") - (TEXT[i] == "}")
        if depth == 0:
            return TEXT[at:i + 1]


def test_a_barrier_before_each_gathering():
    within = _body("Place within(int b")
    loop = within.index("for (;;)")
    assert "__syncthreads()" in within[:loop]                              # behind whatever was gathered before
    again = within[within.index("if (shift == 0) break;"):]
    assert "__syncthreads()" in again[:again.index("count2[i] = 0")]      # ... and from one round to the next
    finish = _body("void finish(const SampleArgs& a")
    assert re.search(r"for \(;;\) \{.*?clear_bins\(\);.*?gather_", finish, re.S) and "__syncthreads()" in _body("void clear_bins()")
    assert len(re.findall(r"s\.listed = 0", TEXT)) == 1 and "s.listed = 0;\n    __syncthreads();" in TEXT
