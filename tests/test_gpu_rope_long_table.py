"""A table of as many positions as its descriptor can name: 2^31 - 1 rows of one pair, 16 GiB."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_table_of_2_31_rows():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1904_08368_amd import binding as B
    rows = 2 ** 31 - 1
    out = torch.empty((rows + 1, 1, 2), device="cuda:0")   # (the row behind the last stays as it is)
    out[-1] = 7.0
    B.relay_rope_table(B.rope_table_desc(rows, 2), out[:rows])
    torch.cuda.synchronize()
    at = torch.tensor([0, 1, 16383, 16384, 2 ** 20 + 1, 2 ** 30, 2 ** 31 - 20000, 2 ** 31 - 3, 2 ** 31 - 2])
    a = at.double().numpy()
    # the angle is the position itself: exact, reduced in 64 bits to 2^-52 x 2^31
    want = np.stack([np.cos(a), np.sin(a)], -1)
    assert np.abs(out[at.cuda(), 0].double().cpu().numpy() - want).max() <= 2.0 ** -24 + 2.0 ** -20
    assert (out[-1] == 7).all()
