"""Shared-prefix decode on the GPU: keys that are not numbers reach the rows that see them, and no others."""
import pytest
import torch

from tests.test_gpu_decode_shared import DEV, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("steep", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_keys_that_are_not_numbers_reach_every_row_that_sees_them(shared, steep):
    """All keys of a tile are NaN, or (steep slopes) one key of a tile whose other weights are zero; the values are numbers.
    The tiles are taken from the last one backwards, so that every row has a maximum when it comes to them."""
    b = Batch(16, 4, 128, 16, sizes=[4], prefix=[320], lens=[400, 410, 200, 500])
    if steep:
        b.slopes = torch.full((16,), 3.0, device=DEV)       # 30 tokens further back a weight is below 2^-127
    before = b.check()
    if shared:
        pages = b.table[0, 16:20] if not steep else b.table[0, 4:5]     # tokens 256 to 319, past sequence 2's end; 64 to 79
    else:
        pages = b.table[3, 24:28] if not steep else b.table[3, 24:25]   # 384 to 447 of sequence 3; 384 to 399
    keys = b.k[pages.long()]
    if steep:
        keys[0, 1, 6, 100] = float("nan")
    else:
        keys[:, 1] = float("nan")
    b.k[pages.long()] = keys
    got = b.run(128 ** -0.5)
    bad = torch.isnan(b.wanted(128 ** -0.5)[0])
    rows = [0, 1, 3] if shared and not steep else [0, 1, 2, 3] if shared else [3]
    assert bad[rows, 4:8].all() and int(bad.sum()) == len(rows) * 4 * 128
    assert torch.equal(torch.isnan(got), bad) and torch.equal(got[~bad], before[~bad])
