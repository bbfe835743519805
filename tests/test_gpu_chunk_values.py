"""How far values that are not finite reach in the chunk attention: new tokens of their own sequence, under their own KV head."""
import pytest
import torch

from tests.test_gpu_chunk import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("extra_pages", [0, 700])
@pytest.mark.parametrize("n", [700, 741])
def test_a_value_row_that_is_not_finite(value, extra_pages, n):
    """Blocks of 32 tokens (G 4), tiles of 64 keys.  Tokens that see the key have it; others of the sequence may where their block
    has the key's tile (a weight of 0 times what is not finite); all others are as without it."""
    b = Batch(8, 2, 128, 16, q_lens=[70, 5, 1], lens=[n, 400, 300], seed=1, extra_pages=extra_pages)
    want = b.run(0.1)
    for token in (40, 69):
        key = n - 70 + token
        page, row = b.table[0, key // 16].long(), key % 16
        kept = b.v[page, 1, row].clone()
        b.v[page, 1, row] = value
        got = b.run(0.1)
        b.v[page, 1, row] = kept
        assert not torch.isfinite(got[token:70, 4:].float()).any()
        assert torch.equal(got[:70, :4], want[:70, :4])             # the other KV head
        for block in range(0, 70, 32):
            last = n - 70 + min(block + 32, 70) - 1
            if last // 64 < key // 64:
                assert torch.equal(got[block:block + 32], want[block:block + 32])
        assert torch.equal(got[70:], want[70:])
    assert torch.equal(b.run(0.1), want)


def test_a_refused_draft_reaches_no_other_sequence():
    """Sequences whose blocks are at work side by side in one CTA, by the list and by an item each."""
    for extra_pages in (0, 700):
        b = Batch(8, 2, 64, 16, q_lens=[4] * 12, lens=[100 + 31 * i for i in range(12)], seed=2, extra_pages=extra_pages)
        want = b.run(0.1)
        for s in range(0, 12, 3):
            key = b.n[s] - 1
            b.v[b.table[s, key // 16].long(), :, key % 16] = float("inf")
        got = b.run(0.1)
        for s in range(12):
            rows = slice(4 * s, 4 * s + 4)
            if s % 3:
                assert torch.equal(got[rows], want[rows])
            else:
                assert not torch.isfinite(got[4 * s + 3].float()).any()
