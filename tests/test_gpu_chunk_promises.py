"""Chunk attention where max_q_len is less than a sequence's new tokens: those past it are not computed, and every other sequence's
rows are as they should be."""
import pytest
import torch

from tests.test_gpu_chunk import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G,D", [(1, 128), (4, 64), (8, 128)])
@pytest.mark.parametrize("extra_pages", [0, 700])
def test_a_longer_chunk_than_promised_whose_first_tokens_are_padding(G, D, extra_pages):
    """The tokens that are computed all lie before position 0, by more than a tile: the sequence has no key to see."""
    q_lens, lens, most = [3, 200, 4, 150, 1, 4], [900, 100, 70, 10, 3000, 4], 4
    b = Batch(2 * G, 2, D, 16, q_lens=q_lens, lens=lens, seed=G, slopes=G == 4, extra_pages=extra_pages)
    got = b.run(0.1, most=most)
    want, size = b.wanted(0.1)
    bound = (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs() + 1e-30      # as for the chunk attention elsewhere
    t = 0
    for m in q_lens:
        done = min(m, most)
        assert bool(((got[t:t + done].double() - want[t:t + done]).abs() <= bound[t:t + done]).all()), t
        assert bool((got[t + done:t + m] == 7).all())
        t += m
    assert not got[3:7].any() and not got[207:211].any()            # padding: zero
