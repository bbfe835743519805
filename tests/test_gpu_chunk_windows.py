"""Chunk attention with windows up to the largest int, sequences of more new tokens than context among others."""
import pytest
import torch

from tests.test_gpu_chunk import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 64, 2 ** 31 - 200, 2 ** 30])
@pytest.mark.parametrize("G,D,bs", [(1, 128, 16), (4, 64, 32), (8, 128, 16)])
def test_windows_near_the_largest_int(window, G, D, bs):
    """A padded sequence's first rows have positions below 0: the first key its block sees is 0 all the same."""
    for q_lens, lens in (([130, 5, 1, 40], [100, 700, 65, 33]), ([4, 4, 4], [2, 1000, 1]), ([200, 1], [1, 3000])):
        b = Batch(2 * G, 2, D, bs, q_lens=q_lens, lens=lens, seed=G + len(lens), slopes=G == 4, lead=1, tail=2)
        got = b.check(window=window)
        assert torch.equal(got, b.run(D ** -0.5))           # as without a window: the tables bound the tiles of both alike


def test_more_items_than_a_wave():
    b = Batch(16, 8, 64, 16, q_lens=[3, 70] * 30, lens=[2, 61, 900, 300] * 15, seed=3)
    for window in (2 ** 31 - 1, 2 ** 31 - 3):
        b.check(window=window)
