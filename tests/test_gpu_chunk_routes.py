"""Which route a batch of more items than a wave takes: a CTA per item leaves the workspace as it was, the list writes its flags there.
The host bounds the contexts by the tables' width (or the window); results are checked on either route."""
import numpy as np
import pytest
import torch

from paper_2505_02351_b200 import binding
from tests.test_gpu_chunk import DEV, Batch

pytestmark = pytest.mark.gpu


def bounds(b, window=0):
    """(items, tiles of the longest, bytes of the keys and values behind all) as the host has them."""
    D, bs = b.q.shape[2], b.bs
    tiles = b.table.shape[1] * bs // 64 + 1
    if window:
        tiles = min(tiles, (window + 128 // b.G + 62) // 64 + 1)
    return -(-max(b.q_lens) * b.G // 128) * b.Hkv * b.B, tiles, b.B * b.Hkv * D * 4 * 64 * tiles


def by_list(b, window=0):
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the bounds here are those of 148 multiprocessors")
    scale = b.q.shape[2] ** -0.5
    need = binding.chunk_workspace_bytes(b.q.shape[1], b.Hkv, b.q.shape[2], max(b.q_lens))
    ws = torch.full((need,), 0xa5, device=DEV, dtype=torch.uint8)
    got = b.run(scale, window, ws=ws)
    torch.cuda.synchronize()
    assert binding.device_status() == 0
    want, size = b.wanted(scale, window)
    # roundings as for the chunk attention elsewhere: weights twice, the result once, 2^-8 each; fp32 sums
    bound = (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs() + 1e-30
    assert bool(((got.double() - want).abs() <= bound).all())
    return not bool((ws == 0xa5).all())


@pytest.mark.parametrize("B,m,Hq,Hkv", [(70, 3, 8, 8), (140, 3, 8, 8), (70, 5, 64, 8), (32, 64, 32, 8)])
def test_one_long_context_among_many_short_ones_is_cut(B, m, Hq, Hkv):
    rng = np.random.default_rng(B)
    lens = [int(x) for x in m + rng.integers(0, 200, size=B)]
    lens[B // 2] = 32768
    b = Batch(Hq, Hkv, 64, 16, q_lens=[m] * B, lens=lens, seed=B)
    assert 296 < bounds(b)[0] and bounds(b)[1] == 513
    assert by_list(b)


@pytest.mark.parametrize("D,B,window,extra,far", [(128, 20, 0, 0, True), (128, 19, 0, 0, False), (64, 39, 0, 0, True), (64, 38, 0, 0, False),
                                                  (64, 39, 1450, 2000, True), (128, 20, 1450, 2000, True), (128, 20, 0, 4, False),
                                                  (64, 39, 1514, 2000, False)])
def test_many_blocks_beyond_l2_get_a_cta_each_where_the_contexts_are_bounded(D, B, window, extra, far):
    """Keys and values that the tables' width or the window puts just past what L2 holds or just below, 25 tiles or 26."""
    rng = np.random.default_rng(B)
    q_lens = [int(x) for x in rng.integers(40, 65, size=B)]
    lens = [q + int(x) for q, x in zip(q_lens, rng.integers(0, 300, size=B))]
    lens[0] = 1536
    b = Batch(32, 8, D, 16, q_lens=q_lens, lens=lens, seed=D + B, slopes=window > 0, extra_pages=extra)
    items, tiles, size = bounds(b, window)
    assert 296 < items <= 4 * 296
    assert far == (tiles == 25 and size > 126e6) and tiles in (25, 26)
    assert by_list(b, window) != far


@pytest.mark.parametrize("tokens,one", [(1024, True), (1040, True), (1088, False)])
def test_more_items_than_a_wave_up_to_the_measured_contexts(tokens, one):
    rng = np.random.default_rng(tokens)
    lens = [int(x) for x in rng.integers(3, 300, size=70)]
    lens[5] = tokens
    b = Batch(8, 8, 64, 16, q_lens=[3] * 70, lens=lens, seed=tokens)
    assert bounds(b)[1] == (17 if one else 18)
    assert by_list(b) != one


@pytest.mark.parametrize("m,one", [(416, True), (385, True), (384, False)])
def test_many_blocks_of_each_sequence_get_a_cta_each_at_any_context(m, one):
    """13 blocks of 8 heads are a third of a wave, 12 are not."""
    b = Batch(32, 8, 64, 16, q_lens=[m, 300, m, 290], lens=[m, 900, m + 100, 400], seed=m, extra_pages=1200)
    items, tiles, size = bounds(b)
    assert items == 4 * 8 * (13 if one else 12) > 296 and tiles > 300 and size > 126e6
    assert by_list(b) != one
