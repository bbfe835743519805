"""Shared-prefix decode on the GPU with values that name their page or token, so that any one that is left out, taken twice
or taken from elsewhere shows in the result; lengths past the table; the routes of small batches."""
import numpy as np
import pytest
import torch

from paper_2505_02351_b200 import binding
from tests.test_gpu_decode_shared import DEV, Batch

pytestmark = pytest.mark.gpu


def named(b, unit):
    """Values of 1 in one dim and 0 in the others: the dim says which `unit` tokens of the pool it is, and which KV head."""
    pool, Hkv, bs, D = b.v.shape
    at = torch.arange(pool * bs, device=DEV).view(pool, 1, bs) // unit + 7 * torch.arange(Hkv, device=DEV)[:, None]
    b.v = torch.where(b.v.isnan(), b.v, torch.nn.functional.one_hot(at % D, D).to(b.v.dtype))


def grown(first, step, count):
    return [first + step * i for i in range(count)]


SHAPES = {
    "one long prefix": (dict(Hq=8, Hkv=1, D=128, bs=16, sizes=[9], prefix=[40000], lens=grown(40000, 37, 9)), 16),
    "two prefixes over every worker": (dict(Hq=8, Hkv=2, D=64, bs=32, sizes=[5, 2], prefix=[20011, 4100],
                                            lens=[20100, 20200, 20011, 20012, 25000, 4300, 4100]), 32),
    "batch behind one prompt": (dict(Hq=32, Hkv=8, D=128, bs=16, sizes=[32], prefix=[1500], lens=grown(1564, 15, 32)), 1),
    "ragged groups": (dict(Hq=64, Hkv=8, D=128, bs=32, sizes=[1, 17, 3, 12, 7], prefix=[2000, 300, 64, 1100, 4000], loose=3,
                           lens=[2100] + grown(290, 9, 17) + [64, 65, 200] + grown(1100, 61, 12) + grown(4001, 5, 7) + [500, 0, 1]), 1),
    "a head per KV head": (dict(Hq=8, Hkv=8, D=64, bs=16, sizes=[3, 140, 5], prefix=[700, 900, 64], lens=grown(699, 1, 3) + grown(900, 4, 140) +
                                grown(60, 30, 5)), 1),
    "two heads per KV head": (dict(Hq=16, Hkv=8, D=64, bs=32, sizes=[70, 2], prefix=[640, 1000], lens=grown(641, 13, 70) + [1000, 900]), 1),
    "own contexts": (dict(Hq=16, Hkv=4, D=128, bs=16, sizes=[2], prefix=[64], lens=[64, 100] + grown(1, 25, 60), loose=60), 1),
}


@pytest.mark.parametrize("name", SHAPES)
def test_every_page_and_token_counts_once(name):
    """Equal scores: every weight is 1 and an output is the share of a dim's name among the keys.  The sums are whole numbers;
    reciprocal, product and merge are off by a few 2^-22, the store by half a step.  At most 50 units share a name, so that one
    too many or too few is 2 % of one dim at least, five times the bound (the CPU's test of the same names shows it)."""
    shape, unit = SHAPES[name]
    b = Batch(**shape)
    named(b, unit)
    b.q.zero_()
    want, _ = b.wanted(1.0)
    assert float((want.amax((1, 2)) * b.lens).max()) <= 50 * unit
    for ws in (None, b.workspace(512, small=True)):
        got = b.run(1.0, ws=ws)
        d = (got.double() - want).abs()
        assert bool((d <= (2.0 ** -8 + 2.0 ** -16) * want).all()), float((d / want.clamp_min(1e-9)).max())
    assert binding.device_status() == 0


@pytest.mark.parametrize("slope", [None, 2.0 ** -14])
@pytest.mark.parametrize("Hq,Hkv,D,bs", [(32, 4, 128, 16), (8, 4, 128, 32), (8, 1, 64, 16)])
def test_named_pages_under_scores_and_small_slopes(Hq, Hkv, D, bs, slope):
    """Ordinary scores, slopes so small that no key is far: a dim holds a few pages, each of them a multiple of the bound."""
    rng = np.random.default_rng(Hq)
    n = 60 * bs * D // 16
    b = Batch(Hq, Hkv, D, bs, sizes=[12, 2], prefix=[n, n // 3], lens=[n + int(x) for x in rng.integers(0, 300, size=12)] + [n // 3 + 1, n // 2])
    named(b, bs)
    if slope is not None:
        b.slopes = torch.full((Hq,), slope, device=DEV) * torch.arange(1, Hq + 1, device=DEV) / Hq
    b.check()


@pytest.mark.parametrize("own", [False, True])
def test_the_one_key_that_matters_wherever_it_lies(own):
    """A key whose score towers over the others', in each tile and at its first and last token in turn."""
    b = Batch(8, 2, 64, 16, sizes=[3], prefix=[1000], lens=[1001, 1030, 1900] if own else [1001, 1002, 1030])
    s = 2 if own else 0
    b.q[..., 0] = 8
    k0, v0 = b.k.clone(), b.v.clone()
    k0[..., 0] = torch.where(k0[..., 0].isnan(), k0[..., 0], 0)
    for at in range(960 if own else 0, 1900 if own else 960, 64):
        for token in (at, min(at + 63, b.n[s] - 1)):
            page = int(b.table[s, token // 16])
            b.k, b.v = k0.clone(), v0.clone()
            b.k[page, :, token % 16, 0] = 64            # a score of 64 before the others' few
            got = b.run(64 ** -0.5)
            sees = [2] if own else [0, 1, 2]
            # the others weigh e^-50 of it together, and its own weight divides out: the value itself, bit for bit
            assert torch.equal(got[sees].view(len(sees), 2, 4, 64), v0[page, :, token % 16][None, :, None].expand(len(sees), 2, 4, 64)), token


def test_lengths_past_the_table_stay_inside_the_buffers_and_disturb_nobody():
    """A length (and a prefix) past the page table, of a group's leader, of another of its sequences, of one in no group: that row
    is wrong, the others' are the definition's and the next call is right.  (Entries past the table are taken as page 0.)"""
    b = Batch(16, 4, 64, 16, sizes=[3, 2], prefix=[256, 128], lens=[300, 310, 320, 200, 210, 90], loose=1, slopes=True)
    b.table.clamp_(min=0)
    first = b.check()
    want, size = b.wanted(64 ** -0.5)
    lens, prefix = b.lens.clone(), b.prefix.clone()
    bound = (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs() + 1e-30
    for s in range(6):
        for told in (int(prefix[s]), 16 * b.table.shape[1] + 200):
            b.lens[s], b.prefix[s] = 16 * b.table.shape[1] + 500, told
            got = b.run(64 ** -0.5)
            torch.cuda.synchronize()
            assert binding.device_status() == 0
            others = [x for x in range(6) if x != s]
            assert bool(((got.double() - want).abs() <= bound)[others].all()), (s, told)
            b.lens.copy_(lens)
            b.prefix.copy_(prefix)
    assert torch.equal(b.check(), first)


@pytest.mark.parametrize("Hq,Hkv,D,bs", [(8, 8, 64, 32), (8, 4, 64, 16), (16, 4, 128, 32), (8, 1, 64, 32), (8, 1, 128, 16)])
@pytest.mark.parametrize("slopes", [False, True])
def test_small_batches_of_every_head_layout(Hq, Hkv, D, bs, slopes):
    for prefix, lens in ((500, [501, 560, 512, 0, 777]), (0, [1, 2, 15, 16, 17]), (1500, [1501, 1600, 1536, 2000, 30])):
        b = Batch(Hq, Hkv, D, bs, sizes=[4], prefix=[prefix], lens=lens, loose=1, slopes=slopes)
        b.check(P=64, ws=b.workspace(64, small=True))


@pytest.mark.parametrize("lens", [[201, 260, 330], [1201, 1260, 1330]])
def test_small_batches_with_pages_past_32_bit_offsets(lens):
    """Both routes of small batches with the pages at the end of a pool of 2^33 bytes."""
    b = Batch(8, 2, 128, 16, sizes=[3], prefix=[200], lens=lens, slopes=True)
    tight = b.workspace(64, small=True)
    want = b.check(P=64, ws=tight)
    pool, used = 2 ** 33 // (2 * 16 * 128 * 2), b.k.shape[0]
    for name in ("k", "v"):
        big = torch.empty(pool, 2, 16, 128, dtype=torch.bfloat16, device=DEV)
        big[pool - used:] = getattr(b, name)
        setattr(b, name, big)
    b.table.copy_(torch.where(b.table >= 0, b.table + (pool - used), b.table))
    assert torch.equal(b.run(128 ** -0.5, P=64, ws=tight), want)


@pytest.mark.parametrize("small", [False, True])
def test_steps_that_grow_over_page_and_tile_ends(small):
    """Rotate, append and attend, one token a step, over the ends of pages and of tiles of 64, without a synchronisation."""
    ends = [(62, 64), (63, 0), (126, 64), (700, 640), (703, 640), (765, 640)]       # length at first, prefix
    b = Batch(32, 8, 128, 16, sizes=[1, 1, 1, 3], prefix=[p for _, p in ends[:4]], lens=[n + 6 for n, _ in ends], seed=3)
    freq = binding.rotary_table(binding.rotary_frequencies(128), DEV)
    ws, out, gen = b.workspace(512, small=small), torch.empty_like(b.q), torch.Generator(DEV).manual_seed(9)
    for step in range(6):
        b.n = [n + step for n, _ in ends]
        b.lens.copy_(torch.tensor(b.n, dtype=torch.int32))
        x = torch.randn(6, (32 + 16) * 128, generator=gen, device=DEV).bfloat16()
        q, k, v = (y.unflatten(1, (-1, 128)) for y in x.split([4096, 1024, 1024], 1))
        pos = b.lens - 1
        page = b.table.gather(1, (pos // 16).long()[:, None])[:, 0].long()
        b.q = torch.empty_like(b.q)
        binding.rotary_append(b.q, q, k, v, b.k, b.v, page * 16 + pos % 16, pos, freq, 0)
        b.run(128 ** -0.5, ws=ws, out=out)
        want, size = b.wanted(128 ** -0.5)
        assert bool(((out.double() - want).abs() <= (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs()).all()), step
        assert torch.equal(b.v[page, :, pos % 16], v)
    assert binding.device_status() == 0
