"""Chunk attention on the GPU against the definition in 64 bits, sequence by sequence over its whole context."""
import numpy as np
import pytest
import torch

from paper_2505_02351_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


class Batch:
    """q_lens new tokens at the end of contexts of `lens` tokens; slots that hold no token are NaN.  lead / tail: rows of q
    before the first and behind the last sequence; wide: q is a slice of rows that are longer by so many values."""

    def __init__(self, Hq, Hkv, D, bs, q_lens, lens, seed=0, slopes=False, lead=0, tail=0, wide=0, extra_pages=0):
        gen = torch.Generator(DEV).manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.B, self.bs, self.Hkv, self.G = len(lens), bs, Hkv, Hq // Hkv
        pages = [-(-n // bs) for n in lens]
        width = max(1, max(pages)) + extra_pages
        pool = sum(pages) + 5
        perm, cur = rng.permutation(pool), 0
        table, filled = np.full((self.B, width), -1), np.zeros((pool, bs), dtype=bool)
        for s, n in enumerate(lens):
            table[s, :pages[s]] = perm[cur:cur + pages[s]]
            cur += pages[s]
            for i in range(pages[s]):
                filled[table[s, i], :min(bs, n - i * bs)] = True
        T = lead + sum(q_lens) + tail
        randn = lambda *sh: torch.randn(*sh, generator=gen, device=DEV).bfloat16()  # noqa: E731
        self.q = randn(T, Hq * D + wide)[:, :Hq * D].unflatten(1, (Hq, D))
        self.k, self.v = randn(pool, Hkv, bs, D), randn(pool, Hkv, bs, D)
        hole = torch.from_numpy(~filled).to(DEV)[:, None, :, None]
        self.k.masked_fill_(hole, float("nan"))
        self.v.masked_fill_(hole, float("nan"))
        self.table, self.lens = i32(table), i32(lens)
        self.start = i32(lead + np.concatenate([[0], np.cumsum(q_lens)]))
        self.q_lens, self.n, self.lead = [int(x) for x in q_lens], [int(x) for x in lens], lead
        self.slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=DEV, dtype=torch.float32) / Hq) if slopes else None

    def workspace(self, most=None):
        need = binding.chunk_workspace_bytes(self.q.shape[1], self.Hkv, self.q.shape[2], most or max(1, max(self.q_lens)))
        return torch.full((need // 4 + 1,), float("nan"), device=DEV).view(torch.uint8)[:need]

    def run(self, scale, window=0, ws=None, out=None, most=None, stream=None):
        out = torch.full(self.q.shape, 7.0, device=DEV, dtype=torch.bfloat16) if out is None else out
        binding.paged_attention_chunk(out, self.q, self.start, most or max(self.q_lens), self.k, self.v, self.table, self.lens,
                                      self.slopes, scale, self.workspace(most) if ws is None else ws, window=window, stream=stream)
        return out

    def wanted(self, scale, window=0):
        """(out, sum of weight * |v|) in 64 bits; rows of no sequence as run() fills them."""
        out = torch.full(self.q.shape, 7.0, dtype=torch.float64, device=DEV)
        size = torch.zeros_like(out)
        t = self.lead
        for s, (m, n) in enumerate(zip(self.q_lens, self.n)):
            rows = slice(t, t + m)
            t += m
            if m == 0:
                continue
            out[rows] = 0.0
            ids = self.table[s, :-(-n // self.bs)].long()
            k, v = (x[ids].transpose(1, 2).reshape(-1, self.Hkv, x.shape[-1])[:n].double() for x in (self.k, self.v))
            pos = torch.arange(n - m, n, device=DEV)
            key = torch.arange(n, device=DEV)
            back = pos[:, None] - key
            hidden = back < 0 if not window else (back < 0) | (back >= window)
            live = (pos >= 0)[:, None]
            for h in range(self.q.shape[1]):
                z = self.q[rows, h].double() @ k[:, h // self.G].T * scale
                if self.slopes is not None:
                    z -= self.slopes[h].double() * back
                p = torch.softmax(z.masked_fill(hidden, -float("inf")), -1)
                out[rows, h] = torch.where(live, p @ v[:, h // self.G], 0.0)
                size[rows, h] = torch.where(live, p @ v[:, h // self.G].abs(), 0.0)
        return out, size

    def check(self, scale=None, window=0, **kw):
        scale = self.q.shape[2] ** -0.5 if scale is None else scale
        want, size = self.wanted(scale, window)
        # Weights are rounded to bf16 (half a step: 2^-8 of each, in the product and in the denominator), the result once more.
        # Scores: fp32 sums of D products of bf16 values, in log2 units off by at most 2^-24 * D * 1.45 * scale * |q| |k| plus
        # the rounding of scale and bias -- below 2^-13 for these inputs (|scores| below 64, distances below 2^17 times a slope
        # below 1 only where the weight is 0); ex2 and the sums: 2^-20.
        bound = (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs() + 1e-30
        table, got = self.table, None
        # as the tables are, and so wide that the host cannot tell that the contexts are short
        for self.table in (torch.cat([table, torch.full_like(table[:, :1], -1).repeat(1, 700)], 1), table):
            got = self.run(scale, window, **kw)
            torch.cuda.synchronize()
            assert binding.device_status() == 0
            d = (got.double() - want).abs()
            assert bool((d <= bound).all()), (self.table.shape, float((d / bound).max()))
        return got


@pytest.mark.parametrize("Hq,Hkv,D,bs", [(8, 8, 128, 16), (8, 4, 64, 32), (16, 4, 128, 32), (32, 4, 128, 16), (8, 1, 64, 16), (3, 3, 64, 16)])
@pytest.mark.parametrize("slopes", [False, True])
def test_head_layouts_and_ragged_chunks(Hq, Hkv, D, bs, slopes):
    b = Batch(Hq, Hkv, D, bs, q_lens=[1, 5, 0, 64, 130, 16, 300, 1], lens=[1, 700, 33, 64, 131, 2000, 300, 777], slopes=slopes,
              seed=Hq + D)
    b.check()


@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 8, 9, 16, 17, 32, 33, 64, 65, 128, 129, 257])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_numbers_of_new_tokens(m, G):
    """Around the widths of a block (16, 32, 64, 128 rows) and past one."""
    Batch(2 * G, 2, 128, 16, q_lens=[m] * 3, lens=[m, m + 63, m + 1000], seed=m, slopes=G > 1).check()


@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 640, 4097])
@pytest.mark.parametrize("D,bs", [(128, 16), (64, 32)])
def test_lengths_of_the_context(n, D, bs):
    Batch(16, 4, D, bs, q_lens=[1, min(n, 6), min(n, 40)], lens=[n, n, n], seed=n, slopes=True).check()


@pytest.mark.parametrize("window", [1, 2, 15, 63, 64, 65, 128, 200, 1000, 100000])
@pytest.mark.parametrize("m", [1, 7, 130])
def test_windows(window, m):
    for G, D in ((4, 128), (1, 64)):
        b = Batch(2 * G, 2, D, 16, q_lens=[m, m, m, 3], lens=[m, m + 70, 1500, 900], seed=window + m, slopes=G == 4)
        b.check(window=window)


def test_what_lies_before_the_window_is_not_looked_at():
    b = Batch(8, 2, 128, 16, q_lens=[5, 40], lens=[1000, 1203], seed=3)
    want = b.run(0.1, window=100)
    for s in range(2):
        first = b.n[s] - b.q_lens[s] - 99            # the first key that any row sees
        for i in range(first // 64 * 64 // 16):      # whole tiles before it
            b.k[b.table[s, i].long()] = float("nan")
            b.v[b.table[s, i].long()] = float("nan")
    assert torch.equal(b.run(0.1, window=100), want)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 1e-30])
@pytest.mark.parametrize("slopes", [False, True])
def test_scales(scale, slopes):
    Batch(8, 2, 64, 16, q_lens=[3, 100, 1], lens=[500, 140, 65], seed=5, slopes=slopes).check(scale=scale)


def test_rows_before_the_context_and_empty_sequences_are_zero():
    """Padding: sequences with new tokens and no context, or with fewer tokens than they claim to add."""
    b = Batch(8, 2, 128, 16, q_lens=[1, 4, 3, 200, 0, 300, 2], lens=[0, 0, 2, 77, 50, 200, 30], seed=6, slopes=True)
    got = b.check()
    assert not got[:5].any() and not got[8:8 + 123].any()
    Batch(8, 8, 64, 16, q_lens=[1, 1], lens=[0, 0], seed=7).check()


@pytest.mark.parametrize("B,lo,hi", [(30, 500, 640), (37, 100, 110), (36, 30, 900), (9, 60, 64), (37, 1400, 1500)])
def test_batches_of_about_as_many_items_as_workers(B, lo, hi):
    """Items are cut or not, by how many there are and how long the longest is."""
    rng = np.random.default_rng(B)
    Batch(32, 8, 128, 16, q_lens=[int(x) for x in rng.integers(1, 5, size=B)], lens=[int(x) for x in rng.integers(lo, hi + 1, size=B)],
          seed=hi, slopes=True).check()


def test_rows_of_no_sequence_are_left_as_they_are():
    b = Batch(16, 4, 128, 16, q_lens=[5, 33, 1], lens=[50, 600, 70], lead=3, tail=9, seed=8)
    got = b.check()
    assert bool((got[:3] == 7).all()) and bool((got[-9:] == 7).all())


@pytest.mark.parametrize("wide", [8, 1024, 2 * 4 * 128])
def test_q_as_a_slice_of_wider_rows(wide):
    b = Batch(16, 4, 128, 16, q_lens=[5, 33, 1], lens=[50, 600, 70], wide=wide, seed=9)
    assert not b.q.is_contiguous()
    b.check()


def test_out_aligned_to_16_bytes_and_no_more():
    for n in (90, 9000):
        b = Batch(16, 4, 128, 16, q_lens=[5, 40, 1], lens=[n, n, 70], seed=n)
        want = b.run(0.1)
        room = torch.full((b.q.numel() + 16,), 7.0, device=DEV, dtype=torch.bfloat16)
        out = room[8:-8].view(b.q.shape)
        assert out.data_ptr() % 32 == 16
        assert torch.equal(b.run(0.1, out=out), want) and bool((room[:8] == 7).all()) and bool((room[-8:] == 7).all())


def test_one_token_with_any_stride():
    b = Batch(16, 4, 128, 16, q_lens=[1], lens=[300], wide=7, seed=10)       # the stride of a single token says nothing
    b.check()


@pytest.mark.parametrize("B,Hq,Hkv,m,n", [(1, 8, 1, 1, 20000), (1, 8, 8, 4, 70000), (2, 32, 4, 8, 30011), (300, 8, 2, 2, 130), (700, 8, 8, 1, 40),
                                         (1, 16, 4, 600, 9000), (64, 16, 8, 3, 1000)])
def test_cuts(B, Hq, Hkv, m, n):
    """One long context over all workers, more sequences than threads, blocks that share their tiles."""
    rng = np.random.default_rng(B + n)
    lens = rng.integers(max(m, n // 2), n + 1, size=B)
    q = rng.integers(1, m + 1, size=B)
    Batch(Hq, Hkv, 128, 16, q_lens=[int(x) for x in q], lens=[int(x) for x in lens], seed=B, slopes=B < 3).check()


@pytest.mark.parametrize("Hq,Hkv,D,bs", [(8, 1, 128, 16), (32, 4, 128, 32), (16, 8, 64, 16), (4, 4, 64, 32), (64, 8, 128, 16)])
@pytest.mark.parametrize("m", [1, 2, 4, 9, 16, 33])
@pytest.mark.parametrize("window", [0, 200])
def test_few_items_of_long_contexts(Hq, Hkv, D, bs, m, window):
    """Items whose tiles a cluster shares: some with fewer tiles than CTAs, padding, none, rows that see nothing of a share."""
    lens = [1500 + m, 700, 65, 64, 1, 0, 130 + m, 5]
    q = [m, m, min(m, 65), 1, 1, 0, m, m]
    b = Batch(Hq, Hkv, D, bs, q_lens=q, lens=lens, seed=Hq + m, slopes=m % 2 == 0, lead=2, tail=3)
    got = b.check(window=window)
    scale = D ** -0.5
    for _ in range(2):
        assert torch.equal(b.run(scale, window).view(torch.int16), got.view(torch.int16))


@pytest.mark.parametrize("D,bs,window", [(128, 16, 0), (64, 32, 150)])
def test_many_blocks_whose_tables_say_that_l2_does_not_hold_them(D, bs, window):
    rng = np.random.default_rng(D)
    q = rng.integers(130, 161, size=9)
    lens = q + rng.integers(0, 400, size=9)
    Batch(32, 8, D, bs, q_lens=[int(x) for x in q], lens=[int(x) for x in lens], seed=D, slopes=D == 64, extra_pages=300).check(window=window)


def test_a_mixed_batch():
    rng = np.random.default_rng(0)
    q = np.concatenate([np.ones(40, dtype=int), rng.integers(2, 9, size=10), [257, 512, 100]])
    lens = np.maximum(q, np.rint(np.exp(rng.uniform(2, 8, size=53))).astype(int))
    order = rng.permutation(53)
    Batch(32, 4, 128, 32, q_lens=[int(x) for x in q[order]], lens=[int(x) for x in lens[order]], seed=11, slopes=True, extra_pages=9).check()


@pytest.mark.parametrize("B,window", [(257, 0), (700, 90), (1500, 0)])
def test_batches_of_more_sequences_than_threads(B, window):
    """Each thread of the list's first pass has several sequences, some without new tokens, without a context, or padding."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 200, size=B)
    q = np.where(rng.random(B) < 0.3, 0, rng.integers(1, 6, size=B))
    q[B // 2], lens[B // 2] = 150, 180
    Batch(4, 2, 64, 16, q_lens=[int(x) for x in q], lens=[int(x) for x in lens], seed=B, slopes=window > 0, lead=3, tail=5).check(window=window)


def test_every_key_counts_once_wherever_the_list_is_cut():
    """Equal scores, values that name their token: each row is the mean of the numbers it sees, so a key too many or too few
    shows.  Numbers below 256 are whole in bf16, and so is what the tensor core sums."""
    for m, n, window in ((6, 5000, 0), (40, 3333, 0), (300, 2100, 0), (5, 4000, 1000), (150, 3000, 333)):
        b = Batch(8, 2, 64, 16, q_lens=[m, m], lens=[n, n - 7], seed=n)
        b.q.zero_()
        for s in range(2):
            tok = torch.arange(b.n[s], device=DEV)
            # dim d < 32: 1 where the token's number modulo 32 is d; the others: which of 32 parts of the context it lies in
            one = torch.zeros(b.n[s], 64, device=DEV)
            one[tok, tok % 32] = 1
            one[tok, 32 + tok * 32 // b.n[s]] = 1
            for i in range(-(-b.n[s] // 16)):
                rows = one[16 * i:16 * i + 16]
                b.v[b.table[s, i].long(), :, :len(rows)] = rows.bfloat16()
        got = b.run(1.0, window=window).double()
        want, _ = b.wanted(1.0, window)
        # weights are 1 and so exact; one division and one rounding to bf16
        assert bool(((got - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs()).all()), (m, n, window)


def test_the_one_key_that_matters_in_every_tile():
    """A key whose score is far above the others', at each tile's ends in turn: the running maximum moves late or early."""
    n, m = 1000, 20
    for at in (0, 1, 63, 64, 500, 511, 979, 980, 990, 999):
        b = Batch(8, 2, 128, 16, q_lens=[m], lens=[n], seed=at)
        b.q[...] = b.q[:1, :1]
        b.k[b.table[0, at // 16].long(), :, at % 16] = 4 * b.q[0, 0]
        b.check(scale=0.2)


def test_unseen_scores_of_any_size_change_nothing():
    """Keys that later tokens alone see, with infinite and NaN entries: earlier rows are as without them."""
    b = Batch(8, 2, 128, 16, q_lens=[9], lens=[300], seed=12)
    want = b.run(0.1)
    for at, x in ((299, float("inf")), (298, float("nan")), (297, -float("inf"))):
        b.k[b.table[0, at // 16].long(), :, at % 16] = x
        got = b.run(0.1)
        assert torch.equal(got[:at - 291], want[:at - 291]), at
        assert not torch.isfinite(got[8].float()).all()


def test_nan_scores_reach_their_row_alone():
    b = Batch(8, 4, 128, 16, q_lens=[7, 3], lens=[700, 40], seed=13)
    want = b.run(0.1)
    b.q[4, 3] = float("nan")
    got = b.run(0.1)
    assert bool(got[4, 3].isnan().all())
    got[4, 3] = want[4, 3]
    assert torch.equal(got, want)


def test_the_lowest_value_and_infinity_as_scores():
    """Every key's score -inf: no weights, NaN as the formula has it; some: they weigh nothing."""
    b = Batch(8, 8, 64, 16, q_lens=[2], lens=[200], seed=14)
    b.q.abs_()
    b.k[b.table[0, :10].long()] = -float("inf")
    got = b.run(0.1)
    want, size = b.wanted(0.1)
    assert bool(((got.double() - want).abs() <= (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs()).all())
    b.k[b.table[0].long()] = -float("inf")
    assert bool(b.run(0.1).isnan().all())
    b.k[b.table[0].long()] = torch.finfo(torch.bfloat16).min
    b.k[b.table[0, 3].long(), :, 5] = 1.0
    b.check(scale=0.001)


def test_behind_32_bit_offsets():
    """Pages past 2^32 bytes of their pool."""
    b = Batch(8, 8, 128, 16, q_lens=[3, 20], lens=[500, 140], seed=15)
    pool = 140000                                    # of 32 KB: 4.6 GB each
    k, v = (torch.empty(pool, 8, 16, 128, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    small = b.k.shape[0]
    k[-small:], v[-small:] = b.k, b.v
    want = b.run(0.1)
    b.k, b.v = k, v
    b.table += pool - small
    got = b.run(0.1)
    assert torch.equal(got, want)


def test_the_workspace_of_the_longest_chunk_serves_all():
    b = Batch(16, 4, 128, 16, q_lens=[300, 1], lens=[900, 5000], seed=16)
    ws = b.workspace()
    b.check(ws=ws)
    Batch(16, 4, 128, 16, q_lens=[2, 1], lens=[9000, 5000], seed=17).check(ws=ws)
    b.check(ws=ws, most=1000)


def test_a_longer_chunk_than_promised_stays_inside():
    """max_q_len is the caller's promise; tokens past it are not computed, and nothing else is touched."""
    b = Batch(16, 4, 128, 16, q_lens=[9, 2], lens=[900, 5000], seed=18)
    need = binding.chunk_workspace_bytes(16, 4, 128, 4)
    big = torch.full((need + 4096,), 0x5a, device=DEV, dtype=torch.uint8)
    got = b.run(0.1, ws=big[:need], most=4)
    torch.cuda.synchronize()
    assert bool((big[need:] == 0x5a).all()) and bool((got[4:9] == 7).all())
    # what is computed is as promised (not the same bits: another number of blocks cuts the list elsewhere)
    want, size = b.wanted(0.1)
    bound = (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs() + 1e-30
    d = (got.double() - want).abs()
    assert bool((d[:4] <= bound[:4]).all()) and bool((d[9:] <= bound[9:]).all())


def test_captured_with_a_workspace_two_graphs_share():
    a = Batch(16, 4, 128, 16, q_lens=[5, 1, 40], lens=[3000, 900, 200], seed=19, slopes=True)
    b = Batch(16, 4, 128, 16, q_lens=[1, 8], lens=[8000, 70], seed=20)
    ws = a.workspace(64)
    want = [x.run(0.1, ws=ws, most=64).clone() for x in (a, b)]         # (the call that is captured: how contexts are cut goes by its bounds)
    outs = [torch.zeros_like(w) for w in want]
    graphs = []
    for x, o in zip((a, b), outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run(0.1, ws=ws, out=o, most=64)
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            o.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    # other lengths in the same graph
    a.lens.copy_(i32([2500, 901, 190]))
    a.n = [2500, 901, 190]
    graphs[0].replay()
    torch.cuda.synchronize()
    # (bits: the second sequence's last token is a slot that holds NaN, and so is its row)
    assert torch.equal(outs[0].view(torch.int16), a.run(0.1, ws=ws).view(torch.int16))
    assert bool(outs[0][5].isnan().all()) and not outs[0][:5].isnan().any() and not outs[0][6:].isnan().any()


def test_on_two_streams_at_once():
    bs = [Batch(16, 4, 128, 16, q_lens=[5, 1, 40], lens=[9000, 900, 200], seed=21 + i) for i in range(2)]
    want = [b.run(0.1).clone() for b in bs]
    ws, outs = [b.workspace() for b in bs], [torch.zeros_like(w) for w in want]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, w, o, st in zip(bs, ws, outs, streams):
            b.run(0.1, ws=w, out=o, stream=st)
    torch.cuda.synchronize()
    assert binding.device_status() == 0
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_the_same_bits_in_every_run():
    b = Batch(32, 4, 128, 16, q_lens=[8, 3, 1, 130], lens=[20000, 3000, 5000, 700], seed=23, slopes=True)
    want = b.run(0.1).clone()
    for _ in range(5):
        assert torch.equal(b.run(0.1), want)


def test_refusals_of_the_binding():
    b = Batch(16, 4, 128, 16, q_lens=[5, 1], lens=[90, 20], seed=24)
    out, ws = torch.empty_like(b.q), b.workspace()
    good = dict(out=out, q=b.q, q_start_loc=b.start, max_q_len=5, k_cache=b.k, v_cache=b.v, block_tables=b.table, context_lens=b.lens,
                alibi_slopes=None, scale=0.1, workspace=ws)
    for bad in (dict(q=b.q.float()), dict(q=b.q.transpose(0, 1).contiguous().transpose(0, 1)), dict(q_start_loc=b.start[:-1]),
                dict(q_start_loc=b.start.long()), dict(context_lens=b.lens.cpu()), dict(block_tables=b.table.long()),
                dict(alibi_slopes=torch.zeros(15, device=DEV)), dict(out=torch.empty(6, 16, 256, device=DEV, dtype=torch.bfloat16)[..., :128])):
        with pytest.raises(ValueError):
            binding.paged_attention_chunk(**dict(good, **bad))
    for code, bad in ((-2, dict(window=-1)), (-2, dict(workspace=ws[:-1024]))):
        with pytest.raises(binding.OptGqaError) as e:
            binding.paged_attention_chunk(**dict(good, **bad))
        assert e.value.code == code


class Elsewhere:
    """A workspace on another device, as the binding sees it."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.t.get_device() + 1


def test_workspaces_of_another_device_or_with_gaps_are_refused():
    b = Batch(8, 2, 64, 16, [2], [30])
    for ws in (Elsewhere(b.workspace()), torch.empty(1 << 24, device=DEV)[::2], torch.empty(1 << 24)):
        with pytest.raises(ValueError):
            b.run(0.125, ws=ws)
    b.run(0.125)
