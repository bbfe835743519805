"""Shared-prefix decode on the GPU against the definition in 64 bits, sequence by sequence over its whole context."""
import numpy as np
import pytest
import torch

from paper_2505_02351_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Batch:
    """sizes: sequences per group (the last `loose` sequences belong to none); prefix: tokens a group's tables share;
    lens: context lengths (0: an empty row).  Whole pages below min(prefix, len) are shared, everything else is a
    sequence's own; slots that hold no token are NaN."""

    def __init__(self, Hq, Hkv, D, bs, sizes, prefix, lens, loose=0, seed=0, slopes=False, told=None, before=0):
        gen = torch.Generator(DEV).manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.B, self.bs, self.Hkv, self.G = len(lens), bs, Hkv, Hq // Hkv
        assert before + sum(sizes) + loose == self.B
        start = before + np.concatenate([[0], np.cumsum(sizes)])
        shared = np.zeros(self.B, dtype=np.int64)
        for g, p in enumerate(prefix):
            shared[start[g]:start[g + 1]] = p
        pages = -(-np.asarray(lens) // bs)
        width = max(1, int(pages.max()))
        pool = int(pages.sum()) + 8 + sum(-(-p // bs) for p in prefix)
        perm = rng.permutation(pool)
        table = np.full((self.B, width), -1, dtype=np.int32)
        cur = 0
        for g, p in enumerate(prefix):
            common = perm[cur:cur + p // bs]
            cur += p // bs
            for s in range(start[g], start[g + 1]):
                k = min(p // bs, pages[s])
                table[s, :k] = common[:k]
        filled = np.zeros((pool, bs), dtype=bool)
        for s in range(self.B):
            k = int(min(shared[s] // bs, pages[s]))
            own = perm[cur:cur + pages[s] - k]
            table[s, k:pages[s]] = own
            cur += len(own)
            for i in range(int(pages[s])):
                filled[table[s, i], :min(bs, lens[s] - i * bs)] = True
        assert cur <= pool
        randn = lambda *sh: torch.randn(*sh, generator=gen, device=DEV).bfloat16()  # noqa: E731
        self.q, self.k, self.v = randn(self.B, Hq, D), randn(pool, Hkv, bs, D), randn(pool, Hkv, bs, D)
        hole = torch.from_numpy(~filled).to(DEV)[:, None, :, None]
        self.k.masked_fill_(hole, float("nan"))
        self.v.masked_fill_(hole, float("nan"))
        i32 = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).to(DEV)  # noqa: E731
        self.table, self.lens, self.start = i32(table), i32(lens), i32(start)
        self.n = [int(x) for x in lens]
        self.prefix = i32(shared if told is None else told)
        self.slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=DEV, dtype=torch.float32) / Hq) if slopes else None

    def workspace(self, P, small=False):
        """small: the bound on the contexts is tight, so that small batches take the route of small batches; otherwise it is
        loose enough for the group pass to run."""
        parts = max(1, -(-max(self.n) // P))
        if not small:
            parts = max(parts, int(33e6 / (self.B * P * self.Hkv * self.q.shape[2] * 4)) + 1)
        need = binding.shared_workspace_bytes(self.B, self.q.shape[1], self.Hkv, self.q.shape[2], self.start.numel() - 1, parts)
        return torch.full((need // 4 + 1,), float("nan"), device=DEV).view(torch.uint8)[:need], parts

    def run(self, scale, P=512, ws=None, out=None, stream=None):
        ws, parts = ws if ws is not None else self.workspace(P)
        out = torch.full_like(self.q, float("nan")) if out is None else out
        binding.paged_attention_decode_shared(out, self.q, self.k, self.v, self.table, self.lens, self.start, self.prefix,
                                              self.slopes, scale, P, ws, parts, stream=stream)
        return out

    def wanted(self, scale):
        """(out, sum of weight * |v|) in 64 bits."""
        B, Hq, D = self.q.shape
        out, size = (torch.zeros(B, Hq, D, dtype=torch.float64, device=DEV) for _ in range(2))
        for s in range(B):
            n = self.n[s]
            if n == 0:
                continue
            ids = self.table[s, :-(-n // self.bs)].long()
            k, v = (x[ids].transpose(1, 2).reshape(-1, self.Hkv, D)[:n].double() for x in (self.k, self.v))
            z = torch.einsum("hgd,jhd->hgj", self.q[s].double().view(self.Hkv, self.G, D), k) * scale
            if self.slopes is not None:
                z -= self.slopes.double().view(self.Hkv, self.G, 1) * torch.arange(n - 1, -1, -1, device=DEV)
            p = torch.softmax(z, -1)
            out[s] = torch.einsum("hgj,jhd->hgd", p, v).reshape(Hq, D)
            size[s] = torch.einsum("hgj,jhd->hgd", p, v.abs()).reshape(Hq, D)
        return out, size

    def check(self, scale=None, P=512, **kw):
        scale = self.q.shape[2] ** -0.5 if scale is None else scale
        got = self.run(scale, P, **kw)
        torch.cuda.synchronize()
        assert binding.device_status() == 0
        want, size = self.wanted(scale)
        # Weights are rounded to bf16 (half a step: 2^-8 of each, in the product and in the own pass's denominator), the
        # result once more.  Scores: fp32 sums of D products of bf16 values, in log2 units off by at most
        # 2^-24 * D * 1.45 * scale * |q| |k| plus the rounding of scale and bias -- below 2^-13 for these inputs (|scores|
        # below 64, distances below 2^17 times a slope below 1 only where the weight is 0); ex2 and the sums: 2^-20.
        bound = (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs() + 1e-30
        d = (got.double() - want).abs()
        worst = float((d / bound.clamp_min(1e-30)).max())
        assert bool((d <= bound).all()), worst
        return got


@pytest.mark.parametrize("Hq,Hkv,D,bs", [(8, 8, 128, 16), (8, 4, 64, 32), (16, 4, 128, 32), (32, 4, 128, 16), (8, 1, 64, 16), (3, 3, 64, 16)])
@pytest.mark.parametrize("slopes", [False, True])
def test_head_layouts_and_ragged_groups(Hq, Hkv, D, bs, slopes):
    b = Batch(Hq, Hkv, D, bs, sizes=[3, 1, 5], prefix=[200, 64, 1000],
              lens=[201, 263, 330, 64, 1000, 1001, 1100, 1064, 2047, 77], loose=1, slopes=slopes, seed=Hq + D)
    b.check()


@pytest.mark.parametrize("prefix", [0, 1, 63, 64, 65, 127, 128, 500, 2048])
@pytest.mark.parametrize("own", [0, 1, 15, 16, 17, 300])
def test_lengths_of_the_prefix_and_behind_it(prefix, own):
    n = prefix + own
    b = Batch(16, 4, 128, 16, sizes=[6], prefix=[prefix], lens=[n] * 6, seed=n)
    b.check(P=64)


@pytest.mark.parametrize("slopes", [False, True])
def test_small_batches_and_tight_bounds(slopes):
    """The same batches with a tight bound on the contexts: whichever route a call takes, the result is the definition's."""
    for sizes, prefix, lens in (([4], [500], [501, 560, 512, 777]), ([2, 2], [64, 700], [0, 70, 701, 700]), ([3], [0], [1, 2, 0]),
                                ([4], [1000], [1001, 1100, 1500, 0]), ([40], [600], [601 + 3 * i for i in range(40)])):
        b = Batch(32, 8, 128, 16, sizes=sizes, prefix=prefix, lens=lens, slopes=slopes)
        b.check(P=64, ws=b.workspace(64, small=True))


def test_rows_without_tokens_give_zero_rows_and_disturb_nobody():
    b = Batch(32, 8, 128, 16, sizes=[4, 2, 2], prefix=[320, 256, 128], lens=[0, 400, 0, 321, 0, 0, 129, 0, 0], loose=1)
    got = b.check()
    for s in (0, 2, 4, 5, 7, 8):
        assert bool((got[s] == 0).all())
    empty = Batch(8, 4, 64, 16, sizes=[2], prefix=[0], lens=[0, 0])
    assert bool((empty.check() == 0).all())


def test_sequences_that_share_less_or_end_inside_the_prefix():
    """prefix_lens that differ inside a group, exceed the context, or are zero; the leader is not the first sequence."""
    lens = [100, 700, 512, 513, 60, 700, 30]
    told = [100, 256, 640, 512, 512, 0, 9999]
    b = Batch(32, 4, 128, 16, sizes=[6], prefix=[512], lens=lens, loose=1, told=told, slopes=True)
    b.check(P=128)


def test_what_a_row_does_not_see_never_reaches_it():
    """Two sequences share 64 tokens, two of them 128 more whose keys and values are not finite: the two that do not see
    those keep their results bit for bit."""
    b = Batch(8, 1, 128, 16, sizes=[4], prefix=[192], lens=[250, 230, 220, 210], told=[192, 64, 192, 64], seed=5)
    # sequences 1 and 3 have pages of their own past token 64
    pages = b.table.clone()
    spare = torch.arange(b.k.shape[0], device=DEV, dtype=torch.int32)
    spare = spare[~torch.isin(spare, pages.flatten())]
    extra = torch.randn(16, 1, 16, 128, generator=torch.Generator(DEV).manual_seed(1), device=DEV).bfloat16()
    base = b.k.shape[0]
    b.k, b.v = torch.cat([b.k, extra]), torch.cat([b.v, extra.flip(0)])
    b.table[1, 4:12] = torch.arange(base, base + 8, device=DEV, dtype=torch.int32)
    b.table[3, 4:12] = torch.arange(base + 8, base + 16, device=DEV, dtype=torch.int32)
    before = b.check()
    shared = b.table[0, 4:12].long()
    for value in (float("nan"), float("inf"), -float("inf")):
        b.k[shared], b.v[shared] = value, value
        after = b.run(128 ** -0.5)
        assert torch.equal(after[[1, 3]], before[[1, 3]])
        assert bool(torch.isnan(after[[0, 2]]).all())


@pytest.mark.parametrize("B,G,D", [(16, 8, 128), (17, 8, 128), (40, 8, 64), (200, 1, 128), (150, 4, 64)])
def test_several_row_blocks(B, G, D):
    rng = np.random.default_rng(B)
    lens = [int(x) for x in 900 + rng.integers(0, 200, size=B)]
    b = Batch(2 * G, 2, D, 16, sizes=[B], prefix=[900], lens=lens, slopes=True, seed=B)
    b.check()


def test_more_groups_than_a_warp_and_empty_ones():
    rng = np.random.default_rng(7)
    sizes = [int(x) for x in rng.integers(0, 4, size=75)]
    prefix = [int(x) for x in rng.integers(0, 700, size=75)]
    lens = []
    for k, p in zip(sizes, prefix):
        lens += [p + int(x) for x in rng.integers(0, 90, size=k)]
    b = Batch(16, 4, 64, 32, sizes=sizes, prefix=prefix, lens=[33, 0] + lens + [90, 0, 8], loose=3, before=2)
    b.check()


def test_the_most_groups():
    b = Batch(2, 2, 64, 16, sizes=[1] * 512, prefix=[64] * 512, lens=[70] * 512 + [40], loose=1)
    b.check()


def test_one_long_prefix_over_every_worker():
    b = Batch(8, 1, 128, 16, sizes=[9], prefix=[40000], lens=[40000 + 37 * i for i in range(9)], slopes=True)
    b.check()
    b = Batch(8, 2, 64, 32, sizes=[5, 2], prefix=[20011, 4100], lens=[20100, 20200, 20011, 20012, 25000, 4300, 4100])
    b.check()


@pytest.mark.parametrize("scale", [0.0, -0.09, 0.3, 1e-20])
@pytest.mark.parametrize("slopes", [False, True])
def test_scales_of_either_sign_and_zero(scale, slopes):
    b = Batch(16, 4, 128, 16, sizes=[3], prefix=[300], lens=[301, 400, 500], slopes=slopes)
    b.check(scale=scale)


def test_steep_slopes_and_slopes_that_fall_towards_the_query():
    b = Batch(16, 4, 64, 16, sizes=[3], prefix=[3000], lens=[3001, 3100, 3064])
    for s in (3.0, -0.004):
        b.slopes = torch.full((16,), s, device=DEV)
        b.check()


def test_same_bits_every_time_on_streams_and_in_graphs():
    """Two batches at a time on two streams with a workspace each; one captured and replayed after its inputs changed."""
    b = Batch(32, 4, 128, 16, sizes=[7], prefix=[1500], lens=[1500 + 11 * i for i in range(7)], slopes=True, seed=1)
    c = Batch(32, 8, 64, 32, sizes=[4, 3], prefix=[900, 2000], lens=[901, 950, 1000, 1200, 2001, 2100, 2500], seed=2)
    first = [x.check(x.q.shape[2] ** -0.5) for x in (b, c)]
    spaces = [x.workspace(512) for x in (b, c)]
    outs = [torch.full_like(x.q, float("nan")) for x in (b, c)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, ws, out, st in zip((b, c), spaces, outs, streams):
            x.run(x.q.shape[2] ** -0.5, ws=ws, out=out, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], first[0]) and torch.equal(outs[1], first[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(128 ** -0.5, ws=spaces[0], out=outs[0])
    b.q.copy_(b.q.flip(0))
    b.lens.copy_(torch.tensor([1500 + 3 * i for i in range(7)], dtype=torch.int32, device=DEV))
    b.n = [1500 + 3 * i for i in range(7)]
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], b.check()) and not torch.equal(outs[0], first[0])


def test_index_data_that_breaks_the_promises_gives_wrong_rows_and_no_access_outside():
    """group_start that does not increase or leaves the batch, lengths past the table: the call comes back, and the next
    one is right.  (Every index is held inside by the kernels' own bounds.)"""
    b = Batch(16, 4, 64, 16, sizes=[3, 3], prefix=[256, 128], lens=[300, 310, 320, 200, 210, 220])
    want = b.check()
    good = b.start.clone()
    for start in ([6, 3, 0], [-4, 3, 99], [0, 6, 2], [5, 5, 5]):
        b.start.copy_(torch.tensor(start, dtype=torch.int32, device=DEV))
        b.run(64 ** -0.5)
        torch.cuda.synchronize()
        assert binding.device_status() == 0
    b.start.copy_(good)
    assert torch.equal(b.check(), want)


def test_rotation_append_and_shared_decode_together():
    """A step of a model with rotary positions, as it would be used: rotate and append the new tokens, then attend behind
    the shared prefix; no synchronisation in between, three steps, against the definition on the cache they leave."""
    b = Batch(32, 8, 128, 16, sizes=[5, 3], prefix=[700, 320], lens=[703, 720, 701, 760, 800, 321, 330, 400], loose=0, seed=3)
    gen = torch.Generator(DEV).manual_seed(9)
    freq = binding.rotary_table(binding.rotary_frequencies(128, scaling="parts", factor=8.0, original_len=8192.0,
                                                           low_turns=1.0, high_turns=4.0), DEV)
    ws = b.workspace(512)
    out = torch.empty_like(b.q)
    q_raw = b.q
    for step in range(3):
        x = torch.randn(8, (32 + 16) * 128, generator=gen, device=DEV).bfloat16()
        q, k, v = (y.unflatten(1, (-1, 128)) for y in x.split([4096, 1024, 1024], 1))
        # the sequences grow by one token; their last page has room (the lengths above end inside a page)
        pos = b.lens - 1
        page = b.table.gather(1, (pos // 16).long()[:, None])[:, 0].long()
        b.q = torch.empty_like(q_raw)
        binding.rotary_append(b.q, q, k, v, b.k, b.v, page * 16 + pos % 16, pos, freq, 0)
        b.run(128 ** -0.5, ws=ws, out=out)
        want, size = b.wanted(128 ** -0.5)
        assert bool(((out.double() - want).abs() <= (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs()).all())
        assert torch.equal(b.v[page, :, pos % 16], v)
        grown = [n + 1 if n % 16 else n for n in b.n]
        b.n = grown
        b.lens.copy_(torch.tensor(grown, dtype=torch.int32, device=DEV))
    assert binding.device_status() == 0


def test_pages_past_32_bit_offsets():
    """The same batch with its pages at the end of a pool of 2^33 bytes: element and byte offsets pass 32 bits."""
    b = Batch(8, 2, 128, 16, sizes=[3], prefix=[200], lens=[201, 260, 330], loose=0, slopes=True)
    want = b.check()
    pool, used = 2 ** 33 // (2 * 16 * 128 * 2), b.k.shape[0]
    for name in ("k", "v"):
        big = torch.empty(pool, 2, 16, 128, dtype=torch.bfloat16, device=DEV)
        big[pool - used:] = getattr(b, name)
        setattr(b, name, big)
    b.table.copy_(torch.where(b.table >= 0, b.table + (pool - used), b.table))
    assert torch.equal(b.run(128 ** -0.5), want)


def test_a_page_named_more_than_once():
    """A page that a sequence names twice, and that two groups and a sequence of none have in common."""
    b = Batch(16, 4, 64, 16, sizes=[3, 2], prefix=[256, 192], lens=[300, 310, 320, 200, 210, 150], loose=1)
    b.table[:3, 5] = b.table[0, 2]
    b.table[3:5, 1] = b.table[0, 2]
    b.table[5, :2] = b.table[0, 2]
    b.table[4, 12] = b.table[0, 17]
    b.check()


@pytest.mark.parametrize("slopes", [False, True])
def test_infinite_scores_reach_the_rows_that_see_them_alone(slopes):
    """An infinite key: a head whose score is -inf gives it no weight, one whose score is +inf has no value, and a row that
    does not see it is not touched."""
    b = Batch(16, 4, 128, 16, sizes=[4], prefix=[200], lens=[60, 190, 260, 300], slopes=slopes, told=[0, 190, 200, 200])
    before = b.check()
    shared, own = int(b.table[1, 6]), int(b.table[3, 17])
    b.k[shared, 1, 3, 0] = float("inf")
    b.k[own, 2, 9, 5] = float("-inf")
    got = b.run(128 ** -0.5)
    want, size = b.wanted(128 ** -0.5)
    bad = torch.isnan(want)
    assert bad.any() and not bad[0].any() and torch.equal(torch.isnan(got), bad)
    bound = (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs() + 1e-30
    assert bool(((got.double() - want).abs() <= bound)[~bad].all())
    assert torch.equal(got[0], before[0])


def test_two_graphs_with_one_workspace():
    """Two batches captured with the same workspace, replayed one behind the other on one stream."""
    b = Batch(32, 8, 128, 16, sizes=[6], prefix=[800], lens=[801 + 13 * i for i in range(6)], seed=4)
    c = Batch(32, 8, 128, 16, sizes=[2, 4], prefix=[300, 1000], lens=[301, 340, 1000, 1010, 1100, 1200], slopes=True, seed=5)
    wants = [x.check() for x in (b, c)]
    ws, parts = max((x.workspace(512) for x in (b, c)), key=lambda t: t[0].numel())
    outs, graphs = [torch.empty_like(x.q) for x in (b, c)], [torch.cuda.CUDAGraph() for _ in range(2)]
    for x, out, graph in zip((b, c), outs, graphs):
        with torch.cuda.graph(graph):
            x.run(128 ** -0.5, ws=(ws, parts), out=out)
    for _ in range(4):
        for out, graph in zip(outs, graphs):
            out.fill_(float("nan"))
            graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], wants[0]) and torch.equal(outs[1], wants[1])
