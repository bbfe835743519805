"""The page operators on the GPU against the operators written out on the host: whole numbers and copied bits are equal."""
import numpy as np
import pytest
import torch

from paper_2505_02351_b200 import binding
from tests.pages_model import State

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


class Cache:
    """A cache whose rows have the given lengths, pages in random order; and the same on the host."""

    def __init__(self, lens, blocks, wide=None, Hkv=2, bs=16, D=64, dtype=torch.bfloat16, pools=2, seed=0):
        rng, gen = np.random.default_rng(seed), torch.Generator(DEV).manual_seed(seed)
        S, need = len(lens), [-(-n // bs) for n in lens]
        wide = wide or max(need) + 2
        perm, tables, refs, cur = rng.permutation(blocks), np.full((S, wide), -1), np.zeros(blocks), 0
        for s, k in enumerate(need):
            tables[s, :k] = perm[cur:cur + k]
            cur += k
        assert cur <= blocks
        refs[perm[:cur]] = 1
        self.pools = [torch.randn(blocks, Hkv, bs, D, generator=gen, device=DEV).to(dtype) for _ in range(pools)]
        self.bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
        self.host = State(tables, lens, refs, [p.view(self.bits).cpu().numpy() for p in self.pools], bs)
        self.tables, self.lens, self.refs = dev(tables), dev(lens), dev(refs)
        self.handle = binding.page_pools(self.pools)

    def workspace(self, n):
        need = binding.pages_workspace_bytes(max(n, 1), self.refs.numel())
        return torch.full((need,), 0xa5, device=DEV, dtype=torch.uint8)

    def call(self, name, a, b, stream=None):
        done = torch.full((len(a),), 7, device=DEV, dtype=torch.int32)
        getattr(binding, "cache_" + name)(self.handle, self.tables, self.lens, self.refs, dev(a), dev(b), done, self.workspace(len(a)),
                                          stream=stream)
        torch.cuda.synchronize()
        want = getattr(self.host, name)([int(x) for x in a], [int(x) for x in b])
        assert done.tolist() == want
        self.same()
        return want

    def compact(self, in_place):
        tables, refs = (self.tables, self.refs) if in_place else (torch.full_like(self.tables, 77), torch.full_like(self.refs, 77))
        page_map, used = torch.full_like(self.refs, 77), torch.full((1,), 77, device=DEV, dtype=torch.int32)
        before = self.tables.clone(), self.refs.clone()
        binding.cache_compact(self.handle, self.tables, self.lens, self.refs, tables, refs, page_map, used, self.workspace(1))
        torch.cuda.synchronize()
        if not in_place:
            assert torch.equal(before[0], self.tables) and torch.equal(before[1], self.refs)
        want = self.host.compact()
        for got, w in zip((tables, refs, page_map), want):
            assert np.array_equal(got.cpu().numpy(), w)
        assert used.tolist() == [want[3]]
        self.tables, self.refs, self.host.tables, self.host.refs = tables, refs, want[0], want[1]
        self.same()

    def same(self):
        for got, want in ((self.tables, self.host.tables), (self.lens, self.host.lens), (self.refs, self.host.refs)):
            assert np.array_equal(got.cpu().numpy(), want)
        for got, want in zip(self.pools, self.host.pools):
            assert np.array_equal(got.view(self.bits).cpu().numpy(), want)

    def consistent(self):
        """Every count is the number of table entries below the rows' lengths that name the page."""
        h = self.host
        count = np.zeros_like(h.refs)
        for s in range(len(h.lens)):
            np.add.at(count, h.tables[s, :h.pages(h.lens[s])], 1)
        assert np.array_equal(count, h.refs)


@pytest.mark.parametrize("Hkv,bs,D,dtype,pools", [(1, 16, 64, torch.bfloat16, 1), (8, 16, 128, torch.bfloat16, 4), (3, 32, 64, torch.float32, 3),
                                                  (5, 32, 128, torch.float32, 256)])
@pytest.mark.parametrize("n", [1, 2, 9])
def test_copy_pages(Hkv, bs, D, dtype, pools, n):
    c = Cache([0], 20, Hkv=Hkv, bs=bs, D=D, dtype=dtype, pools=pools, seed=n)
    perm = np.random.default_rng(n).permutation(20)
    src, dst = perm[:n].copy(), perm[n:2 * n].copy()
    if n > 2:
        src[1], dst[2], src[3], dst[4] = -1, -1, 20, 1 << 30        # pairs that are skipped
        src[6] = src[5]                                             # one page to two places
    binding.cache_copy_pages(c.handle, dev(src), dev(dst))
    c.host.copy(src, dst)
    torch.cuda.synchronize()
    c.same()


def test_copy_of_many_pairs_and_of_none():
    c = Cache([0], 6000, pools=3)
    perm = np.random.default_rng(3).permutation(6000)
    binding.cache_copy_pages(c.handle, dev(perm[:3000]), dev(perm[3000:]))
    c.host.copy(perm[:3000], perm[3000:])
    binding.cache_copy_pages(c.handle, dev([]), dev([]))
    torch.cuda.synchronize()
    c.same()


def test_copy_behind_32_bit_offsets():
    """Pages past 2^32 bytes of their pool."""
    pool = torch.empty(140000, 8, 16, 128, device=DEV, dtype=torch.bfloat16)        # 4.6 GB
    pool[139990:] = torch.randn(10, 8, 16, 128, device=DEV)
    pool[:3] = 0
    want = pool[139995].clone()
    h = binding.page_pools([pool])
    binding.cache_copy_pages(h, dev([139995, 139996]), dev([2, 139999]))
    torch.cuda.synchronize()
    assert torch.equal(pool[2], want) and torch.equal(pool[139999], pool[139996]) and not pool[:2].any()


@pytest.mark.parametrize("n", [0, 1, 15, 16, 17, 100, 128, 2000])
@pytest.mark.parametrize("bs", [16, 32])
def test_fork_lengths(n, bs):
    c = Cache([n, 40, 0, 70, 0, 33], 400, bs=bs, wide=130, seed=n)
    assert c.call("fork", [0, 0, 1], [2, 3, 4]) == [1, 1, 1]       # row 3 held pages
    c.consistent()
    assert c.call("fork", [2], [5]) == [1]                         # a child's child
    c.consistent()


@pytest.mark.parametrize("dtype,Hkv,D", [(torch.float32, 3, 128), (torch.bfloat16, 8, 64)])
def test_fork_copies_only_full_rows(dtype, Hkv, D):
    c = Cache([21, 0, 0], 10, Hkv=Hkv, D=D, dtype=dtype, seed=5)
    c.call("fork", [0, 0], [1, 2])


def test_fork_many_children_of_several_parents_again_and_again():
    rng = np.random.default_rng(1)
    C = 150
    lens = [16 * 1030 + 5, 900, 17, 64] + [0] * C
    c = Cache(lens, 1100 + 60 + 200, wide=1040, seed=2)
    for turn in range(3):                                          # the second time the children hold what they got before
        parents = rng.integers(0, 4, size=C)
        if turn == 1:
            parents = np.sort(parents)
        parents[[3, 50]] = -1
        children = 4 + rng.permutation(C)
        children[[7, 8]] = [-1, 4 + C]
        c.call("fork", parents, children)
        c.consistent()


def test_fork_a_run_whose_first_is_void_or_cannot_be_served():
    c = Cache([40, 33, 0, 0, 0, 0], 6 + 2, seed=3)                  # two free pages
    assert c.call("fork", [0, 0, 0, 1], [-1, 2, 3, 9]) == [0, 1, 1, 0]
    c.consistent()
    c = Cache([40, 32, 33, 0, 0, 0, 0, 40], 8 + 3, seed=4)
    # row 7's pages come free within the call; the fourth request finds none left, the fifth asks for none
    assert c.call("fork", [0, 0, 2, 2, 1], [3, 7, 4, 5, 6]) == [1, 1, 1, 0, 1]
    c.consistent()


def test_fork_without_pages_leaves_the_child_empty():
    c = Cache([40, 32, 0, 20, 0], 3 + 2 + 2 + 1, seed=6)
    assert c.call("fork", [0, 0, 1], [2, 4, 3]) == [1, 1, 1]        # row 3's two pages come free
    c = Cache([40, 32, 0, 0, 20], 3 + 2 + 2 + 1, seed=6)
    assert c.call("fork", [0, 0, 1], [2, 3, 4]) == [1, 1, 1]
    c = Cache([40, 32, 0, 0, 0], 3 + 2 + 1, seed=6)
    assert c.call("fork", [0, 0, 1], [2, 3, 4]) == [1, 0, 1]
    c.consistent()


@pytest.mark.parametrize("old", [0, 1, 15, 16, 17, 32, 100])
@pytest.mark.parametrize("new", [0, 1, 16, 17, 33, 99, 100, 101, 400])
def test_resize_one(old, new):
    c = Cache([5, old, 70], 64, wide=25, seed=old * 1000 + new)
    assert c.call("resize", [1], [new]) == [1]
    c.consistent()


def test_resize_drops_first_gives_then():
    c = Cache([160, 0, 20], 12, wide=12, seed=1)                   # all but no page in use
    assert c.call("resize", [1, 0], [160, 0]) == [1, 1]
    c.consistent()
    assert c.call("resize", [0, 2, 1], [33, 40, 160]) == [0, 0, 1]  # none left: nothing is given
    c.consistent()


def test_resize_void_requests_and_the_order_of_the_list():
    c = Cache([16, 16, 16, 16, 16], 9, wide=4, seed=2)             # four free
    assert c.call("resize", [-1, 1, 7, 0, 2, 3, 4], [9, 65, 5, 48, -3, 49, 17]) == [0, 0, 0, 1, 0, 0, 0]
    c.consistent()
    assert c.call("resize", [1, 2, 3], [32, 16, 48]) == [1, 1, 0]
    c.consistent()


def test_resize_copies_a_shared_page_before_it_grows():
    c = Cache([100, 0, 0, 40], 64, wide=10, seed=3)
    c.call("fork", [0, 0], [1, 2])
    # rows 1 and 2 go back into pages that row 0 holds too, then all three grow
    assert c.call("resize", [1, 2], [41, 37]) == [1, 1]
    assert c.call("resize", [2, 1, 0, 3], [38, 90, 101, 41]) == [1, 1, 1, 1]
    c.consistent()
    assert c.call("resize", [1, 0], [64, 64]) == [1, 1]            # ends of pages: nothing to copy
    assert c.call("resize", [1, 0], [65, 66]) == [1, 1]
    c.consistent()


def test_resize_both_holders_of_a_page_grow():
    c = Cache([20, 0], 8, wide=4, seed=4)
    c.tables[1, :2], c.lens[1] = c.tables[0, :2].clone(), 20
    c.refs[c.tables[0, :2].long()] = 2
    c.host.tables[1, :2], c.host.lens[1] = c.host.tables[0, :2], 20
    c.host.refs[c.host.tables[0, :2]] = 2
    assert c.call("resize", [0, 1], [21, 32]) == [1, 1]
    c.consistent()


@pytest.mark.parametrize("n,blocks,wide", [(1, 40000, 8192), (300, 70001, 600), (5000, 40000, 20)])
def test_resize_sizes(n, blocks, wide):
    """One long request, a batch over pools of several rounds of the scan, more requests than threads of a CTA."""
    rng = np.random.default_rng(n)
    S = n + 3
    lens = np.zeros(S, dtype=int)
    some = rng.permutation(S)[:S // 2]
    lens[some] = rng.integers(0, 16 * wide // 4, size=S // 2) if n > 1 else 0
    while (-(-lens // 16)).sum() > blocks * 3 // 4:
        lens[rng.integers(S)] = 0
    c = Cache([int(x) for x in lens], blocks, wide=wide, Hkv=1, pools=1, seed=n)
    seqs = rng.permutation(S)[:n]
    for turn in range(2):
        new = rng.integers(0, 16 * wide // 3, size=n) if n > 1 else np.array([16 * wide - turn * 70000])
        c.call("resize", seqs, new)
        c.consistent()


@pytest.mark.parametrize("blocks", [1, 3, 4, 5, 63, 1000, 33000, 70001])
@pytest.mark.parametrize("share", [0.0, 0.3, 0.97, 1.0])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(blocks, share, in_place):
    rng = np.random.default_rng(blocks)
    take = int(blocks * share)
    lens = []
    while take > 0:
        k = min(take, int(rng.integers(1, 300)))
        lens.append(16 * k - int(rng.integers(0, 16)))
        take -= k
    c = Cache(lens + [0], blocks, Hkv=1, pools=1 if blocks > 1000 else 2, seed=blocks)
    c.compact(in_place)
    c.consistent()
    assert not (c.host.refs[int((c.host.refs > 0).sum()):] > 0).any()


def test_compact_keeps_pages_held_by_no_table_and_shared_ones():
    c = Cache([100, 50, 0], 40, Hkv=5, bs=32, D=128, dtype=torch.float32, pools=3, seed=9)
    c.call("fork", [0], [2])
    extra = int(np.flatnonzero(c.host.refs == 0)[-1])
    c.refs[extra] = 3
    c.host.refs[extra] = 3
    c.compact(True)


def test_compact_leaves_the_old_tables_readable():
    """Pages keep their contents until they are given away: the old tables name the same tokens."""
    c = Cache([300, 77, 140], 200, Hkv=2, pools=2, seed=10)
    old = [p[c.tables[0, :19].long()].clone() for p in c.pools]
    before = c.tables.clone()
    c.compact(False)
    for p, o in zip(c.pools, old):
        assert torch.equal(p[before[0, :19].long()], o) and torch.equal(p[c.tables[0, :19].long()], o)


@pytest.mark.parametrize("blocks", [4096, 4097])
@pytest.mark.parametrize("n,wide", [(40, 64), (60, 68), (61, 68), (40, 900), (512, 8), (513, 8)])
def test_fork_and_resize_on_both_sides_of_the_launches_choice(blocks, n, wide):
    """One CTA or a cluster, the children's pages dropped by it or before it."""
    rng = np.random.default_rng(n + wide)
    c = Cache([16 * (wide - 2) + 9, 50] + [0] * n, blocks, wide=wide, Hkv=1, pools=1, seed=n)
    for turn in range(2):                                          # the second time the children hold what they got before
        c.call("fork", rng.integers(0, 2, size=n), 2 + rng.permutation(n))
        c.consistent()
    c.call("resize", 2 + rng.permutation(n), rng.integers(0, 16 * wide + 1, size=n))
    c.consistent()


def test_more_requests_than_shared_memory_holds():
    rng = np.random.default_rng(12)
    n, parents = 8200, 3
    c = Cache([75, 64, 5] + [0] * n, 3 * n, wide=8, Hkv=1, pools=1, seed=12)
    c.call("fork", np.sort(rng.integers(0, parents, size=n)), parents + rng.permutation(n))
    c.consistent()
    for _ in range(2):
        c.call("resize", parents + rng.permutation(n), rng.integers(-1, 100, size=n))
        c.consistent()


@pytest.mark.parametrize("blocks", [1024, 1025, 4096, 4097])
def test_compact_on_both_sides_of_the_launches_choice(blocks):
    rng = np.random.default_rng(blocks)
    c = Cache([int(x) for x in rng.integers(0, 16 * blocks // 64, size=80)], blocks, Hkv=1, pools=2, seed=blocks)
    c.compact(True)
    c.consistent()


@pytest.mark.parametrize("seed", range(6))
def test_a_run_of_steps(seed):
    """Forks, steps, ends and compactions in turn, each checked."""
    rng = np.random.default_rng(100 + seed)
    S, bs = 24, int(rng.choice([16, 32]))
    lens = [int(x) for x in rng.integers(1, 300, size=6)] + [0] * (S - 6)
    c = Cache(lens, int(rng.integers(120, 240)), wide=24, Hkv=int(rng.integers(1, 4)), bs=bs, pools=2, seed=seed)
    for turn in range(14):
        kind = rng.random()
        rows = rng.permutation(S)
        if kind < 0.3:
            k = int(rng.integers(1, 6))
            live = [r for r in rows[:12] if c.host.lens[r]] or [int(rows[0])]
            c.call("fork", rng.choice(live, size=k), rows[12:12 + k])
        elif kind < 0.85:
            k = int(rng.integers(1, S + 1))
            old = c.host.lens[rows[:k]]
            new = np.where(rng.random(k) < 0.2, 0, np.maximum(old + rng.integers(-20, 40, size=k), -1))
            c.call("resize", rows[:k], new)
        else:
            c.compact(bool(rng.integers(2)))
        c.consistent()


def test_captured_and_replayed_on_another_stream():
    c = Cache([100, 0, 0, 70], 64, wide=10, seed=11)
    ws, done = c.workspace(2), torch.zeros(2, device=DEV, dtype=torch.int32)
    a, b, seqs, new = dev([0, 0]), dev([1, 2]), dev([1, 3]), dev([117, 40])
    before = [x.clone() for x in (c.tables, c.lens, c.refs)]
    binding.cache_fork(c.handle, c.tables, c.lens, c.refs, a, b, done, ws)           # the first calls outside the capture
    binding.cache_resize(c.handle, c.tables, c.lens, c.refs, seqs, new, done, ws)
    torch.cuda.synchronize()
    for x, o in zip((c.tables, c.lens, c.refs), before):
        x.copy_(o)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        binding.cache_fork(c.handle, c.tables, c.lens, c.refs, a, b, done, ws)
        binding.cache_resize(c.handle, c.tables, c.lens, c.refs, seqs, new, done, ws)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        c.host.fork([0, 0], [1, 2])
        c.host.resize([1, 3], [117, 40])
        c.same()
        c.consistent()


def test_refusals_of_the_binding():
    c = Cache([100, 0], 64, wide=10)
    ws, one, done = c.workspace(1), dev([0]), dev([0])
    good = dict(pools=c.handle, block_tables=c.tables, context_lens=c.lens, ref_counts=c.refs, parents=one, children=dev([1]), done=done,
                workspace=ws)
    for bad in (dict(block_tables=c.tables[0]), dict(block_tables=c.tables.long()), dict(context_lens=c.lens[:1]),
                dict(ref_counts=c.refs[:-1]), dict(children=dev([1, 0])), dict(done=dev([0, 0])), dict(parents=one.cpu()),
                dict(block_tables=c.tables[:, :5])):
        with pytest.raises(ValueError):
            binding.cache_fork(**dict(good, **bad))
    with pytest.raises(binding.OptGqaError) as e:
        binding.cache_fork(**dict(good, workspace=ws[:-256]))
    assert e.value.code == -2
    with pytest.raises(ValueError):
        binding.page_pools([c.pools[0], c.pools[1][:-1]])
    with pytest.raises(ValueError):
        binding.page_pools([c.pools[0].half()])
    torch.cuda.synchronize()
    c.same()


class Elsewhere:
    """A workspace on another device, as the binding sees it."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.t.get_device() + 1


def test_workspaces_of_another_device_or_with_gaps_are_refused():
    c = Cache([30, 0], 8)
    to, used = [torch.empty_like(x) for x in (c.tables, c.refs, c.refs)], dev([0])
    for ws in (Elsewhere(c.workspace(1)), torch.empty(1 << 16, device=DEV)[::2], torch.empty(1 << 16)):
        for f in (binding.cache_fork, binding.cache_resize):
            with pytest.raises(ValueError):
                f(c.handle, c.tables, c.lens, c.refs, dev([0]), dev([1]), dev([0]), ws)
        with pytest.raises(ValueError):
            binding.cache_compact(c.handle, c.tables, c.lens, c.refs, *to, used, ws)
    assert c.call("fork", [0], [1]) == [1]
