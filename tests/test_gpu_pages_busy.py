"""The page operators' clusters behind and beside kernels that leave multiprocessors free at different times, so that the CTAs of a
cluster begin at different times: the sums they tell each other arrive whatever the order."""
import numpy as np
import pytest
import torch

from paper_2505_02351_b200 import binding
from tests.test_gpu_chunk import Batch
from tests.test_gpu_pages import DEV, Cache, dev

pytestmark = pytest.mark.gpu


class Load:
    """Attention over contexts of very different lengths on the call's stream, products on another."""

    def __init__(self):
        rng = np.random.default_rng(0)
        self.batch = Batch(16, 4, 128, 16, q_lens=[1] * 90, lens=[int(x) for x in rng.integers(1, 3000, size=90)], seed=1)
        self.ws, self.out = self.batch.workspace(), torch.empty_like(self.batch.q)
        self.a = torch.randn(2048, 2048, device=DEV, dtype=torch.bfloat16)
        self.other = torch.cuda.Stream()
        torch.cuda.synchronize()

    def go(self):
        self.batch.run(0.1, ws=self.ws, out=self.out)
        with torch.cuda.stream(self.other):
            self.a @ self.a


@pytest.mark.parametrize("blocks", [1025, 5000, 70001])
def test_compact(blocks):
    rng = np.random.default_rng(blocks)
    lens = [int(x) for x in rng.integers(0, 16 * min(blocks, 8000) // 64, size=60)]
    c, load, turns = Cache(lens, blocks, Hkv=1, pools=1, seed=blocks), Load(), 40
    outs = [tuple(torch.full_like(x, 77) for x in (c.tables, c.refs, c.refs)) + (dev([77]),) for _ in range(turns)]
    ws = c.workspace(1)
    for tables, refs, page_map, used in outs:
        load.go()
        binding.cache_compact(c.handle, c.tables, c.lens, c.refs, tables, refs, page_map, used, ws)
    torch.cuda.synchronize()
    want = c.host.compact()
    for got in outs:
        assert all(np.array_equal(g.cpu().numpy(), w) for g, w in zip(got[:3], want)) and got[3].tolist() == [want[3]]
    for got, w in zip(c.pools, c.host.pools):
        assert np.array_equal(got.view(c.bits).cpu().numpy(), w)
    assert binding.device_status() == 0


@pytest.mark.parametrize("wide", [64, 900])
def test_fork_and_resize(wide):
    """Children whose pages the cluster drops itself, and more than that."""
    n, turns = 61, 40
    c, load = Cache([16 * (wide - 2) + 9, 50] + [0] * n, 5000, wide=wide, Hkv=1, pools=1, seed=wide), Load()
    rng = np.random.default_rng(wide)
    parents, children = [int(x) for x in rng.integers(0, 2, size=n)], [int(x) for x in 2 + rng.permutation(n)]
    more = [16 * wide if p == 0 else 70 for p in parents]
    want = [c.host.fork(parents, children), c.host.resize(children, more)]
    assert want[0] == [1] * n
    done, ws = [torch.zeros(2, n, device=DEV, dtype=torch.int32) for _ in range(turns)], c.workspace(n)
    a, b, m = dev(parents), dev(children), dev(more)
    for d in done:                                  # the children are dropped and made again: the same pages each time
        load.go()
        binding.cache_fork(c.handle, c.tables, c.lens, c.refs, a, b, d[0], ws)
        load.go()
        binding.cache_resize(c.handle, c.tables, c.lens, c.refs, b, m, d[1], ws)
    torch.cuda.synchronize()
    assert all(d.tolist() == want for d in done)
    c.same()
    c.consistent()
    assert binding.device_status() == 0
