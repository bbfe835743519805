"""Attention right behind the page operators, in a graph without a pause: it goes by the tables that they have just written, with a
copy of pages between them too."""
import numpy as np
import pytest
import torch

from paper_2505_02351_b200 import binding
from tests.test_gpu_pages import DEV, Cache, dev

pytestmark = pytest.mark.gpu

# parents of different lengths: the children's tables and lengths change with every fork
PARENTS, N = [700, 333, 48], 40


class Step:
    def __init__(self, blocks, copies):
        self.c = Cache(PARENTS + [0] * N, blocks, wide=50, Hkv=2, D=64, pools=2, seed=blocks)
        self.copies = copies
        self.children, self.done, self.ws = dev(3 + np.arange(N)), torch.zeros(N, device=DEV, dtype=torch.int32), self.c.workspace(N)
        self.parents = [dev([p] * N) for p in range(3)]
        self.q = torch.randn(N, 8, 64, generator=torch.Generator(DEV).manual_seed(1), device=DEV).bfloat16()
        self.start = dev(np.arange(N + 1))
        self.chunk_ws = torch.empty(binding.chunk_workspace_bytes(8, 2, 64, 1), device=DEV, dtype=torch.uint8)
        free = np.flatnonzero(self.c.host.refs == 0)[-2:]               # (handed out last: never here)
        self.src, self.dst = dev([int(self.c.host.tables[0, 0]), -1]), dev(free)
        self.map, self.used = torch.zeros_like(self.c.refs), dev([0])

    def fork(self, parent):
        c = self.c
        binding.cache_fork(c.handle, c.tables, c.lens, c.refs, self.parents[parent], self.children, self.done, self.ws)

    def compact(self):
        c = self.c
        binding.cache_compact(c.handle, c.tables, c.lens, c.refs, c.tables, c.refs, self.map, self.used, self.ws)

    def attend(self, out):
        if self.copies:
            binding.cache_copy_pages(self.c.handle, self.src, self.dst)
        binding.paged_attention_chunk(out, self.q, self.start, 1, self.c.pools[0], self.c.pools[1], self.c.tables[3:], self.c.lens[3:], None,
                                      0.125, self.chunk_ws)


@pytest.mark.parametrize("copies", [False, True])
@pytest.mark.parametrize("blocks", [400, 6000])
def test_forks_and_compactions(blocks, copies):
    s = Step(blocks, copies)
    new = lambda: torch.zeros_like(s.q)  # noqa: E731
    want = []
    for parent in range(3):
        s.fork(parent)
        torch.cuda.synchronize()
        assert s.done.tolist() == [1] * N
        out = new()
        s.attend(out)
        torch.cuda.synchronize()
        want.append(out)
    assert not any(torch.equal(a, b) for a, b in ((want[0], want[1]), (want[1], want[2])))
    order = [0, 1, 2, 1, 0, 2, 2, 0]
    outs, packed = [new() for _ in order], [new() for _ in order]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for p, a, b in zip(order, outs, packed):
            s.fork(p)
            s.attend(a)
            if not copies:                      # (compacted, the free pages are others)
                s.compact()
                s.attend(b)
    for _ in range(30):
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, want[p]) for p, a in zip(order, outs))
        assert copies or all(torch.equal(b, want[p]) for p, b in zip(order, packed))
    assert binding.device_status() == 0
