"""The C entry points of the page operators called by their names, against the same calls by a record of their arguments."""
import pytest
import torch

from paper_2505_02351_b200 import binding
from tests.test_gpu_chunk import Batch
from tests.test_gpu_pages import DEV, Cache, dev

pytestmark = pytest.mark.gpu


def ptr(t):
    return t.data_ptr()


class Direct(Cache):
    def call(self, name, a, b, stream=None):
        h, ws, n = self.handle, self.workspace(len(a)), len(a)
        done, x, y = torch.full((n,), 7, device=DEV, dtype=torch.int32), dev(a), dev(b)
        S, W = self.tables.shape
        rc = getattr(binding.load(), "opt_gqa_cache_" + name)(
            h.address, h.count, ptr(self.tables), W, ptr(self.lens), ptr(self.refs), ptr(x), ptr(y), n, ptr(done), S, h.Hkv, h.D, h.bs,
            h.num_blocks, ptr(ws), ws.nbytes, h.code, None)
        torch.cuda.synchronize()
        assert rc == 0
        want = getattr(self.host, name)([int(v) for v in a], [int(v) for v in b])
        assert done.tolist() == want
        self.same()
        return want


@pytest.mark.parametrize("blocks", [300, 6000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_fork_resize_copy_and_compact(blocks, dtype):
    c = Direct([100, 33, 0, 70, 0, 0], blocks, wide=12, Hkv=3, bs=32, D=128, dtype=dtype, pools=3, seed=blocks)
    assert c.call("fork", [0, 0, -1, 1], [2, 4, 5, 3]) == [1, 1, 0, 1]
    c.consistent()
    assert c.call("resize", [2, 0, 9, 4], [101, 64, 5, 384]) == [1, 1, 0, 1]
    c.consistent()
    h, lib = c.handle, binding.load()
    free = [int(p) for p in (c.host.refs == 0).nonzero()[0][-2:]]
    src, dst = dev([int(c.host.tables[0, 0]), -1]), dev(free)
    assert lib.opt_gqa_cache_copy_pages(h.address, h.count, ptr(src), ptr(dst), 2, h.Hkv, h.D, h.bs, h.num_blocks, h.code, None) == 0
    c.host.copy(src.tolist(), free)
    torch.cuda.synchronize()
    c.same()
    tables, refs, page_map, used, ws = (torch.empty_like(c.tables), torch.empty_like(c.refs), torch.empty_like(c.refs), dev([0]), c.workspace(1))
    assert lib.opt_gqa_cache_compact(h.address, h.count, ptr(c.tables), ptr(tables), c.tables.shape[1], ptr(c.lens), ptr(c.refs), ptr(refs),
                                     ptr(page_map), ptr(used), c.tables.shape[0], h.Hkv, h.D, h.bs, h.num_blocks, ptr(ws), ws.nbytes, h.code,
                                     None) == 0
    torch.cuda.synchronize()
    want = c.host.compact()
    assert all(torch.equal(g.cpu(), torch.from_numpy(w)) for g, w in zip((tables, refs, page_map), want)) and used.tolist() == [want[3]]
    c.tables, c.refs, c.host.tables, c.host.refs = tables, refs, want[0], want[1]
    c.same()


def test_chunk_attention():
    b = Batch(16, 4, 128, 16, q_lens=[5, 1, 40], lens=[900, 90, 41], seed=1, slopes=True)
    want, got, ws = b.run(0.1, window=300), torch.full_like(b.q, 7.0), b.workspace()
    rc = binding.load().opt_gqa_paged_attention_chunk(
        ptr(got), ptr(b.q), 16 * 128, ptr(b.start), 46, 40, ptr(b.k), ptr(b.v), ptr(b.table), b.table.shape[1], ptr(b.lens), ptr(b.slopes),
        0.1, 3, 16, 4, 128, 16, b.k.shape[0], 300, ptr(ws), ws.nbytes, 1, None)
    torch.cuda.synchronize()
    assert rc == 0 and torch.equal(got, want)
