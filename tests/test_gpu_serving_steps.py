"""The page operators and the attention calls as a server would run them together: prompts admitted, continued in samples, drafts
verified and taken back, ended, the pools compacted -- attention checked at each step against the tokens' keys and values in 64
bits, kept on the host side of the test apart from any page."""
import numpy as np
import pytest
import torch

from paper_2505_02351_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Server:
    def __init__(self, rows, blocks, Hq=8, Hkv=2, D=64, bs=16, width=40, layers=2, seed=0):
        self.Hq, self.Hkv, self.D, self.bs = Hq, Hkv, D, bs
        self.gen = torch.Generator(DEV).manual_seed(seed)
        self.pools = [torch.full((blocks, Hkv, bs, D), float("nan"), device=DEV, dtype=torch.bfloat16) for _ in range(2 * layers)]
        self.handle = binding.page_pools(self.pools)
        i32 = lambda *s, fill=0: torch.full(s, fill, device=DEV, dtype=torch.int32)  # noqa: E731
        self.table, self.lens, self.refs = i32(rows, width, fill=-1), i32(rows), i32(blocks)
        self.page_map, self.used = i32(blocks), i32(1)
        self.ws = torch.empty(binding.pages_workspace_bytes(rows, blocks), device=DEV, dtype=torch.uint8)
        self.chunk_ws = torch.empty(binding.chunk_workspace_bytes(Hq, Hkv, D, 128), device=DEV, dtype=torch.uint8)
        empty = torch.empty(0, Hkv, D, device=DEV, dtype=torch.bfloat16)
        self.tokens = [[empty] * (2 * layers) for _ in range(rows)]        # what each row holds, by pool
        self.layers = layers

    def dev(self, a):
        return torch.tensor([int(x) for x in a], device=DEV, dtype=torch.int32)

    def randn(self, *s):
        return torch.randn(*s, generator=self.gen, device=DEV).bfloat16()

    def resize(self, rows, lens):
        done = torch.zeros(len(rows), device=DEV, dtype=torch.int32)
        binding.cache_resize(self.handle, self.table, self.lens, self.refs, self.dev(rows), self.dev(lens), done, self.ws)
        assert done.tolist() == [1] * len(rows)
        for r, n in zip(rows, lens):
            self.tokens[r] = [t[:n] for t in self.tokens[r]]

    def fork(self, parents, children):
        done = torch.zeros(len(parents), device=DEV, dtype=torch.int32)
        binding.cache_fork(self.handle, self.table, self.lens, self.refs, self.dev(parents), self.dev(children), done, self.ws)
        assert done.tolist() == [1] * len(parents)
        for p, c in zip(parents, children):
            self.tokens[c] = list(self.tokens[p])

    def compact(self):
        binding.cache_compact(self.handle, self.table, self.lens, self.refs, self.table, self.refs, self.page_map, self.used, self.ws)

    def step(self, rows, new, layer=0, slopes=None, window=0):
        """`new` tokens for each of `rows`: room, keys and values stored in every layer, attention in one; checked."""
        have = [self.tokens[r][0].shape[0] for r in rows]
        self.resize(rows, [h + m for h, m in zip(have, new)])
        T = sum(new)
        row = torch.repeat_interleave(self.dev(rows).long(), self.dev(new).long())
        pos = torch.cat([torch.arange(h, h + m, device=DEV) for h, m in zip(have, new)])
        slots = self.table[row, pos // self.bs].long() * self.bs + pos % self.bs
        for l in range(self.layers):
            k, v = self.randn(T, self.Hkv, self.D), self.randn(T, self.Hkv, self.D)
            binding.cache_append(k, v, self.pools[2 * l], self.pools[2 * l + 1], slots)
            at = 0
            for r, m in zip(rows, new):
                for i, x in ((2 * l, k), (2 * l + 1, v)):
                    self.tokens[r][i] = torch.cat([self.tokens[r][i], x[at:at + m]])
                at += m
        q, out = self.randn(T, self.Hq, self.D), torch.full((T, self.Hq, self.D), float("nan"), device=DEV, dtype=torch.bfloat16)
        start = self.dev(np.concatenate([[0], np.cumsum(new)]))
        at = self.dev(rows).long()
        binding.paged_attention_chunk(out, q, start, max(new), self.pools[2 * layer], self.pools[2 * layer + 1],
                                      self.table[at].contiguous(), self.lens[at].contiguous(), slopes, self.D ** -0.5, self.chunk_ws, window=window)
        self.check(out, q, rows, new, layer, slopes, window)
        return out

    def check(self, out, q, rows, new, layer, slopes=None, window=0):
        t, G = 0, self.Hq // self.Hkv
        for r, m in zip(rows, new):
            k, v = (self.tokens[r][2 * layer + i].double() for i in (0, 1))
            n = k.shape[0]
            back = torch.arange(n - m, n, device=DEV)[:, None] - torch.arange(n, device=DEV)
            hidden = (back < 0) | (back >= window) if window else back < 0
            for h in range(self.Hq):
                z = q[t:t + m, h].double() @ k[:, h // G].T * self.D ** -0.5
                if slopes is not None:
                    z -= slopes[h].double() * back
                p = torch.softmax(z.masked_fill(hidden, -float("inf")), -1)
                want, size = p @ v[:, h // G], p @ v[:, h // G].abs()
                # two roundings of the weights to bf16 and one of the result (2^-8 each), fp32 sums: as for the chunk attention alone
                assert bool(((out[t:t + m, h].double() - want).abs() <= (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs()).all()), (r, h)
            t += m


@pytest.mark.parametrize("bs,seed", [(16, 0), (32, 1)])
def test_prompts_samples_drafts_ends_and_compaction(bs, seed):
    s = Server(rows=20, blocks=300, bs=bs, seed=seed)
    slopes = torch.exp2(-torch.arange(1, 9, device=DEV, dtype=torch.float32))
    s.step([0, 1, 2], [100, 37, 200], slopes=slopes)               # three prompts
    s.step([0, 3, 1], [1, 64, 150], layer=1, slopes=slopes)        # a decode row, a new prompt and a chunk of another
    s.fork([0, 0, 1, 0], [10, 11, 12, 13])                         # samples
    s.step([0, 10, 11, 12, 13, 2], [1, 4, 5, 3, 1, 1], slopes=slopes)      # drafts next to decode rows
    s.resize([10, 11, 12], [103, 101, 188])                        # some of them refused
    s.step([10, 11, 12, 0], [2, 1, 6, 1], slopes=slopes)
    s.resize([0, 3, 13], [0, 0, 0])                                # the parent and others end
    s.compact()
    assert s.used.item() == int((s.refs > 0).sum()) and not (s.refs[s.used.item():] != 0).any()
    s.step([10, 11, 12, 1, 2], [1, 1, 1, 1, 1], layer=1, slopes=slopes)
    s.resize([10], [50])                                           # back into pages that row 11 holds too
    s.step([10, 11], [9, 2], window=40)
    s.fork([10, 12, 12], [0, 3, 4])
    s.compact()
    s.step([0, 3, 4, 12, 10], [3, 1, 2, 1, 30])


def test_samples_attend_through_the_shared_prefix_decode():
    """Tables that the fork made, with the prefix's pages read once for the group."""
    s = Server(rows=40, blocks=3000, Hq=32, Hkv=8, D=128, width=300, layers=1, seed=2)
    s.step([0], [4001])
    s.fork([0] * 32, list(range(4, 36)))
    rows = list(range(4, 36))
    s.step(rows, [1 + i % 3 for i in range(32)])
    q, out = s.randn(32, 32, 128), torch.full((32, 32, 128), float("nan"), device=DEV, dtype=torch.bfloat16)
    ws = torch.empty(binding.shared_workspace_bytes(32, 32, 8, 128, 1, 10), device=DEV, dtype=torch.uint8)
    binding.paged_attention_decode_shared(out, q, s.pools[0], s.pools[1], s.table[4:36].contiguous(), s.lens[4:36].contiguous(), s.dev([0, 32]),
                                          torch.full((32,), 4001 // 16 * 16, device=DEV, dtype=torch.int32), None, 128 ** -0.5, 512, ws, 10)
    s.check(out, q, rows, [1] * 32, 0)
    assert int((s.refs == 33).sum()) == 4001 // 16                  # the parent's full pages, held by all


def test_a_step_captured_once_and_replayed():
    """Growth, storing, attention and taking back as one graph: the same step again and again gives the same rows."""
    s = Server(rows=6, blocks=100, seed=3)
    s.step([0, 1, 2], [70, 16, 33])
    rows, new = [0, 1, 2], [3, 1, 5]
    T, have = sum(new), [70, 16, 33]
    more, back = s.dev([h + m for h, m in zip(have, new)]), s.dev(have)
    at = s.dev(rows)
    row = torch.repeat_interleave(at.long(), s.dev(new).long())
    pos = torch.cat([torch.arange(h, h + m, device=DEV) for h, m in zip(have, new)])
    k, v, q = s.randn(T, 2, 64), s.randn(T, 2, 64), s.randn(T, 8, 64)
    start, done = s.dev([0, 3, 4, 9]), torch.zeros(3, device=DEV, dtype=torch.int32)
    out = torch.zeros_like(q)

    def step():
        binding.cache_resize(s.handle, s.table, s.lens, s.refs, at, more, done, s.ws)
        slots = s.table[row, pos // s.bs].long() * s.bs + pos % s.bs
        binding.cache_append(k, v, s.pools[0], s.pools[1], slots)
        binding.paged_attention_chunk(out, q, start, 5, s.pools[0], s.pools[1], s.table[:3], s.lens[:3], None, 0.125, s.chunk_ws)
        binding.cache_resize(s.handle, s.table, s.lens, s.refs, at, back, done, s.ws)

    step()
    torch.cuda.synchronize()
    want, table, refs = out.clone(), s.table.clone(), s.refs.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(4):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(s.table, table) and torch.equal(s.refs, refs) and s.lens.tolist()[:3] == have
    at_row = 0
    for r, m in zip(rows, new):
        for i, x in ((0, k), (1, v)):
            s.tokens[r][i] = torch.cat([s.tokens[r][i], x[at_row:at_row + m]])
        at_row += m
    s.check(out, q, rows, new, 0)
    assert binding.device_status() == 0
