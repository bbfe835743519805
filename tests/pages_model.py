"""The page operators written out on the host, request by request (numpy, no shared code with the library)."""
import numpy as np


class State:
    """tables [S, W], lens [S], refs [num_blocks] int32; pools: list of arrays [num_blocks, Hkv, bs, D]."""

    def __init__(self, tables, lens, refs, pools, bs):
        self.tables, self.lens, self.refs = (np.array(a, dtype=np.int32) for a in (tables, lens, refs))
        self.pools, self.bs = [np.array(p) for p in pools], bs

    def pages(self, tokens):
        return -(-int(tokens) // self.bs)

    def drop(self, row, lo, hi):
        for i in range(lo, hi):
            self.refs[self.tables[row, i]] -= 1
            self.tables[row, i] = -1

    def free(self):
        return [int(p) for p in np.flatnonzero(self.refs == 0)]

    def copy(self, src, dst):
        nb = self.refs.size
        for s, d in zip(src, dst):
            if 0 <= s < nb and 0 <= d < nb:
                for p in self.pools:
                    p[d] = p[s]

    def fork(self, parents, children):
        S, W = self.tables.shape
        ok = [0 <= p < S and 0 <= c < S for p, c in zip(parents, children)]
        for c, o in zip(children, ok):
            if o:
                self.drop(c, 0, self.pages(self.lens[c]))
                self.lens[c] = 0
        free, asked, done = self.free(), 0, []
        for p, c, o in zip(parents, children, ok):
            if not o:
                done.append(0)
                continue
            n = int(self.lens[p])
            need = int(n % self.bs != 0)
            mine = free[asked:asked + need]
            asked += need
            if len(mine) < need:
                done.append(0)
                continue
            for i in range(n // self.bs):
                self.tables[c, i] = self.tables[p, i]
                self.refs[self.tables[p, i]] += 1
            if need:
                i, r = n // self.bs, n % self.bs
                self.tables[c, i] = mine[0]
                self.refs[mine[0]] = 1
                for pool in self.pools:
                    pool[mine[0]][:, :r] = pool[self.tables[p, i]][:, :r]
            self.lens[c] = n
            done.append(1)
        return done

    def resize(self, seqs, new_lens):
        S, W = self.tables.shape
        ok = [0 <= s < S and 0 <= n <= W * self.bs for s, n in zip(seqs, new_lens)]
        for s, n, o in zip(seqs, new_lens, ok):
            if o and n < self.lens[s]:
                self.drop(s, self.pages(n), self.pages(self.lens[s]))
        held, free, asked, done = self.refs.copy(), self.free(), 0, []
        for s, n, o in zip(seqs, new_lens, ok):
            if not o:
                done.append(0)
                continue
            old, fresh = int(self.lens[s]), 0
            first = self.pages(old)
            if n > old:
                fresh = self.pages(n) - first
                if old % self.bs and held[self.tables[s, first - 1]] > 1:
                    fresh, first = fresh + 1, first - 1
            mine = free[asked:asked + fresh]
            asked += fresh
            if len(mine) < fresh:
                done.append(0)
                continue
            if fresh and first < self.pages(old):
                was = self.tables[s, first]
                for pool in self.pools:
                    pool[mine[0]][:, :old % self.bs] = pool[was][:, :old % self.bs]
                self.refs[was] -= 1
            for i, page in enumerate(mine):
                self.tables[s, first + i] = page
                self.refs[page] = 1
            self.lens[s] = n
            done.append(1)
        return done

    def compact(self):
        """(tables, refs, page map, pages in use); the pools are moved."""
        used = [int(p) for p in np.flatnonzero(self.refs > 0)]
        U = len(used)
        movers, holes = [p for p in used if p >= U], [p for p in range(U) if self.refs[p] <= 0]
        page_map = np.full(self.refs.size, -1, dtype=np.int32)
        page_map[used] = used
        for m, h in zip(movers, holes):
            page_map[m] = h
            for pool in self.pools:
                pool[h] = pool[m]
        refs = np.zeros_like(self.refs)
        refs[page_map[used]] = self.refs[used]
        tables = self.tables.copy()
        for s in range(tables.shape[0]):
            for i in range(self.pages(self.lens[s])):
                tables[s, i] = page_map[tables[s, i]]
        return tables, refs, page_map, U
