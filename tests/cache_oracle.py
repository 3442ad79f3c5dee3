"""The page operations of a cache on host lists, one page and one row at a time, from their definitions."""
import numpy as np
import torch


class CacheOracle:
    def __init__(self, k, v, table, lens, refs):
        self.k, self.v = k.clone(), v.clone()
        self.table, self.lens, self.refs = table.tolist(), lens.tolist(), refs.tolist()
        self.ps, self.max_pages, self.status = k.shape[2], table.shape[1], [0, 0]

    def pages_of(self, n):
        return -(-n // self.ps)

    def free_list(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def grow(self, seqs, counts):
        bad = len(set(seqs)) != len(seqs) or any(not 0 <= s < len(self.lens) for s in seqs)
        bad = bad or any(c < 0 or self.lens[s] + c > self.max_pages * self.ps for s, c in zip(seqs, counts))
        if bad:
            self.status = [1, 0]
            return
        need = [self.pages_of(self.lens[s] + c) - self.pages_of(self.lens[s]) for s, c in zip(seqs, counts)]
        free = self.free_list()
        if sum(need) > len(free):
            self.status = [2, sum(need) - len(free)]
            return
        for s, c, n in zip(seqs, counts, need):
            first = self.pages_of(self.lens[s])
            for j in range(n):
                p = free.pop(0)
                self.table[s][first + j], self.refs[p] = p, 1
            self.lens[s] += c
        self.status = [0, 0]

    def fork(self, parents, children):
        S = len(self.lens)
        bad = any(not 0 <= x < S for x in parents + children) or len(set(children)) != len(children)
        bad = bad or bool(set(parents) & set(children)) or any(self.lens[c] != 0 for c in children)
        if bad:
            self.status = [1, 0]
            return
        free = self.free_list()
        need = sum(self.lens[p] % self.ps != 0 for p in parents)
        if need > len(free):
            self.status = [2, need - len(free)]
            return
        for p, c in zip(parents, children):
            n = self.lens[p]
            row = [-1] * self.max_pages
            for i in range(n // self.ps):
                row[i] = self.table[p][i]
                self.refs[row[i]] += 1
            if n % self.ps:
                new, old = free.pop(0), self.table[p][n // self.ps]
                row[n // self.ps], self.refs[new] = new, 1
                for x in (self.k, self.v):
                    x[:, new, :n % self.ps] = x[:, old, :n % self.ps]
            self.table[c], self.lens[c] = row, n
        self.status = [0, 0]

    def free(self, seqs):
        self.status = [0, 0]
        for s in seqs:
            if not 0 <= s < len(self.lens):
                self.status[0] = 1
                continue
            for i in range(self.pages_of(self.lens[s])):
                self.refs[self.table[s][i]] -= 1
                self.table[s][i] = -1
            self.lens[s] = 0

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] == 0]
        high = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        assert len(holes) == len(high)
        for d, s in zip(holes, high):
            for x in (self.k, self.v):
                x[:, d] = x[:, s]
            self.refs[d], self.refs[s] = self.refs[s], 0
        to = dict(zip(high, holes))
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        self.status = [0, 0]

    def write(self, layer, seqs, counts, k, v, starts=None):
        per = k.shape[0] // len(seqs) if seqs else 0
        for i, (s, c) in enumerate(zip(seqs, counts)):
            first = starts[i] if starts is not None else i * per
            top = k.shape[0] if starts is not None else first + per
            for j in range(c):
                pos, row = self.lens[s] - c + j, first + j
                if row < top and pos >= 0:
                    page = self.table[s][pos // self.ps]
                    self.k[layer, page, pos % self.ps] = k[row]
                    self.v[layer, page, pos % self.ps] = v[row]

    def compare(self, cache):
        torch.cuda.synchronize()
        assert cache.status.tolist() == self.status, (cache.status.tolist(), self.status)
        assert cache.lens.tolist() == self.lens
        assert cache.refs.tolist() == self.refs
        assert cache.table.tolist() == self.table
        for n, a, b in (("k", cache.k, self.k), ("v", cache.v, self.v)):
            assert torch.equal(a.cpu(), b), n
        held = np.bincount([p for row in self.table for p in row if p >= 0], minlength=len(self.refs))
        assert held.tolist() == self.refs
