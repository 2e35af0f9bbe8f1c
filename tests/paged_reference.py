"""Plain form of the paged cache for the tests: bookkeeping one page at a time in Python, attention one row at a time in float64."""
from __future__ import annotations

import math
import random

import torch


class PlainCache:
    """The cache's contents on the CPU; k, v [L, n_pages, Hkv, ps, hd] in the stored type."""

    def __init__(self, k, v, refs, table, length, summary=None):
        self.k, self.v, self.summary = k.clone(), v.clone(), None if summary is None else summary.clone()
        self.refs, self.table, self.len = refs.tolist(), table.tolist(), length.tolist()
        self.ps, self.n_pages, self.max_pages, self.n_seqs = k.shape[3], k.shape[1], len(self.table[0]), len(self.table)

    def _used(self, s):
        return -(-self.len[s] // self.ps)

    def _take(self, n):
        free = [p for p, r in enumerate(self.refs) if r == 0][:n]
        if len(free) < n:
            return None
        for p in free:
            self.refs[p] = 1
        return free

    def append(self, rows_k, rows_v, start, mask=None, node=None):
        status = []
        for s in range(self.n_seqs):
            n = start[s + 1] - start[s]
            if node is None:
                rows = list(range(n))
            elif node[s] >= n:
                status.append(3)
                continue
            else:
                rows = [] if node[s] < 0 else [i for i in range(n) if mask[start[s] + node[s]] >> i & 1]
            if not rows:
                status.append(0)
                continue
            if self.len[s] % self.ps:
                p = self.table[s][self._used(s) - 1]
                if not 0 <= p < self.n_pages or self.refs[p] != 1:
                    status.append(3)
                    continue
            need = -(-(self.len[s] + len(rows)) // self.ps)
            if need > self.max_pages:
                status.append(2)
                continue
            fresh = self._take(need - self._used(s))
            if fresh is None:
                status.append(1)
                continue
            status.append(0)
            u = self._used(s)
            self.table[s][u:u + len(fresh)] = fresh
            for i in rows:
                j, off = divmod(self.len[s], self.ps)
                self.k[:, self.table[s][j], :, off] = rows_k[:, start[s] + i]
                self.v[:, self.table[s][j], :, off] = rows_v[:, start[s] + i]
                self.len[s] += 1
        return status

    def fork(self, src, dst):
        before, status, seen = list(self.len), [], set()
        ok_index = lambda s: 0 <= s < self.n_seqs
        for a, b in zip(src, dst):
            first = b not in seen
            seen.add(b)
            if not ok_index(a) or not ok_index(b) or not first or before[b]:
                status.append(3)
                continue
            full, rest = divmod(before[a], self.ps)
            row = list(self.table[a])
            if rest and not 0 <= row[full] < self.n_pages:
                status.append(3)
                continue
            if rest:
                new = self._take(1)
                if new is None:
                    status.append(1)
                    continue
                for t in (self.k, self.v):
                    t[:, new[0], :, :rest] = t[:, row[full], :, :rest]
                if self.summary is not None:
                    self.summary[:, new[0]] = self.summary[:, row[full]]
                self.table[b][full] = new[0]
            for j in range(full):
                self.table[b][j] = row[j]
                if 0 <= row[j] < self.n_pages:
                    self.refs[row[j]] += 1
            self.len[b] = before[a]
            status.append(0)
        return status

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < self.n_seqs:
                for j in range(self._used(s)):
                    p = self.table[s][j]
                    if 0 <= p < self.n_pages:
                        self.refs[p] -= 1
                    self.table[s][j] = -1
                self.len[s] = 0

    def compact(self):
        used = [p for p, r in enumerate(self.refs) if r > 0]
        low = [p for p in range(len(used)) if self.refs[p] == 0]
        high = [p for p in used if p >= len(used)]
        name = dict(zip(high, low))
        for x, y in name.items():
            for t in (self.k, self.v) + (() if self.summary is None else (self.summary,)):
                t[:, y] = t[:, x]
            self.refs[y], self.refs[x] = self.refs[x], 0
        self.table = [[name.get(p, p) for p in row] for row in self.table]
        return len(used)

    def summarize(self, start=None):
        for s in range(self.n_seqs):
            first = 0 if start is None else max(0, start[s])
            if first >= self.len[s]:
                continue
            for j in range(first // self.ps, self._used(s)):
                p = self.table[s][j]
                if 0 <= p < self.n_pages:
                    rows = self.k[:, p, :, :min(self.ps, self.len[s] - j * self.ps)]
                    self.summary[:, p, :, 0], self.summary[:, p, :, 1] = rows.amin(2), rows.amax(2)

    def select(self, layer, q, start, n_sel, keep_first, keep_last):
        """q [T, Hq, hd]; lists [n_seqs][Hkv][n_sel]."""
        Hkv = self.k.shape[2]
        g, out = q.shape[1] // Hkv, []
        for s in range(self.n_seqs):
            used, heads = self._used(s), []
            for h in range(Hkv):
                value = []
                rows = q[start[s]:start[s + 1], h * g:(h + 1) * g].double().reshape(-1, q.shape[2])
                for j in range(used):
                    p, x = self.table[s][j], -math.inf
                    if 0 <= p < self.n_pages and len(rows):
                        lo, hi = self.summary[layer, p, h].double()
                        x = torch.where(rows > 0, rows * hi, rows * lo).sum(1)
                        x = max([y for y in x.tolist() if y == y], default=-math.inf)
                    value.append((j < keep_first or j >= used - keep_last, x))
                best = sorted(sorted(range(used), key=lambda j: (not value[j][0], 0.0 if value[j][0] else -value[j][1], j))[:n_sel])
                heads.append(best + [-1] * (n_sel - len(best)))
            out.append(heads)
        return out

    def attend(self, layer, q, k, v, start, mask=None, selected=None, scale=1.0):
        """Rows that no sequence has come back as NaN.  mask: a Python integer a row."""
        Hkv, hd = self.k.shape[2], q.shape[2]
        g, out = q.shape[1] // Hkv, torch.full(q.shape, math.nan, dtype=torch.float64)
        for s in range(self.n_seqs):
            for h in range(Hkv):
                slots = range(self._used(s)) if selected is None else [j for j in selected[s][h] if 0 <= j < self._used(s)]
                at = [(self.table[s][j], o) for j in slots if 0 <= self.table[s][j] < self.n_pages
                      for o in range(min(self.ps, self.len[s] - j * self.ps))]
                pages, offs = [p for p, _ in at], [o for _, o in at]
                ck, cv = self.k[layer, pages, h, offs].double(), self.v[layer, pages, h, offs].double()
                n = start[s + 1] - start[s]
                for i in range(n):
                    t = start[s] + i
                    new = [start[s] + j for j in range(n) if mask is None or mask[t] >> j & 1]
                    kk, vv = torch.cat([ck, k[new, h].double()]), torch.cat([cv, v[new, h].double()])
                    for x in range(h * g, h * g + g):
                        if len(kk):
                            out[t, x] = torch.softmax(scale * (kk @ q[t, x].double()), 0) @ vv
                        else:
                            out[t, x] = 0
        return out


def mask_words(rows, words):
    """Python integers -> [T, words] int64."""
    split = [[r >> 64 * w & (1 << 64) - 1 for w in range(words)] for r in rows]
    return torch.tensor([[x - (1 << 64) if x >> 63 else x for x in w] for w in split], dtype=torch.int64).reshape(len(rows), words)


def tree_rows(n, rng):
    rows = [1][:n]
    for i in range(1, n):
        rows.append(rows[rng.randint(max(0, i - 5), i - 1)] | 1 << i)
    return rows


class Setup:
    """A cache whose sequences have the given lengths, pages anywhere in the pool and NaN wherever no row is, with new rows as views of one
    q | k | v buffer."""

    def __init__(self, dtype, Hq, Hkv, hd, ps, lens, nodes, *, layers=1, spare=4, seed=1, behind=0, garbage=True, summaries=False):
        rng, gen = random.Random(seed), torch.Generator().manual_seed(seed)
        self.lens, self.nodes, self.hd, self.Hq, self.Hkv = lens, nodes, hd, Hq, Hkv
        pages = [-(-n // ps) for n in lens]
        n_pages, max_pages = sum(pages) + spare, max(pages) + 3
        ids = list(range(n_pages))
        rng.shuffle(ids)
        self.table = torch.full((len(lens), max_pages), -1, dtype=torch.int32)
        self.refs = torch.zeros(n_pages, dtype=torch.int32)
        shape = (layers, n_pages, Hkv, ps, hd)
        self.k, self.v = (torch.randn(shape, generator=gen).to(dtype) for _ in range(2))
        valid, at = torch.zeros((n_pages, ps), dtype=torch.bool), 0
        for s, n in enumerate(pages):
            for j in range(n):
                self.table[s, j] = ids[at]
                self.refs[ids[at]] = 1
                valid[ids[at], :min(ps, lens[s] - j * ps)] = True
                at += 1
        if garbage:
            for t in (self.k, self.v):
                t.masked_fill_(~valid[None, :, None, :, None], math.nan)
        self.len = torch.tensor(lens, dtype=torch.int32)
        self.start = [0]
        for n in nodes:
            self.start.append(self.start[-1] + n)
        self.T = self.start[-1] + behind
        self.qkv = torch.randn((layers, self.T, Hq + 2 * Hkv, hd), generator=gen).to(dtype)
        self.summary = torch.zeros((layers, n_pages, Hkv, 2, hd), dtype=dtype) if summaries else None
        self.rng = rng

    def plain(self):
        return PlainCache(self.k, self.v, self.refs, self.table, self.len, self.summary)

    def rows(self, layer, dev="cpu"):
        x = self.qkv.to(dev)[layer]
        return x[:, :self.Hq], x[:, self.Hq:self.Hq + self.Hkv], x[:, self.Hq + self.Hkv:]

    def all_rows(self, dev="cpu"):
        x = self.qkv.to(dev)
        return x[:, :, self.Hq:self.Hq + self.Hkv], x[:, :, self.Hq + self.Hkv:]

    def tree(self):
        return [r for n in self.nodes for r in tree_rows(n, self.rng)] + [0] * (self.T - self.start[-1])
