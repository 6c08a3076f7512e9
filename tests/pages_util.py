"""A pool of pages and its definition: forking and compacting step by step on lists."""
from __future__ import annotations

import numpy as np
import torch


def up(n, page):
    return -(-n // page)


def forked(table, held, refs, keep, room, parents, page):
    """(rows, refs, copies): rows as lists (shorter than the table: the rest is -1), copies as (from, to, tokens).  Everything well formed."""
    refs = list(refs)
    old = [list(r[:up(n, page)]) for r, n in zip(table, held)]
    for r in old:
        for p in r:
            refs[p] -= 1
    rows, partial = [], []
    for parent, n in zip(parents, keep):
        rows.append(old[parent][:n // page] if parent >= 0 else [])
        for p in rows[-1]:
            refs[p] += 1
        partial.append(old[parent][n // page] if parent >= 0 and n % page else None)
    kept = [False] * len(rows)
    for b, p in enumerate(partial):
        if p is not None and refs[p] <= 0 and p not in partial[:b]:
            kept[b] = True
    for b, p in enumerate(partial):
        if kept[b]:
            refs[p] = 1
            rows[b].append(p)
    free = [p for p, n in enumerate(refs) if n <= 0]
    copies = []
    for b, (parent, n, m) in enumerate(zip(parents, keep, room)):
        if parent < 0:
            continue
        while len(rows[b]) < up(max(n, m), page):
            p = free.pop(0) if free else -1
            if partial[b] is not None and not kept[b] and len(rows[b]) == n // page and p >= 0:
                copies.append((partial[b], p, n % page))
            if p >= 0:
                refs[p] = 1
            rows[b].append(p)
    return rows, refs, copies


def compacted(refs):
    """(place, refs, used)"""
    used = [p for p, n in enumerate(refs) if n > 0]
    n = len(used)
    holes = [p for p in range(n) if refs[p] <= 0]
    place, after = [-1] * len(refs), [0] * len(refs)
    for p in used:
        place[p] = p if p < n else holes.pop(0)
        after[place[p]] = refs[p]
    return place, after, n


class Pool:
    """Random rows over a pool: some share full pages, some pages are held from outside, entries behind a row's pages are -7."""

    def __init__(self, rows, most, page=16, spare=0.5, heads=2, dim=64, dtype=torch.bfloat16, token_major=False, shared=0.3, outside=0.1, seed=0,
                 wide=None, offset=0):
        r = np.random.default_rng(seed)
        self.page, self.rows = page, rows
        self.held = [int(x) for x in r.integers(0, most + 1, rows)]
        if rows:
            self.held[0] = most
        need = [up(n, page) for n in self.held]
        total = sum(need)
        out = int(total * outside)
        self.n_pages = max(1, int((total + out) * (1 + spare)) + 3)
        order = list(r.permutation(self.n_pages))
        self.refs = [0] * self.n_pages
        self.table = []
        for b in range(rows):
            row = []
            if b and r.random() < shared:                      # the first pages of an earlier row, full in both
                a = int(r.integers(0, b))
                row = self.table[a][:min(self.held[a] // page, self.held[b] // page) // 2]
            row = row + [int(order.pop()) for _ in range(need[b] - len(row))]
            for p in row:
                self.refs[p] += 1
            self.table.append(row)
        for _ in range(min(out, len(order))):
            self.refs[order.pop()] += 1
        self.prefix = [p for p, n in enumerate(self.refs) if n == 1][:5]
        wide = max(need + [1]) if wide is None else wide
        self.wide = wide
        shape = (self.n_pages, page, heads, dim) if token_major else (self.n_pages, heads, page, dim)
        g = torch.Generator().manual_seed(seed)
        self.k, self.v = (torch.randn((int(np.prod(shape)) + offset,), generator=g).to(dtype)[offset:].view(shape) for _ in range(2))
        if token_major:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)

    def padded(self, fill=-7):
        return [r + [fill] * (self.wide - len(r)) for r in self.table]


def ints(x, shape=None):
    t = torch.tensor(x, dtype=torch.int32, device="cuda")
    return t if shape is None else t.view(shape)


def on_gpu(x, offset=0):
    """a copy with the same strides, `offset` elements behind an aligned address"""
    n = sum((s - 1) * st for s, st in zip(x.shape, x.stride())) + 1
    buf = torch.zeros((n + offset,), dtype=x.dtype, device="cuda")[offset:]
    return torch.as_strided(buf, x.shape, x.stride(), buf.storage_offset()).copy_(x)
