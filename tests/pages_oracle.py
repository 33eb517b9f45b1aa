"""The page pool as lists: a row is the list of its pages, holders are counted when they are asked for (with those that the caller
keeps outside the table)."""
import torch


class Pages:
    def __init__(self, batch, width, pages, page, caches=(), outside=None):
        self.rows = [[] for _ in range(batch)]
        self.width, self.pages, self.page = width, pages, page
        self.caches = [c.cpu().clone() for c in caches]
        self.outside = outside or {}

    def refs(self):
        n = [self.outside.get(p, 0) for p in range(self.pages)]
        for r in self.rows:
            for p in r:
                n[p] += 1
        return n

    def fork(self, parents, lens):
        old = self.rows
        self.rows = [old[b] if p == b else [] if p < 0 else old[p][:-(-lens[p] // self.page)] for b, p in enumerate(parents)]
        return [0 if p < 0 else lens[p] for p in parents]

    def reserve(self, lens, new):
        """True, or False where the pool had too few pages."""
        page, cap = self.page, self.page * self.width
        lens = [min(max(x, 0), cap) for x in lens]
        upto = [-(-min(x + max(n, 0), cap) // page) for x, n in zip(lens, new)]
        writes = [min(x + max(n, 0), cap) > x for x, n in zip(lens, new)]
        self.rows = [r[:c] for r, c in zip(self.rows, upto)]
        n = self.refs()
        free = [p for p in range(self.pages) if n[p] == 0]
        writers = {}
        for b, r in enumerate(self.rows):
            if writes[b] and lens[b] % page and lens[b] // page < len(r):
                writers.setdefault(r[lens[b] // page], []).append(b)
        rows, moves = [], []
        for b, r in enumerate(self.rows):
            out = list(r[:lens[b] // page])
            for c in range(len(out), max(len(r), upto[b])):             # (pages that its tokens should have and that it lacks are new ones, too)
                used = lens[b] % page if c == lens[b] // page else 0
                if c < len(r):
                    p = r[c]
                    alone = n[p] <= 1
                    if used and not alone:
                        alone = not writes[b] or (len(writers[p]) == n[p] and writers[p][0] == b)
                    if alone:
                        out.append(p)
                        continue
                    if used:
                        moves.append((p, len(out), used, b))
                out.append(None)
            rows.append(out)
        if sum(p is None for r in rows for p in r) > len(free):
            return False
        it = iter(free)
        for r in rows:
            for c, p in enumerate(r):
                if p is None:
                    r[c] = next(it)
        for src, c, used, b in moves:
            for cache in self.caches:
                cache[rows[b][c], :, :used] = cache[src, :, :used]
        self.rows = rows
        return True

    def compact(self):
        n = self.refs()
        live = [p for p in range(self.pages) if n[p]]
        to = dict(zip([p for p in live if p >= len(live)], [p for p in range(len(live)) if n[p] == 0]))
        for c in self.caches:
            for p, d in to.items():
                c[d] = c[p]
        self.rows = [[to.get(p, p) for p in r] for r in self.rows]
        self.outside = {to.get(p, p): k for p, k in self.outside.items()}
        return [to.get(p, p) for p in range(self.pages)]

    def check(self, pool, caches=()):
        refs = self.refs()
        assert pool.page_table.tolist() == [r + [-1] * (self.width - len(r)) for r in self.rows]
        assert pool.held.tolist() == [len(r) for r in self.rows]
        assert pool.refs.tolist() == refs and pool.free.item() == refs.count(0)
        for mine, theirs in zip(self.caches, caches):
            assert torch.equal(mine, theirs.cpu())
