"""The planner with pages that several requests hold, and their reordering, on the host (test infrastructure)."""
import numpy as np

from tests.cache_ref import Plan


class SharedPlan(Plan):
    """Lists of pages per request; `key` [positions] per request says which token's K and V stands where."""

    def __init__(self, batch, max_pages, n_pages, page):
        super().__init__(batch, max_pages, n_pages, page)
        self.refs = np.zeros(n_pages, np.int64)
        self.moves = []

    def held(self, b):
        return [int(x) for x in self.table[b, :-(-int(self.len[b]) // self.page)]]

    def _drop(self, rows):
        """The rows' pages lose a holder each; those without one go onto the stack, each at the first row that had it."""
        for b in rows:
            for p in self.held(b):
                self.refs[p] -= 1
        there = set(self.free)
        for b in rows:
            for p in self.held(b):
                if self.refs[p] == 0 and p not in there:
                    there.add(p)
                    self.free.append(p)

    def step(self, start, count, rows, reset=False):
        P = self.page
        if reset:
            self.len[:] = 0
            self.free = list(range(self.n_pages - 1, -1, -1))
            self.refs[:] = 0
        gone = [b for b in range(self.B) if count[b] < 0]
        if not reset:
            self._drop(gone)
        self.len[gone] = 0
        status, shared = np.zeros(self.B, np.int64), np.zeros(self.B, bool)
        asked = np.maximum(np.asarray(count), 0)
        for b in range(self.B):
            s, c = int(start[b]), int(asked[b])
            if c > 0 and 0 <= s <= self.len[b] and s + c <= self.max_pages * P:
                shared[b] = any(self.refs[p] > 1 for p in self.held(b)[s // P:-(-(s + c) // P)])
        before = [self.held(b) for b in range(self.B)]
        out = super().step(start, np.where(shared, 0, asked), rows)
        for b in range(self.B):
            for p in self.held(b)[len(before[b]):]:
                self.refs[p] = 1
        out["status"] = np.where(shared, -5, out["status"])
        return out

    def reorder(self, parent):
        P = self.page
        status = np.zeros(self.B, np.int64)
        par = [int(x) for x in parent]
        for b in range(self.B):
            if not -1 <= par[b] < self.B:
                par[b], status[b] = b, -1
        old, n = [self.held(b) for b in range(self.B)], self.len.copy()
        seen, wants = set(), []
        for b in range(self.B):
            if par[b] >= 0:
                if par[b] in seen and n[par[b]] % P:
                    wants.append(b)
                seen.add(par[b])
        self._drop([b for b in range(self.B) if b not in seen])
        new = [list(old[par[b]]) if par[b] >= 0 else [] for b in range(self.B)]
        self.len = np.array([n[par[b]] if par[b] >= 0 else 0 for b in range(self.B)])
        self.moves = []
        for b in wants:
            if not self.free:
                status[b], new[b], self.len[b] = -3, [], 0
                continue
            dst = self.free.pop()
            self.moves.append((new[b][-1], dst, -(-(int(n[par[b]]) % P) // 32)))
            new[b][-1] = dst
        self.refs[:] = 0
        for b in range(self.B):
            for i, p in enumerate(new[b]):
                self.table[b, i] = p
                self.refs[p] += 1
        return status
