"""The paged cache's rules as a plain model on numpy arrays: test infrastructure,
written from the calls' documentation, shares no code with the HIP path."""
from __future__ import annotations

import numpy as np

FULL, BAD_SLOT, TWICE, BAD_COUNT = 1, 2, 4, 8


class Model:
    """k, v: [layers][num_pages][page_size][...], ts [num_pages][page_size]."""

    def __init__(self, k, v, ts, slots, max_pages):
        self.k, self.v, self.ts = k, v, ts
        self.pages, self.P = k.shape[1], k.shape[2]
        self.slots, self.max_pages = slots, max_pages
        self.tables = np.full((slots, max_pages), -1, np.int32)
        self.lens = np.zeros(slots, np.int32)
        self.refs = np.zeros(self.pages, np.int32)
        self.status = 0

    def _blocks(self, n):
        return (int(n) + self.P - 1) // self.P

    def _named(self, s):
        return 0 <= s < self.slots

    def extend(self, slots, counts):
        refs0 = self.refs.copy()
        plans, seen = [], set()
        for s, cnt in zip(slots, counts):
            s, cnt = int(s), int(cnt)
            plan = None
            if not self._named(s):
                self.status |= BAD_SLOT
            elif s in seen:
                self.status |= TWICE
            elif cnt < 0:
                self.status |= BAD_COUNT
            elif self.lens[s] + cnt > self.max_pages * self.P:
                self.status |= FULL
            else:
                n = int(self.lens[s])
                need = self._blocks(n + cnt) - self._blocks(n)
                shared = -1
                if cnt > 0 and n % self.P:
                    last = int(self.tables[s, self._blocks(n) - 1])
                    if refs0[last] > 1:
                        shared, need = last, need + 1
                plan = (s, cnt, n, need, shared)
            seen.add(s)
            plans.append(plan)
        free = [p for p in range(self.pages) if refs0[p] == 0]
        start = np.full(len(plans), -1, np.int32)
        asked = 0
        for r, plan in enumerate(plans):
            if plan is None:
                continue
            s, cnt, n, need, shared = plan
            asked += need
            if need and asked > len(free):
                self.status |= FULL
                continue
            mine = free[asked - need:asked]
            at = self._blocks(n)
            if shared >= 0:
                at -= 1
                to, rows = mine[0], n % self.P
                self.k[:, to, :rows] = self.k[:, shared, :rows]
                self.v[:, to, :rows] = self.v[:, shared, :rows]
                if self.ts is not None:
                    self.ts[to, :rows] = self.ts[shared, :rows]
                self.refs[shared] -= 1
            for x, p in enumerate(mine):
                self.tables[s, at + x] = p
                self.refs[p] = 1
            self.lens[s] += cnt
            start[r] = n
        return start

    def write(self, layer, k, v, slots, start, off, ts=None):
        for r, s in enumerate(slots):
            if not self._named(int(s)) or start[r] < 0:
                continue
            for t in range(int(off[r]), int(off[r + 1])):
                pos = int(start[r]) + t - int(off[r])
                p, x = self.tables[s, pos // self.P], pos % self.P
                self.k[layer, p, x], self.v[layer, p, x] = k[t], v[t]
                if ts is not None:
                    self.ts[p, x] = ts[t]

    def _release(self, s):
        for x in range(self._blocks(self.lens[s])):
            self.refs[self.tables[s, x]] -= 1
        self.tables[s] = -1
        self.lens[s] = 0

    def fork(self, src, dst):
        old = self.tables.copy(), self.lens.copy()
        seen = set()
        todo = []
        for s, d in zip(map(int, src), map(int, dst)):
            none = not self._named(s) or not self._named(d)
            if none:
                self.status |= BAD_SLOT
            elif d in seen:
                self.status |= TWICE
            else:
                todo.append((s, d))
            seen.add(d)
        for _, d in todo:
            self._release(d)
        for s, d in todo:
            self.tables[d], self.lens[d] = old[0][s], old[1][s]
            for x in range(self._blocks(self.lens[d])):
                self.refs[self.tables[d, x]] += 1

    def free(self, slots):
        for s in map(int, slots):
            if not self._named(s):
                self.status |= BAD_SLOT
            else:
                self._release(s)

    def compact(self):
        live = int((self.refs > 0).sum())
        src = [p for p in range(live, self.pages) if self.refs[p] > 0]
        dst = [p for p in range(live) if self.refs[p] == 0]
        for s, d in zip(src, dst):
            self.k[:, d], self.v[:, d] = self.k[:, s], self.v[:, s]
            if self.ts is not None:
                self.ts[d] = self.ts[s]
            self.refs[d], self.refs[s] = self.refs[s], 0
            self.tables[self.tables == s] = d
        return live

    def history(self, s, layer=0):
        """k, v, ts of sequence s, in order."""
        x = np.arange(int(self.lens[s]))
        p = self.tables[s, x // self.P]
        return (self.k[layer, p, x % self.P], self.v[layer, p, x % self.P],
                None if self.ts is None else self.ts[p, x % self.P])

    def check(self):
        """What holds after every call."""
        count = np.zeros(self.pages, np.int64)
        for s in range(self.slots):
            n = self._blocks(self.lens[s])
            assert (self.tables[s, :n] >= 0).all() and (self.tables[s, n:] == -1).all()
            np.add.at(count, self.tables[s, :n], 1)
        assert (count == self.refs).all()
