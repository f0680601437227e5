"""The pages' calls, entry by entry in plain Python: what include/cdsl_ops.h defines."""
import numpy as np


class Pages:
    def __init__(self, table, refs, pool):
        self.table, self.refs, self.pool = table.copy(), refs.copy(), pool.copy()

    def is_page(self, x):
        return 0 <= x < len(self.refs)

    def _set(self, b, i, now):
        old = self.table[b, i]
        if self.is_page(old):
            self.refs[old] -= 1
        if self.is_page(now):
            self.refs[now] += 1
        self.table[b, i] = now

    def fork(self, parents):
        old = self.table.copy()
        B, P = old.shape
        for b in range(B):
            if parents[b] == b:
                continue
            for i in range(P):
                self._set(b, i, old[parents[b], i] if 0 <= parents[b] < B else -1)

    def free(self, lens):
        B, P = self.table.shape
        for b in range(B):
            for i in range(P):
                if 32 * i >= max(int(lens[b]), 0):
                    self._set(b, i, -1)

    def reserve(self, lens, count, most):
        B, P = self.table.shape
        run, got = [], np.zeros(B, np.int64)
        for b in range(B):
            L = max(int(lens[b]), 0)
            got[b] = n = min(max(int(count[b]), 0), most, max(0, 32 * P - L))
            run += [(b, i) for i in range(L // 32, -(-(L + n) // 32) if n else L // 32)]
        start = self.refs.copy()
        leavers = {}
        for b, i in run:
            p = self.table[b, i]
            if self.is_page(p) and start[p] > 1:
                leavers.setdefault(p, []).append((b, i))
        keeper = {p: at[0] for p, at in leavers.items() if len(at) == start[p]}
        free = [p for p in range(len(start)) if start[p] == 0]
        want, needs = {}, 0
        for b, i in run:
            p = self.table[b, i]
            held = self.is_page(p)
            if (not held or start[p] > 1) and keeper.get(p) != (b, i):
                want[b, i] = needs
                needs += 1
        last = {p: max(want.get(x, -1) for x in at) for p, at in leavers.items()}
        copies = []
        for b, i in run:
            p = self.table[b, i]
            L = max(int(lens[b]), 0)
            ok = True
            if (b, i) in want:
                ok = want[b, i] < len(free)
                if ok:
                    if self.is_page(p) and 32 * i < L:
                        copies.append((p, free[want[b, i]]))
                    self._set(b, i, free[want[b, i]])
            elif self.is_page(p) and keeper.get(p) == (b, i):
                ok = last[p] < len(free)
            if not ok:
                got[b] = min(got[b], max(0, 32 * i - L))
        before = self.pool.copy()
        for s, d in copies:
            self.pool[:, d] = before[:, s]
        return got

    def compact(self):
        used = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        U = len(used)
        holes = [p for p in range(U) if self.refs[p] <= 0]
        for d, s in zip(holes, [p for p in used[::-1] if p >= U]):
            self.pool[:, d] = self.pool[:, s]
            self.table[self.table == s] = d
            self.refs[d], self.refs[s] = self.refs[s], 0
        return U
