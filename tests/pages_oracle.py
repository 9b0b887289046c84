"""A cache whose sequences share slots, kept sequence by sequence and block by block in NumPy: what the entry points for pages
have to leave behind, bit for bit."""
import numpy as np


class Book:
    """ctx [B], table [B][Hkv][mb], digest [B][Hkv][mb][...], pools [n_slots][2][S*d] of raw element bits, refs [n_slots]."""

    def __init__(self, S, ctx, table, digest, k_pool, v_pool):
        self.S, self.ctx, self.table, self.digest = S, ctx.copy(), table.copy(), digest.copy()
        self.k_pool, self.v_pool = k_pool.copy(), v_pool.copy()
        self.n_slots = len(k_pool)
        self.init()

    def blocks(self, b):
        return min((max(0, int(self.ctx[b])) + self.S - 1) // self.S, self.table.shape[2])

    def valid(self, e):
        return 0 <= e < self.n_slots

    def init(self):
        self.refs = np.zeros(self.n_slots, np.int32)
        for b in range(len(self.ctx)):
            self.table[b, :, self.blocks(b):] = -1
            for e in self.table[b].ravel():
                if self.valid(e):
                    self.refs[e] += 1

    def take(self, want):
        """The lowest free slots, None where none is left."""
        free = np.flatnonzero(self.refs == 0)[:want].tolist()
        self.refs[free] = 1
        return free + [None] * (want - len(free))

    def reserve(self, n=None):
        n = len(self.ctx) if n is None else n
        Hkv, mb = self.table.shape[1:]
        opens = [b for b in range(n) if 0 <= self.ctx[b] < mb * self.S and self.ctx[b] % self.S == 0]
        got = self.take(len(opens) * Hkv)
        new = np.full((n, Hkv), -1, np.int32)
        for i, b in enumerate(opens):
            new[b] = [-1 if s is None else s for s in got[i * Hkv:(i + 1) * Hkv]]
        return new, got.count(None)

    def fork(self, src, dst, deep):
        status, todo, wanted = [], [], 0
        for i, (a, b) in enumerate(zip(src, dst)):
            rows = range(len(self.ctx))
            ok = a in rows and b in rows and a != b and b not in src and b not in dst[:i] and self.ctx[b] <= 0
            status.append(0 if ok else -1)
            if not ok:
                continue
            nb, moves = self.blocks(a), []
            for g in range(self.table.shape[1]):
                for j in range(nb):
                    if self.valid(self.table[a, g, j]) and (deep or (j == nb - 1 and self.ctx[a] % self.S)):
                        moves.append((g, j))
            todo.append((i, a, b, nb, moves))
            wanted += len(moves)
        got = iter(self.take(wanted))
        for i, a, b, nb, moves in todo:
            moved = set(moves)
            self.table[b] = -1
            for g in range(self.table.shape[1]):
                for j in range(nb):
                    e = self.table[a, g, j]
                    if not self.valid(e):
                        continue
                    if (g, j) not in moved:
                        self.table[b, g, j] = e
                        self.refs[e] += 1
                        continue
                    slot = next(got)
                    if slot is None:
                        status[i] += 1
                        continue
                    self.table[b, g, j] = slot
                    self.k_pool[slot], self.v_pool[slot] = self.k_pool[e], self.v_pool[e]
            self.digest[b, :, :nb] = self.digest[a, :, :nb]
            self.ctx[b] = self.ctx[a]
        return np.array(status, np.int32)

    def free(self, seq):
        for b in dict.fromkeys(x for x in seq if 0 <= x < len(self.ctx)):
            for e in self.table[b].ravel():
                if self.valid(e) and self.refs[e] > 0:
                    self.refs[e] -= 1
            self.table[b], self.ctx[b] = -1, -1

    def compact(self):
        live = int((self.refs > 0).sum())
        holes = iter(np.flatnonzero(self.refs[:live] == 0).tolist())
        where = np.full(self.n_slots, -1, np.int32)
        for s in range(self.n_slots):
            if self.refs[s] > 0:
                where[s] = s if s < live else next(holes)
        for s in range(live, self.n_slots):
            if where[s] >= 0:
                self.k_pool[where[s]], self.v_pool[where[s]] = self.k_pool[s], self.v_pool[s]
                self.refs[where[s]], self.refs[s] = self.refs[s], 0
        named = (self.table >= 0) & (self.table < self.n_slots)
        self.table[named] = where[self.table[named]]
        return where, live
