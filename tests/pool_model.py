"""A pool of pages in plain Python and 64 bits: what the page_pool calls, the paged append and the paged attention are
compared with.  Written from the header's text; nothing of the library is used."""
import numpy as np


class Pool:
    """Table, lengths and reference counts as lists; every call answers whether it was taken."""

    def __init__(self, N, S, M, P):
        self.N, self.S, self.M, self.P = N, S, M, P
        self.table = [[-1] * M for _ in range(S)]
        self.len, self.refs = [0] * S, [0] * N

    def held(self, s):
        return -(-self.len[s] // self.P)

    def free_pages(self):
        return [i for i, n in enumerate(self.refs) if n == 0]

    def reserve(self, seq, want):
        if len(set(seq)) != len(seq) or any(not 0 <= s < self.S for s in seq) or any(w < 0 for w in want):
            return False
        if any(self.len[s] + w > self.M * self.P for s, w in zip(seq, want)):
            return False
        need = [-(-(self.len[s] + w) // self.P) - self.held(s) for s, w in zip(seq, want)]
        free = self.free_pages()
        if sum(need) > len(free):
            return False
        for s, w, n in zip(seq, want, need):
            for _ in range(n):
                page = free.pop(0)
                self.table[s][self.held(s) + self.table[s][self.held(s):].index(-1)] = page
                self.refs[page] = 1
            self.len[s] += w
        return True

    def fork(self, src, dst):
        """(taken, pairs, carries)"""
        none = [[-1, -1] for _ in src]
        if any(not 0 <= s < self.S for s in src + dst) or len(set(dst)) != len(dst) or set(src) & set(dst):
            return False, none, none
        free = self.free_pages()
        if any(self.len[d] for d in dst) or sum(self.len[s] % self.P > 0 for s in src) > len(free):
            return False, none, none
        pairs = []
        for s, d in zip(src, dst):
            full = self.len[s] // self.P
            for j in range(full):
                self.table[d][j] = self.table[s][j]
                self.refs[self.table[s][j]] += 1
            pair = [-1, -1]
            if self.len[s] % self.P:
                pair = [self.table[s][full], free.pop(0)]
                self.table[d][full] = pair[1]
                self.refs[pair[1]] = 1
            self.len[d] = self.len[s]
            pairs.append(pair)
        return True, pairs, [list(x) for x in zip(src, dst)]

    def free(self, seq):
        if len(set(seq)) != len(seq) or any(not 0 <= s < self.S for s in seq):
            return False
        for s in seq:
            for j in range(self.held(s)):
                self.refs[self.table[s][j]] -= 1
                self.table[s][j] = -1
            self.len[s] = 0
        return True

    def compact(self):
        live = [i for i, n in enumerate(self.refs) if n > 0]
        L = len(live)
        move = dict(zip([i for i in live if i >= L], [i for i in range(L) if self.refs[i] == 0]))
        self.table = [[move.get(x, x) for x in row] for row in self.table]
        for a, b in move.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        return [list(x) for x in move.items()]

    def share(self, seq, least):
        def common(a, b):
            if not (0 <= a < self.S and 0 <= b < self.S):
                return 0
            n = 0
            while n < min(self.len[a], self.len[b]) // self.P and self.table[a][n] == self.table[b][n]:
                n += 1
            return n

        runs, out = [], []
        for i, s in enumerate(seq):
            n = common(seq[i - 1], s) if i else 0
            if i and n >= least:
                runs[-1].append((i, n))
            else:
                runs.append([(i, None)])
        for run in runs:
            pages = min((n for _, n in run[1:]), default=0)
            out += [[run[0][0], len(run), pages]] * len(run)
        return out

    def rows(self, s, n=None):
        """Row numbers in the pool of the sequence's tokens."""
        return np.array([self.table[s][t // self.P] * self.P + t % self.P for t in range(self.len[s] if n is None else n)], dtype=np.int64)


def recurrence(state, x, g):
    """s = g s + (1 - g) x over x, g [T, ...] in 64 bits: every state, [T, ...]."""
    out, s = np.zeros(x.shape), np.asarray(state, dtype=np.float64)
    for t in range(x.shape[0]):
        s = g[t].astype(np.float64) * s + (1 - g[t].astype(np.float64)) * x[t].astype(np.float64)
        out[t] = s
    return out


def attention(q, k, v, last, scale):
    """Rows q [n, D] over keys k, v [T, D]; row i sees positions 0 .. last[i].  (out, lse, weighted magnitudes of v, largest sum of
    magnitudes of a score's terms), in 64 bits; what a row does not see counts for nothing, whatever it holds."""
    n, D = q.shape
    out, lse, mag, big = np.zeros((n, D)), np.full(n, -np.inf), np.zeros((n, D)), np.zeros(n)
    for i in range(n):
        if last[i] < 0:
            continue
        kk, vv, qq = k[:last[i] + 1].astype(np.float64), v[:last[i] + 1].astype(np.float64), q[i].astype(np.float64)
        z = scale * (kk @ qq)
        w = np.exp(z - z.max())
        lse[i] = z.max() + np.log(w.sum())
        w /= w.sum()
        out[i], mag[i], big[i] = w @ vv, w @ np.abs(vv), abs(scale) * (np.abs(kk) @ np.abs(qq)).max()
    return out, lse, mag, big
