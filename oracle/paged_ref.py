"""CPU oracle for a cache in pages and the attention that reads it (paper Sec. 4.2.2 / 4.3: the receiver's own tokens).

TEST INFRASTRUCTURE ONLY, like the rest of oracle/: the definitions written out, sequence by sequence and token by token, in float64 and Python
integers.

    attention   a query at place p of its sequence sees t <= p and, with a window, of those t > p - window and t < sinks:
                s_t = scale <q, K_t>, out = sum_t softmax(s)_t V_t, lse = log sum_t exp s_t; nothing seen: 0 and -inf
    pool        table [rows][row_pages], lens [rows], refs [pages]; pages are given out lowest first, in the order of the rows
"""
import numpy as np

BAD_PAGE, BAD_ROW, NO_PAGES = 0x10, 0x20, 0x40


def seen(place, length, window, sinks):
    """Tokens a query at `place` sees, of a sequence that holds `length`."""
    return [t for t in range(min(place + 1, length)) if window == 0 or t > place - window or t < sinks]


def attend(q, K, V, places, scale, window=0, sinks=0, absent=()):
    """q [n, Hq, D], K and V [H, T, D], places [n].  Returns out, lse, and what bounds of errors are made of: sum_t p_t |V_t| ([n, Hq, D]), the
    largest sum_i |q_i K_ti| scale of a seen token and the largest |s_t| ([n, Hq])."""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    n, Hq, D = q.shape
    H, T = K.shape[:2]
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    size, terms, top = np.zeros((n, Hq, D)), np.zeros((n, Hq)), np.zeros((n, Hq))
    for i in range(n):
        ts = [t for t in seen(int(places[i]), T, window, sinks) if t not in absent]
        if not ts:
            continue
        for hq in range(Hq):
            h = hq // (Hq // H)
            s = scale * (K[h, ts] @ q[i, hq])
            m = s.max()
            if m == -np.inf:
                continue
            p = np.exp(s - m)
            z = p.sum()
            lse[i, hq] = m + np.log(z)
            out[i, hq] = (p[:, None] * V[h, ts]).sum(axis=0) / z
            size[i, hq] = (p[:, None] * np.abs(V[h, ts])).sum(axis=0) / z
            terms[i, hq] = abs(scale) * (np.abs(K[h, ts]) @ np.abs(q[i, hq])).max()
            top[i, hq] = np.abs(s).max()
    return out, lse, size, terms, top


def joined(out, lse, other_out, other_lse):
    """Attention over two disjoint sets of tokens, from the results over each."""
    top = np.maximum(lse, other_lse)
    safe = np.where(np.isneginf(top), 0.0, top)
    a, b = np.exp(lse - safe), np.exp(other_lse - safe)
    both = np.where(a + b == 0, 1.0, a + b)
    return (out * a[..., None] + other_out * b[..., None]) / both[..., None], np.where(np.isneginf(top), -np.inf, safe + np.log(a + b + (a + b == 0)))


class Pool:
    """Tables, lengths and counts as lists of ints; pages [layers, pages, heads, size, dim] as numpy arrays of any type."""

    def __init__(self, table, lens, refs, k, v, size):
        self.table, self.lens, self.refs = [list(map(int, r)) for r in table], list(map(int, lens)), list(map(int, refs))
        self.k, self.v, self.size = k.copy(), v.copy(), size

    def _copy(self):
        return [list(r) for r in self.table], list(self.lens), list(self.refs)

    def _entries(self, length):
        return -(-length // self.size)

    def _free(self):
        return [i for i, r in enumerate(self.refs) if r <= 0]

    def reserve(self, more):
        most = len(self.table[0]) * self.size
        if any(m < 0 or n < 0 or n + m > most for n, m in zip(self.lens, more)):
            return BAD_ROW
        free, wants = self._free(), [self._entries(n + m) - self._entries(n) for n, m in zip(self.lens, more)]
        if sum(wants) > len(free):
            return NO_PAGES
        for b, w in enumerate(wants):
            for j in range(w):
                page = free.pop(0)
                self.table[b][self._entries(self.lens[b]) + j] = page
                self.refs[page] = 1
            self.lens[b] += more[b]
        return 0

    def append(self, k, v, starts, layer=0):
        """k, v [layers, tokens, heads, dim]."""
        status = 0
        for b in range(len(self.lens)):
            n = starts[b + 1] - starts[b]
            for i in range(n):
                place = self.lens[b] - n + i
                if place < 0 or place // self.size >= len(self.table[b]):
                    status |= BAD_ROW
                    continue
                page = self.table[b][place // self.size]
                if not 0 <= page < len(self.refs):
                    status |= BAD_PAGE
                    continue
                for l in range(k.shape[0]):
                    self.k[layer + l, page, :, place % self.size] = k[l, starts[b] + i]
                    self.v[layer + l, page, :, place % self.size] = v[l, starts[b] + i]
        return status

    def _count(self, row, by):
        for page in self.table[row][: self._entries(self.lens[row])]:
            if 0 <= page < len(self.refs):
                self.refs[page] += by

    def fork(self, source, target):
        rows = len(self.lens)
        if any(not 0 <= x < rows for x in list(source) + list(target)) or len(set(target)) < len(target) or set(source) & set(target):
            return BAD_ROW
        before, status = self._copy(), 0
        for t in target:
            self._count(t, -1)
        wants = sum(self.lens[s] % self.size != 0 for s in source)
        free = self._free()
        if wants > len(free):
            self.table, self.lens, self.refs = before
            return NO_PAGES
        for s, t in zip(source, target):
            full, part = divmod(self.lens[s], self.size)
            if part:
                page = free.pop(0)
                self.refs[page] = 1
                self.table[t][full] = page
                last = self.table[s][full]
                if 0 <= last < len(self.refs):
                    for pool in (self.k, self.v):
                        pool[:, page, :, :part] = pool[:, last, :, :part]
                else:
                    status |= BAD_PAGE
            self.table[t][:full] = self.table[s][:full]
            self.lens[t] = self.lens[s]
        for s, t in zip(source, target):
            for page in self.table[t][: self.lens[t] // self.size]:
                if 0 <= page < len(self.refs):
                    self.refs[page] += 1
        return status

    def free(self, rows, window=0, sinks=0):
        status = 0
        for b in rows:
            if not 0 <= b < len(self.lens):
                status |= BAD_ROW
                continue
            for j in range(self._entries(self.lens[b])):
                tokens = range(j * self.size, (j + 1) * self.size)
                if window and any(t > self.lens[b] - 1 - window or t < sinks for t in tokens):
                    continue
                page = self.table[b][j]
                self.table[b][j] = -1
                if 0 <= page < len(self.refs):
                    self.refs[page] -= 1
            if not window:
                self.lens[b] = 0
        return status

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [i for i in range(live) if self.refs[i] <= 0]
        movers = [i for i in range(live, len(self.refs)) if self.refs[i] > 0]
        goes = dict(zip(movers, holes))
        for a, b in goes.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
            for pool in (self.k, self.v):
                pool[:, b] = pool[:, a]
        for b, row in enumerate(self.table):
            for j in range(self._entries(self.lens[b])):
                row[j] = goes.get(row[j], row[j])
        return live
