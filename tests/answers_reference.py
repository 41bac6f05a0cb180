"""Plain references, in Python integers and binary64, of the calls for several answers of one prompt:
positions, shared blocks, and the table that attention over shared prefixes reads."""
import numpy as np
import torch


def norm_rotary(x, w, start, freq, pairs, eps):
    """x [sequence, token, head, value] -> (result, magnitude of what a value is made of), binary64."""
    y = x.detach().cpu().double().numpy().copy()
    if w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * w.detach().cpu().double().numpy()
    out, mag = y.copy(), np.abs(y)
    f = freq.detach().cpu().double().numpy()
    half = len(f)
    for b in range(y.shape[0]):
        for i in range(y.shape[1]):
            t = (int(start[b]) + i) * f
            for k in range(half):
                p, q = (2 * k, 2 * k + 1) if pairs else (k, k + half)
                a, c = y[b, i, :, p], y[b, i, :, q]
                out[b, i, :, p] = a * np.cos(t[k]) - c * np.sin(t[k])
                out[b, i, :, q] = c * np.cos(t[k]) + a * np.sin(t[k])
                mag[b, i, :, p] = mag[b, i, :, q] = np.abs(a) + np.abs(c)
    return out, mag


class PlainPages:
    """Table, counts and contents of a pool; contents as one array of bytes for each block."""

    def __init__(self, cache):
        self.table = cache.table.cpu().tolist()
        self.refs = cache.refs.cpu().tolist()
        self.T, self.n = cache.block_tokens, cache.k.shape[0]
        self.data = [self.bytes_of(cache, x) for x in range(self.n)]

    @staticmethod
    def bytes_of(cache, x):
        return tuple(t[x].cpu().contiguous().numpy().tobytes() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale))

    def names(self, x):
        return 0 <= x < self.n

    def fork(self, dst, src=None):
        rows = [list(r) for r in self.table]
        last = {d: i for i, d in enumerate(dst)}
        for d, i in last.items():
            if not 0 <= d < len(rows):
                continue
            s = -1 if src is None else src[i]
            new = rows[s] if 0 <= s < len(rows) else [-1] * len(rows[d])
            for was, now in zip(rows[d], new):
                if self.names(was):
                    self.refs[was] -= 1
                if self.names(now):
                    self.refs[now] += 1
            self.table[d] = list(new)

    def reserve(self, start, n_new, count=None):
        """(missing, free)"""
        asked = []
        for b, row in enumerate(self.table):
            n = n_new if count is None else min(count[b], n_new)
            if start[b] < 0 or n <= 0:
                continue
            for place in range(start[b] // self.T, (start[b] + n - 1) // self.T + 1):
                if place < len(row):
                    asked.append((b, place, row[place]))
        wants = []
        for i, (b, place, x) in enumerate(asked):
            if self.names(x):
                same = [j for j, r in enumerate(asked) if r[2] == x]
                if self.refs[x] <= 1 or (len(same) >= self.refs[x] and same[0] == i):
                    continue
            wants.append((b, place, x))
        free = [x for x in range(self.n) if self.refs[x] <= 0]
        if len(wants) > len(free):
            return len(wants) - len(free), len(free)
        for (b, place, x), new in zip(wants, free):
            self.table[b][place] = new
            self.refs[new] = 1
            if self.names(x):
                self.refs[x] -= 1
                if place * self.T < start[b]:
                    self.data[new] = self.data[x]
        return 0, len(free) - len(wants)

    def compact(self):
        live = [x for x in range(self.n) if self.refs[x] > 0]
        holes = [x for x in range(len(live)) if self.refs[x] <= 0]
        move = dict(zip([x for x in live if x >= len(live)], holes))
        for x, to in move.items():
            self.data[to], self.refs[to], self.refs[x] = self.data[x], self.refs[x], 0
        kept = set(live)
        self.table = [[(move.get(x, x) if x in kept else -1) if self.names(x) else x for x in row] for row in self.table]
        self.refs = [max(0, r) if x < len(live) else 0 for x, r in enumerate(self.refs)]
        return len(live)

    def check(self, cache, table=None, refs=None):
        assert (cache.table if table is None else table).cpu().tolist() == self.table
        assert (cache.refs if refs is None else refs).cpu().tolist() == self.refs
        for x in range(self.n):
            assert self.bytes_of(cache, x) == self.data[x], x


def shared_table(table, T, group_start, prefix, max_prefix, max_group):
    """The table that attention over shared prefixes reads."""
    out = table.copy()
    for g in range(len(prefix)):
        first = int(group_start[g])
        for b in range(first, min(int(group_start[g + 1]), first + max_group)):
            n = max(0, min(int(prefix[g]), max_prefix)) // T
            out[b, :n] = table[first, :n]
    return out
