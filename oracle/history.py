"""Float64 oracle of attention over a request's own history, and the cache of
pages as plain Python lists.

`attention` evaluates the definition request by request and head by head; beside
the result it gives what a rounding analysis of an implementation needs: the
mean weight of |v| (a relative error e of every softmax weight moves an output
by at most 2 e times it) and a bound on the scores' own error in fp32.
`Cache` keeps each page's rows as a list and does every page operator row by row.
"""

import numpy as np

U32 = 2.0 ** -24
CAP_TURN = 128.0      # up to this cap its error may be relative to the cap, beyond it to the score


def attention(q, k, v, q_len, kv_len, *, causal=True, prefix=None, q_docs=None, kv_docs=None,
              slopes=None, cap=0.0, scale=None):
    """q [N, H, d], k / v [L, H_kv, d] (float64), lengths per request. Returns (out, weight of
    |v|, error bound of a row's scores) with shapes [N, H, d], [N, H, d], [N, H]."""
    n, h, d = q.shape
    hk = k.shape[1]
    scale = 1.0 / np.sqrt(d) if not scale else scale
    out, mean, err = np.zeros((n, h, d)), np.zeros((n, h, d)), np.zeros((n, h))
    qa = ka = 0
    for r, (nq, nk) in enumerate(zip(q_len, kv_len)):
        pos = nk - nq + np.arange(nq)[:, None]
        j = np.arange(nk)[None, :]
        seen = np.ones((nq, nk), bool)
        if causal:
            seen = j <= pos
            if prefix is not None:
                seen = seen | (j < prefix[r])
        if q_docs is not None:
            seen = seen & (q_docs[qa:qa + nq, None] == kv_docs[None, ka:ka + nk])
        for head in range(h):
            kh, vh = k[ka:ka + nk, head * hk // h], v[ka:ka + nk, head * hk // h]
            qh = q[qa:qa + nq, head]
            s = qh @ kh.T * scale
            e = (d + 8) * U32 * (np.abs(qh) @ np.abs(kh).T) * abs(scale)
            if cap > 0:
                s = cap * np.tanh(s / cap)
                e = e + 32 * U32 * np.maximum(np.abs(s), min(cap, CAP_TURN))
            if slopes is not None:
                away = slopes[head] * np.abs(pos - j)
                e = e + 4 * U32 * (np.abs(s) + away)
                s = s - away
            e = e + 8 * U32 * np.abs(s)
            for i in range(nq):
                on = np.flatnonzero(seen[i])
                if on.size == 0:
                    continue
                x = s[i, on]
                p = np.exp(x - x.max())
                p /= p.sum()
                out[qa + i, head] = p @ vh[on]
                mean[qa + i, head] = p @ np.abs(vh[on])
                err[qa + i, head] = e[i, on].max()
        qa += nq
        ka += nk
    return out, mean, err


class Cache:
    """Page tables, lengths, reference counts and page contents [layer][page][row]."""

    def __init__(self, layers, pages, page, slots, width):
        self.page, self.width = page, width
        self.table = [[-1] * width for _ in range(slots)]
        self.lens = [0] * slots
        self.refs = [0] * pages
        self.pool = [[[None] * page for _ in range(pages)] for _ in range(layers)]

    def _free(self):
        return [p for p, c in enumerate(self.refs) if c == 0]

    def reserve(self, slots, counts):
        """(rows, status): the pool row of every new row."""
        total = sum(counts)
        if (any(not 0 <= s < len(self.lens) or self.lens[s] < 0 for s in slots)
                or len(set(slots)) < len(slots)):
            return [-1] * total, (3, 0)
        want = [-(-(self.lens[s] + c) // self.page) for s, c in zip(slots, counts)]
        if any(w > self.width for w in want):
            return [-1] * total, (2, 0)
        have = [-(-self.lens[s] // self.page) for s in slots]
        free, need = self._free(), sum(want) - sum(have)
        if need > len(free):
            return [-1] * total, (1, need - len(free))
        rows = []
        for s, c, w, h in zip(slots, counts, want, have):
            for col in range(h, w):
                p = free.pop(0)
                self.table[s][col], self.refs[p] = p, 1
            for at in range(self.lens[s], self.lens[s] + c):
                rows.append(self.table[s][at // self.page] * self.page + at % self.page)
            self.lens[s] += c
        return rows, (0, 0)

    def write(self, layer, rows, values):
        for r, x in zip(rows, values):
            if 0 <= r < len(self.refs) * self.page:
                self.pool[layer][r // self.page][r % self.page] = x

    def fork(self, parents, children):
        n = len(self.lens)
        if (any(not 0 <= s < n for s in list(parents) + list(children))
                or len(set(children)) < len(children) or set(children) & set(parents)
                or any(self.lens[c] for c in children)
                or any(not 0 <= self.lens[a] <= self.width * self.page for a in parents)):
            return 3, 0
        need = sum(self.lens[a] % self.page != 0 for a in parents)
        free = self._free()
        if need > len(free):
            return 1, need - len(free)
        for a, c in zip(parents, children):
            full, rest = divmod(self.lens[a], self.page)
            for col in range(full):
                self.table[c][col] = self.table[a][col]
                self.refs[self.table[a][col]] += 1
            if rest:
                p = free.pop(0)
                self.table[c][full], self.refs[p] = p, 1
                for layer in self.pool:
                    layer[p][:rest] = layer[self.table[a][full]][:rest]
            self.lens[c] = self.lens[a]
        return 0, 0

    def free(self, slots):
        for s in slots:
            if 0 <= s < len(self.lens):
                for p in self.table[s][:-(-self.lens[s] // self.page)]:
                    self.refs[p] -= 1
                self.table[s] = [-1] * self.width
                self.lens[s] = 0

    def compact(self):
        n = sum(c > 0 for c in self.refs)
        holes = [p for p in range(n) if self.refs[p] == 0]
        movers = [p for p in range(n, len(self.refs)) if self.refs[p] > 0]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
            for layer in self.pool:
                layer[b] = list(layer[a])
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return 0, n

    def history(self, layer, slot):
        """The rows of a slot, in order."""
        return [self.pool[layer][self.table[slot][i // self.page]][i % self.page]
                for i in range(self.lens[slot])]
