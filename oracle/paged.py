"""A paged key-value cache and the attention of one new token over it, in plain Python and float64.

Written from the definitions alone: a sequence's token j lies in slot j % page of page table[seq][j // page]; pages are taken
lowest first; compaction sends the k-th page in use at or behind the number in use to the k-th free page before it."""
import numpy as np

OK, FULL, BAD = 0, 1, 2


class PagedMap:
    """page_ref, page_table and seq_len, and the pages' contents k, v [layers, pages, page, hkv, d] (any numpy arrays, changed in place)."""

    def __init__(self, page, ref, table, length, k=None, v=None):
        self.page, self.ref, self.table, self.length, self.k, self.v = page, ref, table, length, k, v

    def held(self, s):
        return -(-int(self.length[s]) // self.page)

    def _lowest(self, n):
        free = [p for p in range(len(self.ref)) if self.ref[p] == 0]
        return free[:n] if len(free) >= n else None

    def reserve(self, seqs, new):
        status, named, full = [], set(), False
        for s, x in zip(seqs, new):
            if s < 0:
                status.append(OK)
                continue
            if s >= len(self.length) or s in named or x < 0 or self.length[s] + x > self.table.shape[1] * self.page:
                named.add(s)
                status.append(BAD)
                continue
            named.add(s)
            need = -(-(int(self.length[s]) + int(x)) // self.page) - self.held(s)
            pages = None if full and need else self._lowest(need)
            if pages is None:
                full = True
                status.append(FULL)
                continue
            for k, p in enumerate(pages):
                self.table[s, self.held(s) + k] = p
                self.ref[p] = 1
            self.length[s] += x
            status.append(OK)
        return status

    def append(self, seqs, cu, k_new, v_new, status, layer=0):
        for i, s in enumerate(seqs):
            if s < 0 or s >= len(self.length) or status[i] != OK:
                continue
            n = int(cu[i + 1] - cu[i])
            for j in range(n):
                pos = int(self.length[s]) - n + j
                p = self.table[s, pos // self.page]
                self.k[layer, p, pos % self.page] = k_new[cu[i] + j]
                self.v[layer, p, pos % self.page] = v_new[cu[i] + j]

    def fork(self, src, dst):
        n_seqs, status, full = len(self.length), [], False
        pairs = [(a, b) for a, b in zip(src, dst) if 0 <= a < n_seqs and 0 <= b < n_seqs]
        targets, named, was = {b for _, b in pairs}, set(), self.length.copy()
        for a, b in zip(src, dst):
            if a < 0:
                status.append(OK)
                continue
            if not (0 <= a < n_seqs and 0 <= b < n_seqs):
                status.append(BAD)
                continue
            first = b not in named
            named.add(b)
            if not first or a in targets or was[b] != 0:
                status.append(BAD)
                continue
            whole, part = divmod(int(self.length[a]), self.page)
            pages = None if full and part else self._lowest(1 if part else 0)
            if pages is None:
                full = True
                status.append(FULL)
                continue
            for x in range(whole):
                self.table[b, x] = self.table[a, x]
                self.ref[self.table[a, x]] += 1
            if part:
                self.table[b, whole] = pages[0]
                self.ref[pages[0]] = 1
                for kv in (self.k, self.v):
                    kv[:, pages[0], :part] = kv[:, self.table[a, whole], :part]
            self.length[b] = self.length[a]
            status.append(OK)
        return status

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < len(self.length):
                for x in range(self.held(s)):
                    self.ref[self.table[s, x]] -= 1
                    self.table[s, x] = -1
                self.length[s] = 0

    def compact(self):
        used = int((self.ref > 0).sum())
        holes = [p for p in range(used) if self.ref[p] == 0]
        high = [p for p in range(used, len(self.ref)) if self.ref[p] > 0]
        to = dict(zip(high, holes))
        for p, q in to.items():
            for kv in (self.k, self.v):
                kv[:, q] = kv[:, p]
            self.ref[q], self.ref[p] = self.ref[p], 0
        for s in range(len(self.length)):
            for x in range(self.held(s)):
                self.table[s, x] = to.get(int(self.table[s, x]), int(self.table[s, x]))
        return [used, len(high)]


def seen_keys(length, window, sink):
    """Positions that the token at length - 1 sees."""
    j = np.arange(length)
    return j if window == 0 else j[(length - 1 - j < window) | (j < sink)]


def attend(q, k, v, scale):
    """q [hq, d] over k, v [keys, hkv, d] in float64: (out [hq, d], lse [hq], mean of |v| under the weights [hq, d], largest scale * sum |q k| [hq])."""
    hq, d = q.shape
    group = hq // k.shape[1]
    out, lse, mean, size = np.zeros((hq, d)), np.full(hq, -np.inf), np.zeros((hq, d)), np.zeros(hq)
    if not len(k):
        return out, lse, mean, size
    for h in range(hq):
        kh, vh = k[:, h // group], v[:, h // group]
        s = kh @ q[h] * scale
        w = np.exp(s - s.max())
        out[h], mean[h] = w @ vh / w.sum(), w @ np.abs(vh) / w.sum()
        lse[h] = s.max() + np.log(w.sum())
        size[h] = (np.abs(kh) @ np.abs(q[h])).max() * scale
    return out, lse, mean, size
