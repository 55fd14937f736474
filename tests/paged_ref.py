"""A paged cache on the host, written from include/kvmix.h's statement: bookkeeping in plain loops, records and attention by the oracle,
one sequence at a time."""
import numpy as np

from oracle.kvmix_ref import RefCache

EXHAUSTED, BAD_ROW, BAD_ID, OCCUPIED = 1, 2, 4, 8


def tiles_of(n, W):
    return 0 if n < W + 32 else (n - W) // 32


class PagedRef:
    def __init__(self, n_slots, n_pages, max_tiles, window):
        self.n_slots, self.n_pages, self.max_tiles, self.W = n_slots, n_pages, max_tiles, window
        self.table = np.zeros((n_slots, max_tiles), np.int32)
        self.lens, self.grown = np.zeros(n_slots, np.int32), np.zeros(n_slots, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        self.status = 0

    @property
    def used(self):
        words = np.zeros((self.n_pages + 31) // 32, np.uint32)
        for p in np.flatnonzero(self.refs > 0):
            words[p // 32] |= np.uint32(1) << np.uint32(p % 32)
        return words

    def grow(self, rows, fresh):
        free = int((self.refs == 0).sum())
        wanted = 0
        for i, (r, n) in enumerate(zip(rows, fresh)):
            if r < 0:
                continue
            if r >= self.n_slots or r in rows[:i] or n < 0 or int(self.lens[r]) + n > 0x7fffffff:
                self.status |= BAD_ROW
                continue
            a, b = tiles_of(int(self.lens[r]), self.W), tiles_of(int(self.lens[r]) + n, self.W)
            if b > self.max_tiles:
                self.status |= EXHAUSTED
                self.grown[r] = 0
                continue
            wanted += b - a
            if b > a and wanted > free:
                self.status |= EXHAUSTED
                self.grown[r] = 0
                continue
            for t in range(a, b):
                p = int(np.argmin(self.refs))
                self.table[r, t] = p
                self.refs[p] = 1
            self.lens[r] += n
            self.grown[r] = n

    def free(self, rows):
        for r in rows:
            if r < 0:
                continue
            if r >= self.n_slots:
                self.status |= BAD_ROW
                continue
            for t in range(tiles_of(int(self.lens[r]), self.W)):
                self.refs[self.table[r, t]] -= 1
            self.lens[r] = self.grown[r] = 0

    def fork(self, src, dst):
        pairs = [(s, d) for s, d in zip(src, dst) if s >= 0 and d >= 0]
        for s, d in pairs:
            if s >= self.n_slots or d >= self.n_slots:
                self.status |= BAD_ROW
            elif self.lens[d] != 0 or [x for _, x in pairs].count(d) > 1 or s in [x for _, x in pairs] or d in [x for x, _ in pairs]:
                self.status |= OCCUPIED
            else:
                for t in range(tiles_of(int(self.lens[s]), self.W)):
                    self.table[d, t] = self.table[s, t]
                    self.refs[self.table[s, t]] += 1
                self.lens[d], self.grown[d] = self.lens[s], 0

    def compact(self):
        """-> [(source, destination)]"""
        live = int((self.refs > 0).sum())
        src = [p for p in range(live, self.n_pages) if self.refs[p] > 0]
        dst = [p for p in range(live) if self.refs[p] == 0]
        to = dict(zip(src, dst))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        for r in range(self.n_slots):
            for t in range(tiles_of(int(self.lens[r]), self.W)):
                self.table[r, t] = to.get(int(self.table[r, t]), self.table[r, t])
        return list(to.items())


def one_sequence(k, v, kb, vb, W, G=1):
    """The oracle's cache of one sequence: k, v fp16 [Hkv][n][128]."""
    Hkv, n, _ = k.shape
    T = tiles_of(n, W)
    rc = RefCache(1, G * Hkv, Hkv, kb, vb, W, max(32, 32 * T), (W + 95) // 32 * 32)
    bits = lambda x: np.ascontiguousarray(x)[None].view(np.uint16)
    if T:
        assert rc.quantize_pack(bits(k[:, :32 * T]), bits(v[:, :32 * T])) == 0
    rc.set_window(bits(k[:, 32 * T:]), bits(v[:, 32 * T:]))
    return rc
