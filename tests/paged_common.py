"""Helpers of the paged cache's GPU tests: sequences kept on the host next to the device's state."""
import numpy as np

import kvmix_synth as synth
from gpu_common import assert_attn_close, t16
from paged_ref import PagedRef, one_sequence, tiles_of

DEAD = 0x7E01      # an fp16 NaN: what slots and pages without tokens hold


class Serving:
    """One layer and its pages on the device, and on the host what they have to hold."""

    def __init__(self, Hkv, G, bits, W, n_slots, n_pages, max_tiles, W_cap=None, seed=0):
        import torch
        import paper_2506_08018_amd as kv
        self.kv, self.Hkv, self.G, self.W = kv, Hkv, G, W
        self.kb, self.vb = bits
        self.cfg = kv.LayerCfg(self.kb, self.vb, W)
        self.pages = kv.Pages(n_slots, n_pages, max_tiles, W)
        self.cache = kv.PagedCache(self.shape(1), self.cfg, n_pages, n_slots, W_cap or W + 32)
        for ring in (self.cache.k_win, self.cache.v_win):
            ring.view(torch.int16).fill_(DEAD)
        self.cache.pool.fill_(DEAD << 16 | DEAD)
        self.pages.table.fill_(0x7FFFFFFF)               # an id that no pool has: must not be followed
        self.ref = PagedRef(n_slots, n_pages, max_tiles, W)
        self.ref.table[:] = 0x7FFFFFFF
        self.k = [np.zeros((Hkv, 0, 128), np.float16) for _ in range(n_slots)]
        self.v = list(self.k)
        self.rng = np.random.default_rng([synth.BASE_SEED, seed])

    def shape(self, B):
        return self.kv.Shape(B, self.G * self.Hkv, self.Hkv)

    def ints(self, x):
        import torch
        return torch.tensor(list(x), dtype=torch.int32, device="cuda")

    def draw(self, n):
        k = self.rng.standard_normal((self.Hkv, n, 128), dtype=np.float32)
        k[:, :, 7] *= 10
        return k.astype(np.float16), self.rng.standard_normal((self.Hkv, n, 128), dtype=np.float32).astype(np.float16)

    def grow(self, rows, fresh):
        cu = np.concatenate([[0], np.cumsum(fresh)])
        self.kv.pages_grow(self.pages, self.ints(rows), self.ints(cu))
        self.ref.grow(list(rows), list(fresh))

    def append(self, rows, fresh, cu=True, max_new=None):
        """New tokens for the rows (room made before): as one call takes them, side by side, the Values out of wider rows."""
        import torch
        new = [self.draw(n) for n in fresh]
        for r, n, (k, v) in zip(rows, fresh, new):
            if r >= 0 and r < self.ref.n_slots and self.ref.grown[r] == n and n:
                self.k[r], self.v[r] = np.concatenate([self.k[r], k], 1), np.concatenate([self.v[r], v], 1)
        if sum(fresh) == 0:
            return
        k = torch.from_numpy(np.concatenate([x[0] for x in new], 1)).cuda().transpose(0, 1)                 # [tokens][Hkv][128], strided
        wide = torch.zeros((sum(fresh), 2 * self.Hkv, 128), dtype=torch.float16, device="cuda")
        wide[:, self.Hkv:] = torch.from_numpy(np.concatenate([x[1] for x in new], 1)).cuda().transpose(0, 1)
        self.kv.paged_append(self.shape(len(rows)), self.cfg, k, wide[:, self.Hkv:], self.cache, self.pages, rows=self.ints(rows),
                             cu=self.ints(np.concatenate([[0], np.cumsum(fresh)])) if cu else None, max_new=max_new or max(fresh))

    def step(self, rows, fresh):
        self.grow(rows, fresh)
        self.append(rows, fresh)

    def check_pages(self, what=""):
        p = self.pages
        got = {n: getattr(p, n).cpu().numpy() for n in ("table", "lens", "grown", "refs", "used", "status")}
        for n in ("table", "lens", "grown", "refs"):
            assert np.array_equal(got[n].reshape(getattr(self.ref, n).shape), getattr(self.ref, n)), (what, n)
        assert np.array_equal(got["used"].view(np.uint32), self.ref.used), (what, "used")
        assert got["status"][0] == self.ref.status, (what, got["status"][0], self.ref.status)

    def check_cache(self, what=""):
        """Records of every live page and every live ring row bit for bit; everything else as it was filled."""
        pool = self.cache.pool.cpu().numpy().view(np.uint32)
        rings = [t16(w) for w in (self.cache.k_win, self.cache.v_win)]
        W_cap = self.cache.W_cap
        seen = set()
        for s in range(self.ref.n_slots):
            n = int(self.ref.lens[s])
            assert n == self.k[s].shape[1], (what, s, n, self.k[s].shape)
            T = tiles_of(n, self.W)
            rc = one_sequence(self.k[s], self.v[s], self.kb, self.vb, self.W)
            for t in range(T):
                page = int(self.ref.table[s, t])
                assert np.array_equal(pool[page], rc.packed[:, t]), (what, "slot", s, "tile", t, "page", page)
                seen.add(page)
            live = np.arange(32 * T, n)
            for ring, x in zip(rings, (self.k[s], self.v[s])):
                assert np.array_equal(ring[s][:, live % W_cap], x[:, live].view(np.uint16)), (what, "ring of slot", s)
        return pool, seen

    def attend(self, rows, max_len=0, ws=None, scale=0.0):
        """-> (out bits, q, out tensor): q drawn, out filled with a pattern first."""
        import torch
        B = len(rows)
        q = self.rng.standard_normal((B, self.G * self.Hkv, 128), dtype=np.float32).astype(np.float16)
        out = torch.full((B, self.G * self.Hkv, 128), 7.0, dtype=torch.float16, device="cuda")
        longest = max_len or self.pages.max_tiles * 32 + self.W + 31
        if ws is None:
            ws = torch.zeros(self.kv.paged_workspace_bytes(self.shape(B), longest), dtype=torch.uint8, device="cuda")
        self.kv.paged_decode_attn(self.shape(B), self.cfg, torch.from_numpy(q).cuda(), self.cache, self.pages, out, ws, rows=self.ints(rows),
                                  max_len=max_len, softmax_scale=scale)
        torch.cuda.synchronize()
        return t16(out), q

    def check_attention(self, rows, what="", max_len=0, ws=None, scale=0.0):
        got, q = self.attend(rows, max_len, ws, scale)
        for b, s in enumerate(rows):
            if s < 0:
                assert (got[b].view(np.float16) == 7.0).all(), (what, "padding row", b)
            elif self.ref.lens[s] == 0:
                assert (got[b] == 0).all(), (what, "row without tokens", b)
            else:
                st, want = one_sequence(self.k[s], self.v[s], self.kb, self.vb, self.W, self.G).decode_attn(q[b:b + 1].view(np.uint16), scale)
                assert st == 0
                assert_attn_close(got[b:b + 1], want, f"{what} row {b} slot {s} of {self.ref.lens[s]} tokens", tight=True)
