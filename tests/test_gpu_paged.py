"""The paged cache on the GPU against the oracle, one sequence at a time: ragged appends, decode attention, and both as a serving program runs them."""
import numpy as np
import pytest

from gpu_common import assert_attn_close, t16
from paged_common import Serving
from paged_ref import BAD_ID, BAD_ROW, EXHAUSTED, one_sequence, tiles_of

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("bits,W,Hkv,W_cap", [((2, 2), 32, 2, 64), ((3, 4), 64, 1, 128), ((1, 1), 0, 3, 32), ((4, 3), 0, 1, 64), ((2, 4), 128, 8, 160),
                                              ((1, 3), 32, 2, 96), ((3, 3), 96, 2, 128), ((4, 4), 32, 1, 64)])
def test_ragged_append(bits, W, Hkv, W_cap):
    """Tokens in stretches of every kind (none, one, a tile's end, many tiles): records of all pages and all ring rows."""
    s = Serving(Hkv, 1, bits, W, n_slots=7, n_pages=150, max_tiles=40, W_cap=W_cap, seed=W + Hkv)
    rounds = [([5, 0, 3, 6], [1, 31, 32, 33]), ([0, 1, 5, 6, 3], [W, 500, 0, 64, 1]), ([2, 1, 4, 6], [W + 32, 1, W + 31, 97]),
              ([4], [1]), ([-1, 6, 4, -3], [5, 300, 31, 2])]
    for i, (rows, fresh) in enumerate(rounds):
        s.step(rows, fresh)
        s.check_pages(f"round {i}")
        s.check_cache(f"round {i}")
    for i in range(40):                                  # single tokens, some slot overflows on most steps
        s.grow(range(7), [1] * 7)
        s.append(range(7), [1] * 7, cu=False)
    s.check_pages("single tokens")
    pool, seen = s.check_cache("single tokens")
    untouched = [p for p in range(150) if p not in seen]
    assert (pool[untouched] == np.uint32(0x7E017E01)).all()


@pytest.mark.parametrize("bits", [(kb, vb) for kb in (1, 2, 3, 4) for vb in (1, 2, 3, 4)])
def test_append_of_every_width(bits):
    s = Serving(2, 1, bits, 32, n_slots=3, n_pages=60, max_tiles=30, seed=10 * bits[0] + bits[1])
    s.step([2, 0], [333, 70])
    s.step([0, 2], [1, 97])
    s.check_cache(str(bits))


@pytest.mark.parametrize("B,n,bits", [(9, 32 * 29, (2, 2)), (33, 32 * 9, (3, 4)), (40, 32 * 30, (2, 4)), (36, 32 * 16, (3, 2)), (70, 32 * 16 + 5, (2, 1))])
def test_append_of_many_tiles(B, n, bits):
    """Launches past 2048, 4096 and 8192 tiles, which run in other forms (sampled slots; the pages of all slots differ)."""
    s = Serving(8, 1, bits, 32, n_slots=B, n_pages=B * 32, max_tiles=32, seed=B)
    fresh = [n - (b * 37) % min(300, n) for b in range(B)]
    s.grow(range(B), fresh)
    s.append(range(B), fresh)
    keep = [0, 1, B // 2, B - 1]
    for b in range(B):
        if b not in keep:                                # nothing to compare: an empty sequence
            s.ref.lens[b] = 0
            s.k[b], s.v[b] = s.k[b][:, :0], s.v[b][:, :0]
    s.check_cache("many tiles")


@pytest.mark.parametrize("B,bits", [(65, (2, 2)), (200, (1, 3)), (4200, (2, 1))])
def test_append_of_many_rows(B, bits):
    """More rows than a wave looks over at once, and more than the square of that: which row a tile belongs to; a first offset that is not 0."""
    s = Serving(1, 1, bits, 0, n_slots=B, n_pages=4 * B, max_tiles=6, W_cap=64, seed=B)
    rows = [int(r) for r in s.rng.permutation(B)]
    for most in (70, 40):
        fresh = [int(n) for n in s.rng.integers(0, most, B)]
        for i in range(0, B, 4096):                            # (as many rows as a call of grow takes)
            s.grow(rows[i:i + 4096], fresh[i:i + 4096])
        s.append(rows, fresh)
    s.check_pages()
    s.ref.lens[:] *= np.arange(B) % (B // 50) == 0             # (fifty slots looked at)
    for b in range(B):
        if not s.ref.lens[b]:
            s.k[b], s.v[b] = s.k[b][:, :0], s.v[b][:, :0]
    s.check_cache("many rows")


def test_append_keeps_within_its_inputs():
    """Offsets that go past the inputs' tokens, or below none: nothing is read there, the rows are left alone."""
    import torch
    s = Serving(1, 1, (2, 2), 0, n_slots=4, n_pages=16, max_tiles=8, seed=8)
    s.grow([0, 1, 2], [32, 32, 32])
    k = torch.randn((64, 1, 128), device="cuda").half()
    pool = s.cache.pool.clone()
    for cu in ([40, 72, 104, 136], [-64, -32, 0, 32 + 64], [33, 65, 97, 129]):
        s.kv.paged_append(s.shape(3), s.cfg, k, k, s.cache, s.pages, rows=s.ints([0, 1, 2]), cu=s.ints(cu), max_new=32)
        assert torch.equal(s.cache.pool, pool) and int(s.pages.status[0]) == BAD_ROW
        s.pages.status.zero_()
    s.kv.paged_append(s.shape(3), s.cfg, k, k, s.cache, s.pages, rows=s.ints([0, 1, 2]), cu=s.ints([0, 32, 64, 96]), max_new=32)      # two of three
    changed = (s.cache.pool != pool).flatten(1).any(1).nonzero().view(-1).tolist()
    assert changed == [0, 1] and int(s.pages.status[0]) == BAD_ROW


def test_append_leaves_rows_alone_that_were_not_granted():
    s = Serving(1, 1, (2, 2), 32, n_slots=4, n_pages=4, max_tiles=8, seed=3)
    s.step([0, 1], [100, 40])                            # two pages of four
    s.grow([2, 0, 3], [200, 10, 90])                     # slot 2 wants 5, slot 0 none, slot 3 what then is not granted either
    assert s.ref.status == EXHAUSTED and list(s.ref.grown) == [10, 40, 0, 0]
    s.append([2, 0, 3], [200, 10, 90])
    s.check_pages()
    pool, seen = s.check_cache()
    assert len(seen) == 2 and (pool[[p for p in range(4) if p not in seen]] == np.uint32(0x7E017E01)).all()


def test_append_refuses_counts_that_disagree():
    """Another token count than the granted one, more than max_new, a slot out of range, a page id out of range: nothing is written for that row,
    the status says so, the other rows are done."""
    s = Serving(1, 1, (2, 2), 0, n_slots=4, n_pages=16, max_tiles=8, seed=4)
    s.step([0, 1, 2], [40, 40, 40])
    s.grow([0, 1, 2], [33, 5, 24])
    s.check_pages()
    before, pool = t16(s.cache.k_win), s.cache.pool.cpu().numpy()
    s.ref.grown[[0, 1]] = -1                             # (the host's model does not take these rows)
    s.append([0, 1, 2], [33, 4, 24], max_new=32)         # 33 > 32; 4 of the 5 that were granted
    assert int(s.pages.status[0]) == BAD_ROW
    after, pool2 = t16(s.cache.k_win), s.cache.pool.cpu().numpy()
    assert np.array_equal(before, after)                 # (slot 2's tokens are all packed)
    rc = one_sequence(s.k[2], s.v[2], 2, 2, 0)
    for t in range(2):
        assert np.array_equal(pool2[s.ref.table[2, t]].view(np.uint32), rc.packed[:, t])
    rest = [p for p in range(16) if p not in s.ref.table[2, :2]]
    assert np.array_equal(pool[rest], pool2[rest])
    s.pages.status.zero_()
    s.ref.status = 0
    s.grow([3], [32])
    s.pages.table[3, 0] = 16                             # one past the pool
    s.append([3, 99], [32, 1])
    assert np.array_equal(s.cache.pool.cpu().numpy(), pool2) and int(s.pages.status[0]) == BAD_ID | BAD_ROW


# ------------------------------------------------------------------------------------------------------------- attention
@pytest.mark.parametrize("G,Hkv", [(1, 3), (2, 2), (4, 2), (8, 2), (16, 1), (24, 2), (72, 1)])
@pytest.mark.parametrize("bits", [(2, 2), (3, 4), (2, 3), (4, 1)])
def test_ragged_attention(G, Hkv, bits):
    """Lengths around every border in one batch, slots in another order, padding rows, a slot twice; dead pages and rows hold NaN."""
    W = 32
    lens = [0, 1, 31, W + 31, W + 32, W + 33, 200, 32 * 9 + 5, 700, 1, 64]
    s = Serving(Hkv, G, bits, W, n_slots=len(lens) + 1, n_pages=60, max_tiles=30, W_cap=96, seed=G)
    s.step(list(range(len(lens))), lens)
    rows = [10, -1, 0, 5, 3, 8, 1, 2, 4, -7, 6, 7, 9, 8, 11]
    s.check_attention(rows, f"G {G} bits {bits}")
    s.check_attention(rows, f"G {G} bits {bits}, max_len", max_len=700)
    s.check_attention([8, 0], "two rows", max_len=700, scale=0.25)


@pytest.mark.parametrize("bits", [(kb, vb) for kb in (1, 2, 3, 4) for vb in (1, 2, 3, 4)])
def test_attention_of_every_width(bits):
    for G in (1, 2, 4, 8, 16):
        s = Serving(1, G, bits, 64, n_slots=3, n_pages=40, max_tiles=20, seed=G)
        s.step([0, 1, 2], [333, 96, 17])
        s.check_attention([2, 0, 1], f"{bits} G {G}")


@pytest.mark.parametrize("W,W_cap", [(0, 32), (0, 64), (256, 288), (64, 96), (160, 2048)])
def test_attention_over_rings_of_every_size(W, W_cap):
    """The ring's oldest row anywhere in it, more window tiles than waves, windows of no length."""
    s = Serving(2, 4, (2, 2), W, n_slots=9, n_pages=80, max_tiles=40, W_cap=W_cap, seed=W)
    s.step(range(9), [W + 32 * i + 5 * i for i in range(9)])
    for i in range(3):
        s.check_attention(list(range(9)), f"W {W} ring {W_cap} step {i}")
        s.step(range(9), [1, 7, 13, 19, 25, 30, 31, 32, 40])


@pytest.mark.parametrize("G", [1, 2, 4, 8, 16])
def test_long_contexts_in_many_splits(G):
    """Shares of 8 to 64 tiles, up to some hundred of them, on one workspace that every call leaves as it found it."""
    import torch
    s = Serving(1, G, (2, 4), 32, n_slots=4, n_pages=1700, max_tiles=1200, seed=G)
    s.step([1, 0, 3], [32 * 1100 + 45, 32 * 500 + 32, 300])
    ws = torch.zeros(s.kv.paged_workspace_bytes(s.shape(4), 32 * 1200 + 63), dtype=torch.uint8, device="cuda")
    for i in range(3):
        s.check_attention([0, 1, 2, 3], f"call {i}", ws=ws)
    s.check_attention([3, 3, 0, -1], "shorter ones next", ws=ws, max_len=32 * 500 + 32)
    if G <= 4:
        assert not ws.any()


@pytest.mark.parametrize("bits", [(kb, vb) for kb in (1, 2, 3, 4) for vb in (1, 2, 3, 4)])
def test_one_sequence_in_workgroups_of_twelve_waves(bits):
    """One row with more than 20 tiles for each compute unit that it gets: the other form of the kernel, every width and group size; a shorter sequence
    than max_len, an empty one and a padding row in the same form. Some heads against the oracle, the others against a batch of two."""
    import torch
    Hkv = 128
    s = Serving(Hkv, 1, bits, 32, n_slots=3, n_pages=70, max_tiles=60, seed=20 + bits[0])
    s.step([2, 0], [1429, 77])
    for G in (1, 2, 4, 8):
        s.G = G
        q = s.rng.standard_normal((1, G * Hkv, 128), dtype=np.float32).astype(np.float16)
        ws = torch.zeros(s.kv.paged_workspace_bytes(s.shape(2), 1800), dtype=torch.uint8, device="cuda")

        def run(rows, max_len):
            qt = torch.from_numpy(np.repeat(q, len(rows), 0)).cuda()
            out = torch.full_like(qt, 7.0)
            ws.zero_()
            s.kv.paged_decode_attn(s.shape(len(rows)), s.cfg, qt, s.cache, s.pages, out, ws, rows=s.ints(rows), max_len=max_len)
            torch.cuda.synchronize()
            return out
        both = run([2, 0], 1800)
        for row, want in ((2, both[0]), (0, both[1])):
            got = run([row], 1429)[0]
            assert (got.float() - want.float()).abs().max().item() <= 4e-3, (G, row)      # (an fp16 spacing below 4: sums in another order)
            heads = [0, 5, Hkv - 1]
            st, ref = one_sequence(s.k[row][heads], s.v[row][heads], *bits, 32, G).decode_attn(q.reshape(1, Hkv, G, 128)[:, heads].reshape(1, -1, 128).view(np.uint16))
            assert st == 0
            assert_attn_close(t16(got).reshape(Hkv, G, 128)[heads].reshape(1, -1, 128), ref, f"{bits} G {G} slot {row}", tight=True)
        assert (run([1], 1429) == 0).all() and (run([-1], 1429) == 7).all() and torch.isnan(run([2], 1428)).all()


@pytest.mark.parametrize("G,bits", [(1, (2, 2)), (2, (3, 3)), (4, (3, 4)), (8, (2, 4)), (8, (4, 1)), (16, (2, 2))])
def test_a_few_long_sequences(G, bits):
    """Four rows whose tiles are many for their few units: workgroups of 12 waves (8 with 16 heads), pieces of every row."""
    s = Serving(2, G, bits, 32, n_slots=5, n_pages=2500, max_tiles=1300, seed=30 + G)
    s.step([4, 0, 2, 1], [32 * 1200 + 50, 45, 32 * 700 + 33, 3000])
    s.check_attention([2, 4, 1, 0], f"G {G}", max_len=32 * 1200 + 50)
    s.check_attention([4, -1, 3, 4], f"G {G}, one twice", max_len=32 * 1200 + 50)


@pytest.mark.parametrize("B,G,bits", [(64, 1, (2, 2)), (65, 4, (2, 3)), (300, 2, (1, 2)), (512, 1, (3, 2)), (513, 4, (2, 2)), (1300, 1, (4, 1))])
def test_batches_of_many_rows(B, G, bits):
    """More rows than a lane has one of, and more than a launch has: short contexts, empty ones and a few long ones; with the rows named and without."""
    import torch
    s = Serving(1, G, bits, 32, n_slots=B + 1, n_pages=9 * B, max_tiles=130, seed=B)
    rows = [int(r) for r in s.rng.permutation(B + 1)[:B]]
    fresh = [int(n) for n in s.rng.integers(0, 130, B)]
    for b in (0, B // 2, B - 1):
        fresh[b] = 3000 + b % 100
    s.step(rows, fresh)
    rows[1] = -1
    looked_at = sorted({0, 2, B // 2 - 1, B // 2, B - 2, B - 1, *range(5, B, B // 25)})
    ws = torch.zeros(s.kv.paged_workspace_bytes(s.shape(B), 130 * 32 + 63), dtype=torch.uint8, device="cuda")
    for named in (rows, None, rows):
        q = s.rng.standard_normal((B, G, 128), dtype=np.float32).astype(np.float16)
        out = torch.full((B, G, 128), 7.0, dtype=torch.float16, device="cuda")
        s.kv.paged_decode_attn(s.shape(B), s.cfg, torch.from_numpy(q).cuda(), s.cache, s.pages, out, ws, rows=None if named is None else s.ints(named))
        got = t16(out)
        for b in looked_at:
            slot = b if named is None else named[b]
            if s.ref.lens[slot] == 0:
                assert (got[b] == 0).all()
                continue
            st, want = one_sequence(s.k[slot], s.v[slot], s.kb, s.vb, s.W, G).decode_attn(q[b:b + 1].view(np.uint16))
            assert st == 0
            assert_attn_close(got[b:b + 1], want, f"row {b} slot {slot} of {s.ref.lens[slot]} tokens, named {named is not None}", tight=True)
        if named is not None:
            assert (got[1].view(np.float16) == 7.0).all()


@pytest.mark.parametrize("B,G", [(1, 4), (2, 8), (7, 1), (70, 2), (200, 16), (515, 1)])
def test_batches_of_padding_and_of_empty_sequences(B, G):
    """Nothing but padding: nothing is written, by any of the calls; nothing but empty sequences: zeros."""
    import torch
    s = Serving(2, G, (2, 3), 32, n_slots=B, n_pages=4, max_tiles=20, seed=B)
    pool, ring = s.cache.pool.clone(), s.cache.k_win.clone()
    s.grow([-1] * B, [40] * B)
    s.append([-1] * B, [40] * B)
    s.kv.paged_append(s.shape(B), s.cfg, *torch.zeros((2, B, 2, 128), dtype=torch.float16, device="cuda"), s.cache, s.pages, rows=s.ints([-1] * B))
    s.check_attention([-1] * B, "padding")
    s.grow(range(B), [0] * B)
    s.append(range(B), [0] * B)
    s.check_attention(list(range(B)), "empty")
    s.check_pages()
    assert torch.equal(s.cache.pool, pool) and torch.equal(s.cache.k_win.view(torch.int16), ring.view(torch.int16))


@pytest.mark.parametrize("G", [1, 4, 8, 16])
def test_one_workspace_for_layers_of_other_widths(G):
    """Layers of one shape share a workspace that was zeroed once: other widths, bounds on the length that make other launches, results that are NaN."""
    import torch
    layers = [Serving(2, G, bits, 32, n_slots=4, n_pages=600, max_tiles=1300, seed=50 + G) for bits in ((2, 2), (3, 4), (1, 3))]
    for s in layers:
        s.step([1, 3, 0, 2], [5000, 40, 3000, 4500])
    ws = torch.zeros(layers[0].kv.paged_workspace_bytes(layers[0].shape(4), 1300 * 32 + 63), dtype=torch.uint8, device="cuda")
    for turn in range(3):
        for s in layers:
            for max_len in (0, 5000, 1300 * 32):
                s.check_attention([0, 1, 2, 3], f"{s.kb}/{s.vb} {max_len} turn {turn}", max_len=max_len, ws=ws)
            got, _ = s.attend([0, 1, 2, 3], max_len=4800, ws=ws)
            assert np.isnan(got[1].view(np.float16)).all() and np.isfinite(got[[0, 2, 3]].view(np.float16)).all()


def test_offsets_past_32_bits():
    """A pool of more than 16 GB (2^32 words), rings of more than 4 GB, a table of more than 2^31 entries: what lies at their ends."""
    import torch
    import paper_2506_08018_amd as kv
    Hkv, G, W, n_slots, n_pages = 8, 2, 32, 34000, 720000
    shape, cfg, rng = kv.Shape(2, G * Hkv, Hkv), kv.LayerCfg(2, 2, W), np.random.default_rng(3)
    pages = kv.Pages(n_slots, n_pages, 65000, W)
    cache = kv.PagedCache(shape, cfg, n_pages, n_slots, 64)
    assert cache.pool.numel() > 2 ** 32 and cache.k_win.numel() * 2 > 2 ** 32 and pages.table.numel() > 2 ** 31
    pages.used[:-4] = -1                                    # the last 128 pages are free
    pages.refs[:n_pages - 128] = 1
    rows, fresh = [n_slots - 1, n_slots - 2], [2000, 700]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    data = [[rng.standard_normal((Hkv, n, 128), dtype=np.float32).astype(np.float16) for _ in "kv"] for n in fresh]
    k, v = (torch.from_numpy(np.concatenate([d[i] for d in data], 1)).cuda().transpose(0, 1) for i in (0, 1))
    cu = ints([0, 2000, 2700])
    kv.pages_grow(pages, ints(rows), cu)
    kv.paged_append(shape, cfg, k, v, cache, pages, rows=ints(rows), cu=cu, max_new=2000)
    q = rng.standard_normal((2, G * Hkv, 128), dtype=np.float32).astype(np.float16)
    refs = [one_sequence(d[0], d[1], 2, 2, W, G) for d in data]

    def look(rows, first_page, what):
        at = first_page
        for slot, rc, n in zip(rows, refs, fresh):
            T = tiles_of(n, W)
            ids = pages.table[slot, :T]
            assert ids.tolist() == list(range(at, at + T)), what
            at += T
            assert np.array_equal(cache.pool[ids.long()].cpu().numpy().view(np.uint32), rc.packed[:, :T].transpose(1, 0, 2)), (what, slot)
        out = torch.zeros((2, G * Hkv, 128), dtype=torch.float16, device="cuda")
        ws = torch.zeros(kv.paged_workspace_bytes(shape, 2100), dtype=torch.uint8, device="cuda")
        kv.paged_decode_attn(shape, cfg, torch.from_numpy(q).cuda(), cache, pages, out, ws, rows=ints(rows), max_len=2100)
        for b, rc in enumerate(refs):
            st, want = rc.decode_attn(q[b:b + 1].view(np.uint16))
            assert st == 0
            assert_attn_close(t16(out[b:b + 1]), want, f"{what} row {b}", tight=True)

    look(rows, n_pages - 128, "at the ends")
    pages.used[:-4] = 0
    pages.refs[:n_pages - 128] = 0
    kv.pages_fork(pages, ints(rows), ints([n_slots - 5, 1]))
    kv.copy_windows(shape, cfg, cache, ints(rows), ints([n_slots - 5, 1]))
    kv.pages_compact(pages)
    kv.move_records(shape, cfg, cache, pages)
    look([n_slots - 5, 1], 0, "forked and moved to the front")
    look(rows, 0, "the first ones")
    kv.pages_free(pages, ints([n_slots - 5, 1, *rows]))
    assert not pages.refs.any() and not pages.used.any() and int(pages.status[0]) == 0
    del pages, cache
    torch.cuda.empty_cache()


def test_attention_says_nan_where_it_cannot_know():
    """A page id out of range, a length past max_len, below zero or past the table: NaN for that row, the others as ever."""
    import torch
    s = Serving(2, 4, (2, 2), 32, n_slots=6, n_pages=80, max_tiles=20, seed=9)
    s.step(range(6), [300, 200, 100, 400, 90, 64])
    good_table, good_lens = s.pages.table.clone(), s.pages.lens.clone()
    s.pages.table[1, 2], s.pages.table[3, 0] = 80, -1
    s.pages.lens[2], s.pages.lens[4] = -5, 32 * 20 + 64 + 32
    for max_len in (0, 420):
        got, q = s.attend([0, 1, 2, 3, 4, 5], max_len=max_len)
        for b in (1, 2, 3, 4):
            assert np.isnan(got[b].view(np.float16)).all(), b
        assert np.isfinite(got[[0, 5]].view(np.float16)).all()
    s.pages.table.copy_(good_table); s.pages.lens.copy_(good_lens)
    s.check_attention([0, 1, 2, 3, 4, 5], "mended")
    got, _ = s.attend([0, 3, 5], max_len=300)             # slot 3 has 400
    assert np.isnan(got[1].view(np.float16)).all() and np.isfinite(got[[0, 2]].view(np.float16)).all()


# ------------------------------------------------------------------------------------------------------------- together
def test_serving_run():
    """Prompts, single tokens, forks that go their own ways, sequences that end, a compacted pool: every page, ring row and output after each."""
    s = Serving(2, 4, (2, 4), 32, n_slots=8, n_pages=64, max_tiles=20, seed=77)
    kv = s.kv
    s.step([0, 1, 2], [150, 400, 33])
    for i in range(35):
        s.step([2, 0, 1], [1, 1, 1])
    s.check_attention([1, 2, 0], "prompts and steps")
    kv.pages_fork(s.pages, s.ints([1, 1, 0]), s.ints([4, 5, 7]))
    kv.copy_windows(s.shape(1), s.cfg, s.cache, s.ints([1, 1, 0]), s.ints([4, 5, 7]))
    s.ref.fork([1, 1, 0], [4, 5, 7])
    for a, b in ((1, 4), (1, 5), (0, 7)):
        s.k[b], s.v[b] = s.k[a], s.v[a]
    s.check_pages("forked")
    for i in range(40):                                  # each goes on with tokens of its own; shared pages stay shared
        s.step([1, 4, 5, 0, 7], [1, 1, 1, 1, 1])
    s.check_pages("forks apart")
    s.check_cache("forks apart")
    s.check_attention([4, 1, 5, 7, 0, 2], "forks apart")
    kv.pages_free(s.pages, s.ints([1, 0, 1, 6, -1]))     # one twice, one that is empty
    s.ref.free([1, 0])
    for r in (0, 1):
        s.k[r], s.v[r] = s.k[r][:, :0], s.v[r][:, :0]
    s.check_pages("freed")
    s.step([3], [200])
    s.check_cache("freed and filled")
    kv.pages_free(s.pages, s.ints([5]))
    s.ref.free([5])
    s.k[5], s.v[5] = s.k[5][:, :0], s.v[5][:, :0]
    kv.pages_compact(s.pages)
    kv.move_records(s.shape(1), s.cfg, s.cache, s.pages)
    moves = s.ref.compact()
    assert moves and int(s.pages.moves[0]) == len(moves)
    s.check_pages("compacted")
    s.check_cache("compacted")
    s.step([0, 7], [65, 1])
    s.check_cache("on a compacted pool")
    s.check_attention([0, 4, 7, 3, 2, 1], "on a compacted pool")


def test_captured_decode_loop():
    """A step of two layers (grow, rotation, append, attention) captured once and replayed, with eager steps and synchronizations between: every replay
    against the same steps made eagerly on a second copy of everything."""
    import torch
    import paper_2506_08018_amd as kv
    B, Hkv, G, W, kb, vb, L = 3, 2, 4, 32, 2, 3, 2
    shape, cfg = kv.Shape(B, G * Hkv, Hkv), kv.LayerCfg(kb, vb, W)
    gen = torch.Generator(device="cuda").manual_seed(5)
    steps = 40
    freqs = torch.tensor(kv.rope_frequencies(64)[0], device="cuda")
    xs = torch.randn((steps, L, B, (G + 2) * Hkv, 128), generator=gen, device="cuda").to(torch.bfloat16)
    prompt = torch.randn((2, 300, Hkv, 128), generator=gen, device="cuda").half()

    class Side:
        def __init__(self):
            self.pages = kv.Pages(4, 40, 20, W)
            self.layers = [kv.PagedCache(shape, cfg, 40, 4, 64) for _ in range(L)]
            self.rows = torch.tensor([3, 0, 2], dtype=torch.int32, device="cuda")
            cu = torch.tensor([0, 100, 163, 300], dtype=torch.int32, device="cuda")
            kv.pages_grow(self.pages, self.rows, cu)
            for c in self.layers:
                kv.paged_append(shape, cfg, prompt[0], prompt[1], c, self.pages, rows=self.rows, cu=cu, max_new=137)
            self.x = torch.zeros_like(xs[0])
            self.q = torch.zeros((B, G * Hkv, 128), dtype=torch.float16, device="cuda")
            self.k, self.v = (torch.zeros((B, Hkv, 128), dtype=torch.float16, device="cuda") for _ in range(2))
            self.out = torch.zeros((L, B, G * Hkv, 128), dtype=torch.float16, device="cuda")
            self.ws = torch.zeros(kv.paged_workspace_bytes(shape, 700), dtype=torch.uint8, device="cuda")
            self.pos = torch.zeros(B, dtype=torch.int32, device="cuda")

        def step(self):
            torch.index_select(self.pages.lens, 0, self.rows, out=self.pos)
            kv.pages_grow(self.pages, self.rows)
            for i, c in enumerate(self.layers):
                x = self.x[i]
                kv.qk_norm_rope(shape, x[:, :G * Hkv], x[:, G * Hkv:(G + 1) * Hkv], self.pos, freqs, self.q, self.k, v=x[:, (G + 1) * Hkv:], v_out=self.v)
                kv.paged_append(shape, cfg, self.k, self.v, c, self.pages, rows=self.rows)
                kv.paged_decode_attn(shape, cfg, self.q, c, self.pages, self.out[i], self.ws, rows=self.rows, max_len=700)

    a, b = Side(), Side()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for side in (a, b):                              # eager steps first, the stream's own
            side.x.copy_(xs[0])
            side.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for i in range(1, steps):
        a.x.copy_(xs[i])
        if i % 7 == 3:
            a.step()                                     # an eager step between the replays
        else:
            graph.replay()
        b.x.copy_(xs[i])
        b.step()
        torch.cuda.synchronize()
        diff = (a.out.float() - b.out.float()).abs().max().item()
        assert torch.isfinite(a.out).all() and diff <= 4e-3, (i, diff)       # (waves take tiles in any order: the last bit may differ)
        assert (a.pages.lens == b.pages.lens).all() and (a.pages.table == b.pages.table).all()
    for x, y in zip(a.layers, b.layers):
        assert torch.equal(x.pool, y.pool) and torch.equal(x.k_win, y.k_win) and torch.equal(x.v_win, y.v_win)
    assert int(a.pages.status[0]) == 0 and tiles_of(int(a.pages.lens[0]), W) > tiles_of(63, W)


def test_calls_on_another_stream():
    """The stream argument is the stream of the work: a call behind a long kernel of that stream sees what it wrote."""
    import torch
    s = Serving(2, 4, (2, 2), 32, n_slots=3, n_pages=40, max_tiles=20, seed=12)
    s.step([0, 1, 2], [300, 40, 97])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    q = torch.randn((3, 8, 128), device="cuda").half()
    out, want = torch.zeros_like(q), torch.zeros_like(q)
    ws = torch.zeros(s.kv.paged_workspace_bytes(s.shape(3), 700), dtype=torch.uint8, device="cuda")
    s.kv.paged_decode_attn(s.shape(3), s.cfg, q, s.cache, s.pages, want, ws)
    torch.cuda.synchronize()
    late = torch.zeros_like(q)
    with torch.cuda.stream(stream):
        a = torch.randn((4096, 4096), device="cuda")
        for _ in range(8):
            a = a @ a * 1e-3
        late.copy_(q)
    s.kv.paged_decode_attn(s.shape(3), s.cfg, late, s.cache, s.pages, out, ws, stream=stream)
    torch.cuda.synchronize()
    assert (out.float() - want.float()).abs().max().item() <= 4e-3
