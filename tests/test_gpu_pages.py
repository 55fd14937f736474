"""Bookkeeping of the paged cache on the GPU against plain loops on the host: whole numbers, all equal."""
import numpy as np
import pytest

from paged_common import Serving
from paged_ref import BAD_ID, BAD_ROW, EXHAUSTED, OCCUPIED, tiles_of

pytestmark = pytest.mark.gpu


def bare(n_slots, n_pages, max_tiles, W, seed=0):
    return Serving(1, 1, (1, 1), W, n_slots, n_pages, max_tiles, W_cap=W + 32, seed=seed)


@pytest.mark.parametrize("n_slots,n_pages,max_tiles,W,seed", [(5, 1, 3, 0, 1), (9, 31, 8, 32, 2), (40, 700, 64, 64, 3), (200, 9000, 300, 128, 4),
                                                             (64, 33, 40, 32, 5), (300, 4097, 30, 0, 6)])
def test_random_traffic(n_slots, n_pages, max_tiles, W, seed):
    """Grow, free, fork and compact in random order, pools that run out among them."""
    s = bare(n_slots, n_pages, max_tiles, W, seed)
    rng, kv = s.rng, s.kv
    for i in range(30):
        what = rng.choice(["grow", "grow", "step", "free", "fork", "compact"])
        rows = [int(r) for r in rng.permutation(n_slots)[:rng.integers(1, n_slots + 1)]]
        if rng.random() < 0.3:
            rows[rng.integers(len(rows))] = -1
        if what in ("grow", "step"):
            fresh = [1] * len(rows) if what == "step" else [int(rng.integers(0, 32 * max_tiles // 3 + 40)) for _ in rows]
            s.grow(rows, fresh)
        elif what == "free":
            rows = rows[:max(1, len(rows) // 2)]
            kv.pages_free(s.pages, s.ints(rows))
            s.ref.free(rows)
        elif what == "fork":
            half = len(rows) // 2
            if not half:
                continue
            src = [rows[int(j)] for j in rng.integers(0, half, half)]
            dst = rows[half:2 * half]
            kv.pages_fork(s.pages, s.ints(src), s.ints(dst))
            s.ref.fork(src, dst)
        else:
            kv.pages_compact(s.pages)
            moves = s.ref.compact()
            m = s.pages.moves.cpu().numpy()
            assert m[0] == len(moves) and m[1] == int((s.ref.refs > 0).sum())
            assert [(int(m[4 + j]), int(m[4 + n_pages + j])) for j in range(m[0])] == moves
        s.check_pages(f"{i} {what}")
        s.pages.status.zero_()
        s.ref.status = 0


def test_grow_takes_the_lowest_free_pages_in_order():
    s = bare(6, 5000, 2000, 0)
    s.grow([2, 0], [32 * 3, 32 * 2])
    assert s.ref.table[2, :3].tolist() == [0, 1, 2] and s.ref.table[0, :2].tolist() == [3, 4]
    s.grow([5, 1], [32 * 1900, 32 * 1700 + 31])                # over several stretches of 4096 ids
    s.check_pages()
    s.kv.pages_free(s.pages, s.ints([2, 1]))
    s.ref.free([2, 1])
    s.grow([3, 4], [32, 32 * 1800])
    s.check_pages()


def test_grow_grants_rows_in_order():
    s = bare(6, 10, 9, 32)
    s.grow([3, 1, 0, 2, 5], [32 + 32 * 6, 32 + 32 * 5, 40, 32 + 32 * 2, 0])     # 6 of 10; 5 more are too many; none; then no more
    assert s.ref.lens.tolist() == [40, 0, 0, 224, 0, 0] and s.ref.status == EXHAUSTED
    s.check_pages()
    s.pages.status.zero_(); s.ref.status = 0
    s.grow([4], [32 + 32 * 10])                                # more than a row of the table holds
    assert s.ref.status == EXHAUSTED
    s.check_pages()


def test_grow_refuses_bad_rows():
    s = bare(4, 20, 9, 32)
    s.grow([1, 4, 1, 2, 100000], [50, 3, 60, 70, 1])           # a slot past the end twice, slot 1 twice
    assert s.ref.lens.tolist() == [0, 50, 70, 0] and s.ref.status == BAD_ROW
    s.check_pages()
    s.kv.pages_grow(s.pages, s.ints([0, 2]), s.ints([10, 4, 2 ** 31 - 1]))      # fewer than no tokens; more than a length holds
    assert s.pages.lens.cpu().tolist() == [0, 50, 70, 0]


def test_grow_grants_nothing_where_a_count_cannot_be():
    s = bare(4, 20, 9, 32)
    s.grow([0, 1, 2], [50, 60, 70])
    s.kv.pages_grow(s.pages, s.ints([0, 2, 1]), s.ints([10, 4, 2 ** 31 - 1, 2 ** 31 - 1]))      # fewer than no tokens; more than a length holds; none
    assert s.pages.grown.cpu().tolist() == [0, 0, 0, 0] and s.pages.lens.cpu().tolist() == [50, 60, 70, 0]
    assert int(s.pages.status[0]) == BAD_ROW


def test_grow_without_rows_or_counts():
    s = bare(5, 20, 9, 0)
    for _ in range(33):
        s.kv.pages_grow(s.pages, n_rows=4)
        s.ref.grow(list(range(4)), [1] * 4)
    s.check_pages()


def test_pools_of_more_than_32768_pages():
    """Free ids that lie far apart in a large pool, more of them than a list holds, and slots past 32768 that share a place in the table of names."""
    s = bare(70000, 100000, 4200, 0)
    rows = [5, 32773, 65541, 69999, 37]
    s.grow(rows, [32 * 4100, 32 * 4200, 32 * 4000, 32 * 4199, 32 * 4200])
    s.kv.pages_free(s.pages, s.ints([32773, 37]))
    s.ref.free([32773, 37])
    s.grow([100, 32868, 65636], [32 * 10, 32 * 4150, 32 * 3000])
    s.grow([7, 32775, 7], [32, 64, 96])
    assert s.ref.status == BAD_ROW
    s.check_pages()
    few = [100 + i for i in range(20)]
    for i in range(3):                                         # a full pool but for some pages near its end
        s.grow(few, [32 * 4000] * 20)
    s.check_pages()
    s.kv.pages_compact(s.pages)
    s.ref.compact()
    s.check_pages()


@pytest.mark.parametrize("B", [1, 1023, 1025, 4096])
def test_grow_of_many_rows(B):
    s = bare(4096, 9000, 4, 0)
    rng = np.random.default_rng(B)
    rows = [int(r) for r in rng.permutation(4096)[:B]]
    fresh = [int(n) for n in rng.integers(0, 100, B)]
    s.grow(rows, fresh)
    s.check_pages()


def test_fork_refuses_what_would_race():
    s = bare(8, 60, 9, 32)
    s.grow([0, 1, 2], [200, 100, 64])
    src, dst = [0, 0, 1, 2, 3, 1, 9, -1, 1, 4], [3, 4, 4, 1, 5, 1, 6, 7, 7, 6]
    # 3 is a source too; 4 is named twice and a source; 1 holds tokens and is a source and a destination; 9 is no slot
    s.kv.pages_fork(s.pages, s.ints(src), s.ints(dst))
    s.ref.fork(src, dst)
    assert s.ref.status == OCCUPIED | BAD_ROW
    s.check_pages()
    s.kv.pages_fork(s.pages, s.ints([0, 0, 7, 1]), s.ints([3, 4, 5, 6]))        # 7 is empty: an empty fork
    s.ref.fork([0, 0, 7, 1], [3, 4, 5, 6])
    assert s.ref.lens.tolist()[3:7] == [200, 200, 0, 100]
    s.check_pages()


def test_free_of_everything_and_of_bad_rows():
    s = bare(4, 20, 9, 0)
    s.grow([0, 1, 2], [100, 64, 31])
    s.kv.pages_free(s.pages, s.ints([2, 0, 0, 4, -2, 1, 0]))
    s.ref.free([2, 0, 4, 1])
    s.check_pages()
    assert not s.ref.refs.any() and s.ref.status == BAD_ROW
    s.pages.status.zero_(); s.ref.status = 0
    s.grow([3], [64])
    s.pages.table[3, 1] = 20                                   # an id that the pool does not have
    s.kv.pages_free(s.pages, s.ints([3]))
    assert int(s.pages.status[0]) == BAD_ID and int(s.pages.refs.sum()) == 1


@pytest.mark.parametrize("Hkv,bits,W", [(1, (1, 1), 0), (3, (3, 4), 32), (8, (2, 2), 128)])
def test_copies(Hkv, bits, W):
    """Rings and records move whole, everything else stays; slots out of range are left out."""
    import torch
    import paper_2506_08018_amd as kv
    shape, cfg = kv.Shape(1, Hkv, Hkv), kv.LayerCfg(*bits, W)
    cache = kv.PagedCache(shape, cfg, 70, 9, W + 64)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for t in (cache.pool, cache.k_win.view(torch.int16), cache.v_win.view(torch.int16)):
        t.random_(generator=gen)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    want = [cache.k_win.clone(), cache.v_win.clone()]
    for w in want:
        w[[3, 8, 5]] = w[[0, 0, 2]]
    kv.copy_windows(shape, cfg, cache, ints([0, 0, 2, -1, 1, 9]), ints([3, 8, 5, 4, 9, 6]))
    assert torch.equal(cache.k_win.view(torch.int16), want[0].view(torch.int16)) and torch.equal(cache.v_win.view(torch.int16), want[1].view(torch.int16))
    pages = kv.Pages(9, 70, 20, W)
    kv.pages_grow(pages, ints([0, 1, 2]), ints([0, W + 32 * 10, 2 * W + 32 * 30, 3 * W + 32 * 48]))
    kv.pages_free(pages, ints([1]))
    kv.pages_compact(pages)
    want = cache.pool.clone()
    n = int(pages.moves[0])
    assert n == 18
    want[pages.moves[4 + 70:4 + 70 + n].long()] = want[pages.moves[4:4 + n].long()]
    kv.move_records(shape, cfg, cache, pages)
    assert torch.equal(cache.pool, want)
    kv.pages_compact(pages)                                    # nothing left to move
    assert int(pages.moves[0]) == 0
    kv.move_records(shape, cfg, cache, pages)
    assert torch.equal(cache.pool, want)


def test_moves_that_no_compaction_wrote():
    """A list whose count is more than there can be, of ids that no pool has: nothing is moved, and status says so."""
    s = Serving(2, 1, (2, 2), 32, 3, 10, 4, seed=8)
    s.kv.pages_compact(s.pages)
    s.pages.moves.fill_(-1)
    s.pages.moves[0] = 2 ** 31 - 1
    before = s.cache.pool.clone()
    s.kv.move_records(s.shape(1), s.cfg, s.cache, s.pages)
    assert bool((s.cache.pool == before).all()) and int(s.pages.status[0]) == BAD_ID
