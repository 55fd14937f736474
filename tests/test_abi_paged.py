"""Host-side refusals of the paged cache's entry points, and the frequencies of the rotation (host arithmetic): nothing is launched, no GPU."""
import ctypes as C
import math

import numpy as np
import pytest

A = 4096          # an aligned address that nobody follows


@pytest.fixture(scope="module")
def kv():
    import paper_2506_08018_amd as kv
    kv.lib()
    return kv


def pages(**change):
    from paper_2506_08018_amd.binding import _PagesStruct
    f = dict(table=A, lens=A, grown=A, refs=A, used=A, status=A, moves=A, n_slots=8, n_pages=100, max_tiles=16, window=64)
    f.update(change)
    return _PagesStruct(*f.values())


def cache(**change):
    from paper_2506_08018_amd.binding import _PagedCacheStruct
    f = dict(pool=A, k_win=A, v_win=A, n_pages=100, n_slots=8, W_cap=96)
    f.update(change)
    return _PagedCacheStruct(*f.values())


BAD_PAGES = [(dict(table=None), -1), (dict(lens=None), -1), (dict(grown=None), -1), (dict(refs=None), -1), (dict(used=None), -1), (dict(status=None), -1),
             (dict(table=A + 2), -5), (dict(status=A + 1), -5), (dict(n_slots=0), -4), (dict(n_pages=0), -4), (dict(n_pages=1 << 22), -4),
             (dict(max_tiles=0), -4), (dict(max_tiles=(1 << 23) + 1), -4), (dict(window=-1), -4), (dict(window=40), -4)]


@pytest.mark.parametrize("change,status", BAD_PAGES)
def test_every_call_checks_the_pages(kv, change, status):
    L, p, sh, cfg, c = kv.lib(), pages(**change), kv.Shape(2, 8, 4), kv.LayerCfg(2, 2, 64), cache()
    r = C.byref
    a = C.c_void_p(A)
    assert L.kvmix_pages_grow(r(p), a, a, 2, None) == status
    assert L.kvmix_pages_free(r(p), a, 2, None) == status
    assert L.kvmix_pages_fork(r(p), a, a, 2, None) == status
    assert L.kvmix_pages_compact(r(p), None) == status
    assert L.kvmix_move_records(r(sh), r(cfg), r(c), r(p), None) == status
    assert L.kvmix_paged_append(r(sh), r(cfg), a, 512, 128, a, 512, 128, 9, r(c), r(p), a, a, 1, None) == status
    assert L.kvmix_paged_decode_attn(r(sh), r(cfg), a, r(c), r(p), a, 100, C.c_float(0), a, a, 1 << 30, None) == status


@pytest.mark.parametrize("shape,cfg,status", [((2, 8, 4, 64, 32), (2, 2, 64), -4), ((2, 8, 4, 128, 16), (2, 2, 64), -3), ((2, 12, 4, 128, 32), (2, 2, 64), -4),
                                              ((2, 8, 4, 128, 32), (0, 2, 64), -2), ((2, 8, 4, 128, 32), (16, 16, 64), -2),
                                              ((2, 8, 4, 128, 32), (2, 2, -1), -4), ((2, 8, 4, 128, 32), (2, 2, 32), -4)])
def test_shape_widths_and_window(kv, shape, cfg, status):
    """16-bit layers have nothing to page, the count policy has no single front; the window is the pages'."""
    L, sh, cf, p, c, r, a = kv.lib(), kv.Shape(*shape), kv.LayerCfg(*cfg), pages(), cache(), C.byref, C.c_void_p(A)
    assert L.kvmix_move_records(r(sh), r(cf), r(c), r(p), None) == status
    assert L.kvmix_paged_append(r(sh), r(cf), a, 512, 128, a, 512, 128, 9, r(c), r(p), a, a, 1, None) == status
    assert L.kvmix_paged_decode_attn(r(sh), r(cf), a, r(c), r(p), a, 100, C.c_float(0), a, a, 1 << 30, None) == status
    if cfg != (2, 2, 32):
        assert L.kvmix_copy_windows(r(sh), r(cf), r(c), a, a, 2, None) == status


@pytest.mark.parametrize("change,status", [(dict(pool=None), -1), (dict(k_win=None), -1), (dict(v_win=None), -1), (dict(pool=A + 8), -5), (dict(v_win=A + 4), -5),
                                           (dict(W_cap=64), -4), (dict(W_cap=100), -4), (dict(n_pages=99), -4), (dict(n_slots=9), -4)])
def test_the_cache(kv, change, status):
    L, sh, cfg, p, c, r, a = kv.lib(), kv.Shape(2, 8, 4), kv.LayerCfg(2, 2, 64), pages(), cache(**change), C.byref, C.c_void_p(A)
    assert L.kvmix_paged_append(r(sh), r(cfg), a, 512, 128, a, 512, 128, 9, r(c), r(p), a, a, 1, None) == status
    assert L.kvmix_paged_decode_attn(r(sh), r(cfg), a, r(c), r(p), a, 100, C.c_float(0), a, a, 1 << 30, None) == status


def test_counts_and_pointers(kv):
    L, sh, cfg, p, c, r, a, odd = kv.lib(), kv.Shape(2, 8, 4), kv.LayerCfg(2, 2, 64), pages(), cache(), C.byref, C.c_void_p(A), C.c_void_p(A + 8)
    assert L.kvmix_pages_grow(None, a, a, 2, None) == -1
    assert L.kvmix_pages_grow(r(p), a, a, -1, None) == L.kvmix_pages_grow(r(p), a, a, 4097, None) == -4
    assert L.kvmix_pages_grow(r(p), C.c_void_p(A + 1), a, 1, None) == -5
    assert L.kvmix_pages_grow(r(p), None, None, 0, None) == 0
    assert L.kvmix_pages_free(r(p), a, -1, None) == -4 and L.kvmix_pages_free(r(p), a, 0, None) == 0
    assert L.kvmix_pages_fork(r(p), None, a, 1, None) == -1 and L.kvmix_pages_fork(r(p), a, a, 4097, None) == -4 and L.kvmix_pages_fork(r(p), None, None, 0, None) == 0
    assert L.kvmix_pages_compact(r(pages(moves=None)), None) == -1 and L.kvmix_pages_compact(r(pages(moves=A + 8)), None) == -5
    assert L.kvmix_move_records(r(sh), r(cfg), r(c), r(pages(moves=None)), None) == -1
    assert L.kvmix_copy_windows(r(sh), r(cfg), r(c), a, None, 1, None) == -1 and L.kvmix_copy_windows(r(sh), r(cfg), r(c), a, a, 65536, None) == -4
    assert L.kvmix_copy_windows(r(sh), r(cfg), r(c), None, None, 0, None) == 0

    def append(k=a, ks=(512, 128), v=a, vs=(512, 128), n=9, rows=a, cu=a, max_new=3):
        return L.kvmix_paged_append(r(sh), r(cfg), k, *ks, v, *vs, n, r(c), r(p), rows, cu, max_new, None)

    assert append(k=None) == append(v=None) == -1
    assert append(k=odd) == append(v=odd) == append(ks=(4, 128)) == append(ks=(512, 4)) == append(vs=(-512, 128)) == append(vs=(512, 12)) == -5
    assert append(max_new=-1) == append(cu=None, max_new=2) == append(n=-1) == append(cu=None, max_new=1, n=1) == -4
    big = kv.Shape(2, 8 * 16, 8 * 16)
    assert L.kvmix_paged_append(r(big), r(cfg), a, 128 * 128, 128, a, 128 * 128, 128, 2 ** 31 - 1, r(c), r(p), a, a, 2 ** 31 - 1, None) == -4
    assert append(k=None, v=None, max_new=0) == append(k=None, v=None, n=0) == 0
    assert append(rows=C.c_void_p(A + 2)) == -5

    def attn(q=a, rows=a, max_len=100, out=a, ws=a, n=1 << 30, sh=sh, p=p):
        return L.kvmix_paged_decode_attn(r(sh), r(cfg), q, r(c), r(p), rows, max_len, C.c_float(0), out, ws, n, None)

    assert attn(q=None) == attn(out=None) == -1
    assert attn(q=odd) == attn(out=odd) == attn(max_len=500, ws=odd) == -5
    assert attn(max_len=500, ws=None) == -1 and attn(max_len=500, n=64) == -6          # 500 tokens of 8 units are split
    assert attn(rows=None, sh=kv.Shape(9, 36, 4)) == -4                                # more batch rows than slots


def test_sizes_past_what_is_counted_in_32_bits(kv):
    """Windows whose lengths would not fit, more workgroups than a launch has."""
    L, sh, r, a, W = kv.lib(), kv.Shape(2, 8, 4), C.byref, C.c_void_p(A), 2 ** 31 - 32
    assert L.kvmix_pages_grow(r(pages(window=W)), a, a, 2, None) == L.kvmix_pages_compact(r(pages(window=2 ** 30 + 32)), None) == -4
    cfg, c = kv.LayerCfg(2, 2, W), cache(W_cap=2 ** 31 - 32)
    assert L.kvmix_copy_windows(r(sh), r(cfg), r(c), a, a, 2, None) == -4
    assert L.kvmix_paged_append(r(sh), r(cfg), a, 512, 128, a, 512, 128, 9, r(c), r(pages(window=W)), a, a, 1, None) == -4
    assert L.kvmix_paged_decode_attn(r(sh), r(cfg), a, r(c), r(pages(window=W)), a, 100, C.c_float(0), a, a, 1 << 30, None) == -4
    cfg, c = kv.LayerCfg(2, 2, 64), cache()
    assert L.kvmix_paged_append(r(sh), r(cfg), a, 0, 0, a, 0, 0, 2 ** 27, r(c), r(pages()), a, a, 2 ** 27, None) == -4
    from paper_2506_08018_amd.binding import _rope_struct
    rope = _rope_struct(A, 64, 0, 1.0, 1e-6, 0, 0, A, A, 0, 0, *[0] * 8)
    assert L.kvmix_qk_norm_rope(r(sh), rope, 0, 2 ** 24, a, None) == -4
    assert kv.paged_workspace_bytes(sh, 2 ** 31 - 1) >= kv.paged_workspace_bytes(sh, 2 ** 30) > 0


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """kvmix_paged_decode_attn with its launch taken down: (B, Hkv, G, v_bits, W, max_len, workspace) -> status and, of the last
    launch, pieces, batch rows, heads per block, bytes of counters, tiles of a share of one sequence, waves."""
    import os
    import subprocess
    from paper_2506_08018_amd import build
    so = str(tmp_path_factory.mktemp("plan") / "paged_plan.so")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(build.COMMON + ["-shared", os.path.join(here, "paged_plan.hip"), "-o", so], check=True, capture_output=True)
    f = C.CDLL(so).paged_plan
    f.argtypes = [C.c_int] * 6 + [C.c_size_t, C.c_void_p]

    def run(*args):
        out = (C.c_longlong * 6)()
        return (f(*args, out), *out)

    return run


def packed(n, W):
    return 0 if n < W + 32 else (n - W) // 32


def test_workspace_is_enough_for_every_window_and_width(kv, plan):
    for B, Hkv, G in [(1, 1, 1), (1, 8, 4), (3, 2, 8), (16, 8, 4), (64, 8, 8), (2, 1, 72), (700, 32, 1), (1000, 64, 8)]:
        for n in (1, 40, 300, 1000, 5000, 40000, 300000, 2 ** 31 - 1):
            need = kv.paged_workspace_bytes(kv.Shape(B, G * Hkv, Hkv), n)
            for W in (0, 32, 64, 256, 4096):
                for vb in (2, 3):
                    for m in {n, max(1, n // 2), max(1, n - 33)}:
                        st, pieces, rows, block, counters, _, _ = plan(B, Hkv, G, vb, W, m, need)
                        assert st == 0, (B, Hkv, G, n, W, vb, m)
                        assert pieces <= min(B, 512) or counters + pieces * Hkv * G * 520 <= need


def pieces_of(lens, W, fair, share):
    """What the kernel works out (find_piece) in shares of 2.2 times what each workgroup would get, in its arithmetic: fp32; of one sequence by the host's share."""
    if len(lens) == 1:
        return max(1, -(-packed(lens[0], W) // share))
    units = np.array([0 if n <= 0 else packed(n, W) + 3 * -(-(n - 32 * packed(n, W)) // 32) for n in lens], np.int64)
    size = int(np.ceil(np.float32(units.astype(np.float32).sum(dtype=np.float32)) * np.float32(fair) * np.float32(2.2)))
    return int(np.maximum(1, -(-units // max(8, size))).sum())


def test_the_grid_holds_every_piece(kv, plan):
    """However the lengths are spread below max_len, the launch has workgroups for whole contexts and for pieces of the largest share (smaller shares
    are taken where their pieces fit)."""
    rng = np.random.default_rng(1)
    for B, Hkv, G in [(1, 1, 1), (1, 8, 4), (1, 40, 8), (1, 300, 2), (1, 1, 72), (2, 16, 1), (5, 2, 16), (64, 8, 8), (300, 1, 4), (512, 32, 1), (2, 1, 72), (7, 600, 1),
                      (31, 8, 4), (32, 8, 4), (33, 8, 4), (4, 113, 1), (2, 255, 1), (2, 256, 1), (3, 8, 4)]:
        for max_len in (1, 33, 95, 300, 5000, 70000, 2000000):
            for W in (0, 32, 256):
                need = kv.paged_workspace_bytes(kv.Shape(B, G * Hkv, Hkv), max_len)
                st, pieces, rows, block, _, share, waves = plan(B, Hkv, G, 2, W, max_len, need)
                assert st == 0 and rows == B and (waves == 8 or (B <= 64 and block == G <= 8))
                assert pieces >= (rows if B > 1 else 1)
                HH = Hkv * -(-G // block)
                for lens in ([max_len] * B, [max_len] + [0] * (B - 1), [max_len] + [1] * (B - 1), rng.integers(0, max_len + 1, B).tolist(),
                             np.exp(rng.uniform(0, np.log(max_len + 1), B)).astype(int).tolist(), [max(0, max_len - 31)] * B):
                    assert pieces_of(lens, W, HH / (256 if waves == 12 else 512), share) <= pieces, (B, Hkv, G, max_len, W, lens[:8])


def test_rotation_refusals(kv):
    from paper_2506_08018_amd.binding import _rope_struct
    L, r, a = kv.lib(), C.byref, C.c_void_p(A)
    sh = kv.Shape(1, 8, 2)

    def call(dtype=1, n=3, pos=a, q=A, q_out=A, v=0, v_out=0, tok=1024, head=128, **rope):
        f = dict(frequencies=A, rotary_dim=128, interleaved=0, amplitude=1.0, eps=1e-6, q_weight=0, k_weight=0)
        f.update(rope)
        return L.kvmix_qk_norm_rope(r(sh), _rope_struct(*f.values(), q, q_out, tok, head, 0, 0, 0, 0, v, v_out, tok, head), dtype, n, pos, None)

    assert L.kvmix_qk_norm_rope(r(sh), None, 0, 1, a, None) == -1
    assert call(dtype=3) == call(n=-1) == call(rotary_dim=8) == call(rotary_dim=144) == call(rotary_dim=-16) == call(eps=-1.0) == call(eps=float("nan")) == -4
    assert call(q_out=0) == call(q=0) == call(v_out=A) == call(v=A) == call(pos=None) == call(frequencies=0) == -1
    assert call(q=A + 8) == call(q_out=A + 8) == call(tok=1028) == call(head=4) == call(q_weight=A + 2) == call(frequencies=A + 4) == call(pos=C.c_void_p(A + 2)) == -5
    assert call(n=0) == 0 and call(q=0, q_out=0) == 0
    assert call(dtype=2, n=0, tok=1028, head=132) == 0          # four fp32 elements are 16 bytes


def test_frequencies(kv):
    for r in (2, 16, 96, 128):
        f, amplitude = kv.rope_frequencies(r, 10000.0)
        assert np.allclose(f, 10000.0 ** (-np.arange(0, r, 2) / r), rtol=1e-7, atol=0) and amplitude == 1.0
    plain = np.array(kv.rope_frequencies(128, 500000.0)[0], np.float64)
    assert np.allclose(kv.rope_frequencies(128, 500000.0, "linear", 8.0)[0], plain / 8, rtol=1e-6)
    base = np.array(kv.rope_frequencies(128, 500000.0, "base", 8.0)[0])
    assert base[0] == 1.0 and base[-1] == pytest.approx(plain[-1] / 8, rel=1e-6)
    turns = np.array(kv.rope_frequencies(128, 500000.0, "turns", 8.0, 8192, 1.0, 4.0)[0], np.float64)
    made = 8192 * plain / (2 * math.pi)
    assert np.allclose(turns[made >= 4], plain[made >= 4], rtol=1e-6) and np.allclose(turns[made <= 1], plain[made <= 1] / 8, rtol=1e-6)
    part = (made > 1) & (made < 4)
    keep = (made[part] - 1) / 3
    assert part.any() and np.allclose(turns[part], plain[part] * keep + plain[part] / 8 * (1 - keep), rtol=1e-6)
    index, amplitude = kv.rope_frequencies(64, 10000.0, "index", 16.0, 4096, 1.0, 32.0)
    plain = 10000.0 ** (-np.arange(0, 64, 2) / 64)
    at = lambda t: 64 * math.log(4096 / (2 * math.pi * t)) / (2 * math.log(10000.0))
    keep = np.clip((at(1.0) - np.arange(32)) / (at(1.0) - at(32.0)), 0, 1)
    assert np.allclose(index, plain * keep + plain / 16 * (1 - keep), rtol=1e-6) and amplitude == pytest.approx(0.1 * math.log(16.0) + 1)
    assert (np.diff(index) < 0).all()


@pytest.mark.parametrize("args", [(3, 1e4), (0, 1e4), (130, 1e4), (64, 1.0), (64, float("inf")), (64, 1e4, "none such"), (64, 1e4, "linear", 0.5), (2, 1e4, "base", 2.0),
                                  (64, 1e4, "turns", 2.0, 0, 1.0, 4.0), (64, 1e4, "turns", 2.0, 4096, 4.0, 1.0), (64, 1e4, "index", float("nan"), 4096),
                                  (64, 1e4, "index", 2.0, 4096, 0.0, 4.0)])
def test_frequency_refusals(kv, args):
    with pytest.raises(kv.KVMixError) as e:
        kv.rope_frequencies(*args)
    assert e.value.status == -4


def test_bindings_check_their_tensors(kv):
    import torch
    p = kv.Pages(4, 40, 8, 32, device="cpu")
    assert p.table.shape == (4, 8) and p.used.numel() == 2 and p.moves is None
    with pytest.raises(AssertionError):
        kv.Pages(4, 40, 8, 32, device="cpu", buffers=dict(lens=torch.zeros(3, dtype=torch.int32)))
    with pytest.raises(AssertionError):
        kv.Pages(4, 40, 8, 32, device="cpu", buffers=dict(lens=torch.zeros(4, dtype=torch.int64)))
    with pytest.raises(AssertionError):
        kv.Pages(4, 40, 8, 32, device="cpu", buffers=dict(length=torch.zeros(4, dtype=torch.int32)))
    c = kv.PagedCache(kv.Shape(1, 8, 2), kv.LayerCfg(2, 3, 32), 40, 4, 64, device="cpu")
    assert c.pool.shape == (40, 2, 256 + 128 * 5) and c.k_win.shape == (4, 2, 64, 128)
    with pytest.raises(AssertionError):
        kv.PagedCache(kv.Shape(1, 8, 2), kv.LayerCfg(2, 3, 32), 41, 4, 64, device="cpu", buffers=dict(pool=c.pool))
