"""Norm, rotation and conversion of queries, Keys and Values on the GPU against the definition in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = ["float16", "bfloat16", "float32"]


def definition(x, w, eps, pos, freqs, interleaved, amplitude):
    """[n][heads][128] in 64 bits."""
    x = x.astype(np.float64)
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w.astype(np.float64)
    if freqs is not None:
        r = 2 * len(freqs)
        angle = pos.astype(np.float64)[:, None, None] * freqs.astype(np.float64)
        c, s = np.cos(angle) * amplitude, np.sin(angle) * amplitude
        a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
        y = x.copy()
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        x = y
    return x


def close(got, want, row):
    """One rounding to fp16 (half a step, 2^-11 of the value or 2^-25 below the normal range) on top of fp32 arithmetic: some twenty roundings of
    2^-24 on terms of the pair's size, under 2^-19 of the largest value of the row. From 65520 on (65504 and half a step) rounding to fp16 gives
    infinity."""
    past = np.abs(want) >= 65520
    assert (np.isinf(got) == past).all() and (np.sign(got[past]) == np.sign(want[past])).all()
    got, want = np.where(past, 0, got), np.where(past, 0, want)
    err = np.abs(got.astype(np.float64) - want)
    bound = np.maximum(np.abs(want) * 2.0 ** -11, 2.0 ** -25) + row * 2.0 ** -19
    assert (err <= bound).all(), (np.argwhere(err > bound)[:4], err.max())


def run(dtype, N, Hq, Hkv, rot, interleaved, norm, far, factor=1.0, seed=0, spread=1.0):
    import torch
    import paper_2506_08018_amd as kv
    t = getattr(torch, dtype)
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn((N, Hq + 2 * Hkv + 1, 128 + 16), generator=gen) * spread).to(t).cuda()[:, :, 8:136]       # strided in tokens and heads
    pos = torch.randint(-far, far, (N,), generator=gen, dtype=torch.int64).int()
    freqs, amplitude = (None, 1.0) if rot == 0 else kv.rope_frequencies(rot, 10000.0, "index" if factor > 1 else "plain", factor, 4096)
    qw, kw = ((1 + 0.3 * torch.randn(128, generator=gen)).to(t) if norm else None for _ in range(2))
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:Hq + 2 * Hkv]
    outs = [torch.full(y.shape, 9.0, dtype=torch.float16, device="cuda") for y in (q, k, v)]
    up = lambda y: None if y is None else y.cuda()
    f = None if freqs is None else torch.tensor(freqs, dtype=torch.float32)
    kv.qk_norm_rope(kv.Shape(1, Hq, Hkv), q, k, pos.cuda(), up(f), outs[0], outs[1], v=v, v_out=outs[2], q_weight=up(qw), k_weight=up(kw), eps=1e-5,
                    interleaved=interleaved, amplitude=amplitude)
    torch.cuda.synchronize()
    host = lambda y: None if y is None else y.float().cpu().numpy()
    for y, w, o, fr in ((q, qw, outs[0], f), (k, kw, outs[1], f), (v, None, outs[2], None)):
        want = definition(host(y), host(w), np.float64(np.float32(1e-5)), pos.numpy(), None if fr is None else fr.numpy(), interleaved, np.float64(np.float32(amplitude)))
        close(o.cpu().numpy(), want, np.abs(want).max(-1, keepdims=True))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 48, 64, 128])
def test_types_layouts_and_parts(dtype, interleaved, rot):
    for norm in (False, True):
        run(dtype, 7, 8, 2, rot, interleaved, norm, 5000, seed=rot)


@pytest.mark.parametrize("N,Hq,Hkv", [(1, 1, 1), (1, 32, 8), (2, 72, 1), (64, 64, 8), (513, 4, 4), (3000, 32, 8), (1, 512, 1), (1000, 1, 1), (77, 2, 2), (31, 4, 2), (600, 24, 1), (1200, 64, 8)])
def test_sizes(N, Hq, Hkv):
    run("bfloat16", N, Hq, Hkv, 128, False, True, 100000, seed=N)
    run("float16", N, Hq, Hkv, 96, True, False, 100000, seed=N)


@pytest.mark.parametrize("far", [2 ** 17, 10 ** 6, 2 ** 31 - 1])
def test_far_positions(far):
    """The angle of a far position: taken in 32 bits it would be off by whole hundredths of a radian."""
    run("float16", 40, 8, 2, 128, False, False, far, seed=3)
    run("bfloat16", 40, 8, 2, 128, True, True, far, factor=16.0, seed=4)


def test_small_and_large_heads():
    """Heads of next to nothing next to eps, heads of large values, a head of zeros."""
    run("float32", 9, 4, 4, 64, False, True, 100, spread=1e-6)
    run("float32", 9, 4, 4, 64, False, True, 100, spread=1e6)
    run("float16", 9, 4, 4, 64, False, False, 100, spread=1000.0)
    import torch
    import paper_2506_08018_amd as kv
    x = torch.zeros((2, 4, 128), device="cuda", dtype=torch.bfloat16)
    w = torch.ones(128, device="cuda", dtype=torch.bfloat16)
    o = torch.full((2, 4, 128), 5.0, device="cuda", dtype=torch.float16)
    kv.qk_norm_rope(kv.Shape(1, 4, 4), x, None, torch.tensor([3, 4], dtype=torch.int32, device="cuda"), None, o, None, q_weight=w)
    assert not o.any()


def test_one_side_alone_and_in_place():
    import torch
    import paper_2506_08018_amd as kv
    shape = kv.Shape(1, 8, 2)
    freqs = torch.tensor(kv.rope_frequencies(128)[0], device="cuda")
    pos = torch.arange(5, dtype=torch.int32, device="cuda") * 1000
    x = torch.randn((5, 8, 128), device="cuda").half()
    k = torch.randn((5, 2, 128), device="cuda").half()
    a, b = torch.zeros_like(x), torch.zeros_like(k)
    kv.qk_norm_rope(shape, x, k, pos, freqs, a, b)
    only = torch.zeros_like(k)
    kv.qk_norm_rope(shape, None, k, pos, freqs, None, only)
    assert torch.equal(only, b)
    kv.qk_norm_rope(shape, x, k, pos, freqs, x, k)             # over the inputs
    assert torch.equal(x, a) and torch.equal(k, b)
    kv.qk_norm_rope(shape, x[:0], None, pos[:0], freqs, a[:0], None)
    one = torch.randn((1, 128), device="cuda").half().expand(4, 8, 128)            # one row for all heads and tokens
    out = torch.zeros((4, 8, 128), dtype=torch.float16, device="cuda")
    kv.qk_norm_rope(shape, one, None, torch.zeros(4, dtype=torch.int32, device="cuda"), freqs, out, None)
    assert torch.equal(out, one.contiguous())                 # position 0 turns nothing


def test_scores_depend_on_distances_alone():
    """q at position a + s, k at b + s: the same product for every s, as far as fp16 outputs tell (each is rounded by up to 2^-11 of its value)."""
    import torch
    import paper_2506_08018_amd as kv
    shape = kv.Shape(1, 1, 1)
    freqs = torch.tensor(kv.rope_frequencies(128, 500000.0)[0], device="cuda")
    q, k = torch.randn((1, 1, 128), device="cuda"), torch.randn((1, 1, 128), device="cuda")
    for interleaved in (False, True):
        got = []
        for s in (0, 1, 777, 131072, 10 ** 6):
            a, b = torch.zeros((1, 1, 128), dtype=torch.float16, device="cuda"), torch.zeros((1, 1, 128), dtype=torch.float16, device="cuda")
            kv.qk_norm_rope(shape, q, None, torch.tensor([40 + s], dtype=torch.int32, device="cuda"), freqs, a, None, interleaved=interleaved)
            kv.qk_norm_rope(shape, None, k, torch.tensor([9 + s], dtype=torch.int32, device="cuda"), freqs, None, b, interleaved=interleaved)
            got.append((a.double() * b.double()).sum().item())
        # each factor off by half a step: at most 2 * 2^-11 * sum |q_i k_i| <= 2^-10 |q| |k|
        assert max(got) - min(got) <= 2 * 2 ** -10 * (q.norm() * k.norm()).item(), got


def test_frequencies_reach_the_kernel_scaled():
    import torch
    import paper_2506_08018_amd as kv
    for scaling, more in (("linear", {}), ("base", {}), ("turns", dict(original_len=8192, low=1.0, high=4.0)), ("index", dict(original_len=4096))):
        f, amplitude = kv.rope_frequencies(64, 10000.0, scaling, 4.0, **more)
        x = torch.randn((3, 2, 128), device="cuda").half()
        o = torch.zeros_like(x)
        pos = torch.tensor([5, 20000, 99999], dtype=torch.int32)
        kv.qk_norm_rope(kv.Shape(1, 2, 2), x, None, pos.cuda(), torch.tensor(f, device="cuda"), o, None, amplitude=amplitude)
        want = definition(x.float().cpu().numpy(), None, 0, pos.numpy(), np.array(f), False, np.float64(np.float32(amplitude)))
        close(o.cpu().numpy(), want, np.abs(want).max(-1, keepdims=True))
        assert amplitude == pytest.approx(0.1 * math.log(4.0) + 1 if scaling == "index" else 1.0)
