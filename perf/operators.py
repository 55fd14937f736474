"""Performance cases of the paged cache: ragged sequences in pages of mixed-bit tiles, as a serving program steps them.

A page is one tile of 32 tokens, of all kv heads: pool[n_pages][Hkv][record], the records of include/kvmix.h. Sequence slot s has the
page ids table[s][0 .. P - 1] and lens[s] tokens, of which the oldest 32 P are packed, P = 0 below window + 32 tokens and
(lens - window) // 32 from there on; token t behind them is row t % W_cap of the slot's two fp16 rings. refs[p] counts the slots that
hold page p, bit p % 32 of used[p // 32] says that there is one.

Kinds
  rope    norm of every query and Key head, rotation by the token's position, conversion to the cache's fp16
  append  new tokens of a ragged batch into rings and pages (lens holds the lengths with them)
  attn    one new token of every sequence over its pages and its ring
  pages   bookkeeping of sequences that come and go: `admit` frees slots and grows others, `children` frees forks, forks their parents
          again and copies the rings, `turnover` frees slots, closes the gaps that they leave in the pool and grows them anew
"""
import functools
import math
import random

import torch

own = False

DEVICE = "cuda"
D = 128
TILE = 32
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # the newest token of a lone sequence on its way into one layer: nothing but a launch
        dict(name="rope_one_token", kind="rope", dtype="fp16", N=1, Hq=32, Hkv=8, rot=128, pairs="half", norm=False, far=4096, factor=1.0),
        # a decode step of 64 sequences of a model that norms its heads, positions up to 128 k on stretched frequencies
        dict(name="rope_step_64", kind="rope", dtype="bf16", N=64, Hq=64, Hkv=8, rot=128, pairs="half", norm=True, far=131072, factor=8.0),
        # a prompt of 8191 tokens, half of each head rotated in neighbouring pairs
        dict(name="rope_prompt_8k", kind="rope", dtype="bf16", N=8191, Hq=32, Hkv=8, rot=64, pairs="next", norm=True, far=1000000, factor=1.0),
        # a decode step of 64 sequences: one token each, two of the rings on average have 32 tokens due
        dict(name="append_step_64", kind="append", B=64, Hkv=8, bits="2/2", W=128, lo=1, hi=4096, new=1, mix=11),
        # chunks of ragged prompts, some to empty slots, some behind what is there
        dict(name="append_prompts", kind="append", B=7, Hkv=8, bits="3/4", W=128, lo=1, hi=2048, new=8000, mix=12),
        # one small layer, one sequence: launch and latency
        dict(name="attn_one_small", kind="attn", B=1, Hq=32, Hkv=32, bits="2/2", W=32, lo=1024, hi=1024, pad=0, mix=1),
        # 16 ragged sequences of the grouped-query shape
        dict(name="attn_ragged_16", kind="attn", B=16, Hq=32, Hkv=8, bits="2/4", W=128, lo=64, hi=8192, pad=1, mix=2),
        # a large batch of middling lengths on the 70B-class shape
        dict(name="attn_batch_64", kind="attn", B=64, Hq=64, Hkv=8, bits="2/2", W=128, lo=2048, hi=4096, pad=0, mix=3),
        # one long sequence next to a short one
        dict(name="attn_long_32k", kind="attn", B=2, Hq=32, Hkv=8, bits="3/4", W=256, lo=32, hi=32768, pad=0, mix=4),
        # requests end, others start: table and counts of 256 slots
        dict(name="pages_admit", kind="pages", op="admit", S=256, Hkv=8, bits="2/2", W=128, lo=1, hi=4096, n=32, mix=21),
        # four continuations of each of 8 prompts, started over
        dict(name="pages_children", kind="pages", op="children", S=40, Hkv=8, bits="2/2", W=128, lo=512, hi=8192, n=32, mix=22),
        # a quarter of the sequences leave a fragmented pool, the rest moves down
        dict(name="pages_turnover", kind="pages", op="turnover", S=64, Hkv=8, bits="2/4", W=128, lo=512, hi=4096, n=16, mix=23),
    ]


def draw(rng):
    """A case of the same ranges: 1-64 sequences of 1-32768 tokens, 1-32 kv heads, groups of 1-72, 1-4 bits, windows of 0-256."""
    def log_int(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    while True:
        kind = rng.choice(["rope", "rope", "append", "append", "attn", "attn", "attn", "attn", "pages"])
        Hkv, mix = rng.choice([1, 2, 4, 8, 8, 16, 32]), rng.randrange(1 << 30)
        bits = "%d/%d" % (rng.choice([1, 2, 2, 3, 4]), rng.choice([1, 2, 2, 3, 4]))
        W, hi = 32 * rng.randint(0, 8), log_int(1, 32768)
        lo = rng.choice([0, 1, max(1, hi // 64), hi])
        if kind == "rope":
            c = dict(kind=kind, dtype=rng.choice(["fp16", "bf16", "bf16", "fp32"]), N=log_int(1, 8192), Hq=Hkv * rng.choice([1, 2, 4, 8]), Hkv=Hkv,
                     rot=16 * rng.randint(1, 8), pairs=rng.choice(["half", "next"]), norm=rng.random() < 0.5, far=log_int(16, 1000000),
                     factor=rng.choice([1.0, 4.0, 32.0]))
        elif kind == "append":
            c = dict(kind=kind, B=log_int(1, 64), Hkv=Hkv, bits=bits, W=W, lo=lo, hi=hi, new=rng.choice([1, 1, 5, log_int(1, 8000)]), mix=mix)
        elif kind == "attn":
            G = rng.choice([1, 1, 2, 4, 4, 8, 8, 16, 48, 72])
            if G > 8 and Hkv > 8:
                continue
            c = dict(kind=kind, B=log_int(1, 64), Hq=G * Hkv, Hkv=Hkv, bits=bits, W=W, lo=lo, hi=hi, pad=rng.choice([0, 0, 1]), mix=mix)
            if c["B"] * Hkv * (hi // TILE + 1) > 66000:
                continue
        else:
            op = rng.choice(["admit", "children", "turnover"])
            S = log_int(8, 128)
            c = dict(kind=kind, op=op, S=S, Hkv=min(Hkv, 8), bits=bits, W=W, lo=lo, hi=min(hi, 8192), n=max(1, S // 4) * (3 if op == "children" else 1), mix=mix)
            if S * c["Hkv"] * (c["hi"] // TILE + 1) > 100000:
                continue
        w = work(c)
        if 1 <= w["bytes"] <= 1.9e8 and w["flops"] <= 6.2e9:
            return c


def _bits(case):
    return tuple(int(b) for b in case["bits"].split("/"))


def _record_words(case):
    kb, vb = _bits(case)
    return 256 + 128 * kb + 128 * vb


def _packed_tiles(n, W):
    return 0 if n < W + TILE else (n - W) // TILE


def _log_ints(rng, n, lo, hi):
    """n lengths, even over their logarithm (0 as often as 1)."""
    a, b = max(lo, 1), max(hi, 1)
    return [min(hi, int(a * (b / a) ** rng.random()) if lo or rng.random() < 0.9 else 0) for _ in range(n)]


def _plan(case):
    """What the case alone decides: lengths and which slots."""
    rng, W = random.Random(case.get("mix", 0)), case.get("W", 0)
    if case["kind"] == "append":
        old = _log_ints(rng, case["B"], case["lo"], case["hi"])
        old[0] = case["hi"]
        new = [1] * case["B"] if case["new"] == 1 else _log_ints(rng, case["B"], 0, case["new"])
        if case["new"] > 1:
            new[-1] = case["new"]
            old[-1] = 0
        return dict(old=old, new=new, lens=[a + b for a, b in zip(old, new)])
    if case["kind"] == "attn":
        lens = _log_ints(rng, case["B"], case["lo"], case["hi"])
        lens[0] = case["hi"]
        return dict(lens=lens)
    S, n = case["S"], case["n"]
    lens = _log_ints(rng, S, case["lo"], case["hi"])
    if case["op"] == "children":
        parents = S - n
        src = [i % parents for i in range(n)]
        return dict(lens=[lens[s] for s in range(parents)] + [lens[s] for s in src], src=src, dst=list(range(parents, S)))
    return dict(lens=lens, rows=[rng.sample(range(S), n) for _ in range(2)])


def work(case):
    kind = case["kind"]
    if kind == "rope":
        el = case["N"] * (case["Hq"] + 2 * case["Hkv"]) * D
        return {"bytes": el * (4 if case["dtype"] == "fp32" else 2) + el * 2 + 4 * case["N"], "flops": 8 * el}
    p, W, rec = _plan(case), case["W"], 4 * _record_words(case)
    if kind == "append":
        nbytes = 0
        for old, new in zip(p["old"], p["new"]):
            due = _packed_tiles(old + new, W) - _packed_tiles(old, W)
            kept = min(new, old + new - TILE * _packed_tiles(old + new, W))
            nbytes += case["Hkv"] * (due * (TILE * 512 + rec) + kept * 1024)
        return {"bytes": nbytes, "flops": nbytes}
    if kind == "attn":
        G = case["Hq"] // case["Hkv"]
        nbytes = flops = 0
        for n in p["lens"]:
            t = _packed_tiles(n, W)
            nbytes += case["Hkv"] * (t * rec + (n - TILE * t) * 512 + G * 512)
            flops += case["Hq"] * n * 4 * D
        return {"bytes": nbytes, "flops": flops}
    tiles = [_packed_tiles(n, W) for n in p["lens"]]
    if case["op"] == "admit":          # ids read and counts cleared, counts set and ids written
        return {"bytes": 24 * sum(tiles[s] for s in p["rows"][0]) + 16 * case["n"], "flops": 0}
    if case["op"] == "children":
        ring = case["Hkv"] * _ring(case) * 1024
        return {"bytes": 36 * sum(tiles[s] for s in p["dst"]) + 2 * case["n"] * ring, "flops": 0}
    gone = sum(tiles[s] for s in p["rows"][0])
    moved = min(gone, sum(tiles) - gone) * gone // max(1, sum(tiles))      # about as many pages above the new end as gaps below it
    return {"bytes": 2 * moved * case["Hkv"] * rec + 24 * gone, "flops": 0}


def _ring(case):
    return case["W"] + 2 * TILE


# ------------------------------------------------------------------------------------------------------- layout of a tile record
@functools.lru_cache(maxsize=None)
def _places(side, bits, device):
    """Word and bit of the code of every (token, channel) of a tile inside its section, and of the third bit of 3-bit codes."""
    tau, d = torch.meshgrid(torch.arange(TILE), torch.arange(D), indexing="ij")
    if side == "k":
        kq, i, j, hh, slot = d % 32 // 8, 4 * (tau // 8) + tau % 4, d % 8 // 2, d % 2, d // 32 + 4 * (tau % 8 // 4)
    else:
        kq, i, j, hh, slot = tau // 8, d % 16, tau % 8 // 2, tau % 2, d // 16
    col = 16 * kq + i
    plane = (2 * col + j // 2, 16 * hh + 8 * (j % 2) + 2 * (slot % 4) + slot // 4)
    if bits == 1:
        parts = [(plane[0], plane[1], 0, 1)]
    elif bits == 4:
        parts = [(256 * (slot // 4) + 4 * col + j, 16 * hh + 4 * (slot % 4), 0, 15)]
    else:
        parts = [(4 * col + j, 16 * hh + 2 * slot, 0, 3)]
        if bits == 3:
            parts.append((256 + plane[0], plane[1], 2, 1))
    return [(w.reshape(-1).to(device), b.reshape(-1).to(device), up, mask) for w, b, up, mask in parts]


@functools.lru_cache(maxsize=None)
def _meta_places(device):
    """Half-words of scale and minimum of the Key group of a channel, and of the Value group (token, block)."""
    d = torch.arange(D)
    key = [2 * (4 * (d // 2) + f) + d % 2 for f in (0, 1)]
    tau, g = torch.meshgrid(torch.arange(TILE), torch.arange(4), indexing="ij")
    val = [(2 * (4 * (16 * g + tau // 2) + 2 + f) + tau % 2).reshape(-1) for f in (0, 1)]
    return [x.to(device) for x in key + val]


def _quantize(x, bits, dim):
    """Codes, scale and minimum (fp16) of groups of 32 along `dim`; x fp16."""
    x32 = x.float()
    mn, mx = x32.amin(dim, keepdim=True), x32.amax(dim, keepdim=True)
    mn = torch.where(mn == 0, torch.zeros_like(mn), mn)
    span = mx - mn
    top = 2 ** bits - 1
    scale = (span if bits == 1 else (span.double() / top).float()).clamp(max=65504.0).half()      # quotients in 64 bits, rounded: IEEE's
    step = scale.float()
    high = torch.full_like(step, float(top))
    if bits == 3:                    # in-group elements 10 and 21 have two bits over the same range
        shape = [1] * x.dim()
        shape[dim] = TILE
        two = torch.zeros(TILE, dtype=torch.bool, device=x.device)
        two[10] = two[21] = True
        two = two.view(shape)
        step = torch.where(two, ((step * 7.0).double() / 3.0).float(), step)
        high = torch.where(two, torch.full_like(step, 3.0), torch.full_like(step, 7.0))
    q = torch.round(((x32 - mn).double() / step).float())
    codes = torch.where(step == 0, torch.zeros_like(q), torch.minimum(q.clamp(min=0), high)).int()
    return codes, scale, mn.half()


def _pack(codes, side, bits, out):
    """codes [n][32 * 128] into the words of `out` [n][128 * bits] (int32)."""
    words = torch.zeros((codes.shape[0], 128 * bits), dtype=torch.int64, device=codes.device)
    for w, b, up, mask in _places(side, bits, codes.device):
        words.index_add_(1, w, ((codes.long() >> up) & mask) << b)
    out.copy_(torch.where(words >= 1 << 31, words - (1 << 32), words))


def _records(k, v, kb, vb):
    """Tile records [n][words] (int32) of k, v: fp16 [n][32][128]."""
    n = k.shape[0]
    rec = torch.empty((n, 256 + 128 * kb + 128 * vb), dtype=torch.int32, device=k.device)
    meta = torch.empty((n, 512), dtype=torch.float16, device=k.device)
    ks, kz, vs, vz = _meta_places(k.device)
    c, s, z = _quantize(k, kb, 1)
    meta[:, ks], meta[:, kz] = s[:, 0], z[:, 0]
    _pack(c.reshape(n, TILE * D), "k", kb, rec[:, 256:256 + 128 * kb])
    c, s, z = _quantize(v.reshape(n, TILE, 4, 32), vb, 3)
    meta[:, vs], meta[:, vz] = s.reshape(n, TILE * 4), z.reshape(n, TILE * 4)
    _pack(c.reshape(n, TILE * D), "v", vb, rec[:, 256 + 128 * kb:])
    rec[:, :256] = meta.view(torch.int32)
    return rec


def _unpack(words, side, bits):
    """Codes [..., 32, 128] of a section's words [..., 128 * bits] (int32), as floats."""
    got = 0
    for w, b, up, mask in _places(side, bits, words.device):
        got = got + (((words[..., w] >> b.int()) & mask) << up)
    return got.view(words.shape[:-1] + (TILE, D)).float()


def _dequantize(rec, kb, vb):
    """Keys and Values [..., 32, 128] that records stand for, in 32 bits."""
    ks, kz, vs, vz = _meta_places(rec.device)
    meta = rec[..., :256].contiguous().view(torch.float16).float()
    lead = rec.shape[:-1]

    def steps(s, bits, at):          # at: index of an element inside its group
        return torch.where((at == 10) | (at == 21), s * 7.0 / 3.0, s) if bits == 3 else s

    tau, d = torch.arange(TILE, device=rec.device).view(TILE, 1), torch.arange(D, device=rec.device) % 32
    k = _unpack(rec[..., 256:256 + 128 * kb], "k", kb) * steps(meta[..., ks].unsqueeze(-2), kb, tau) + meta[..., kz].unsqueeze(-2)
    s = meta[..., vs].view(lead + (TILE, 4, 1)).expand(lead + (TILE, 4, 32)).reshape(lead + (TILE, D))
    z = meta[..., vz].view(lead + (TILE, 4, 1)).expand(lead + (TILE, 4, 32)).reshape(lead + (TILE, D))
    v = _unpack(rec[..., 256 + 128 * kb:], "v", vb) * steps(s, vb, d) + z
    return k, v


# ---------------------------------------------------------------------------------------------------------------- inputs
def _frequencies(rot, factor, device):
    """Radians per position of each pair: base 10000, the slower pairs stretched for contexts `factor` times as long (a ramp over the turns
    that a pair makes in 8192 positions, 1 to 4)."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    turns = f * 8192 / (2 * math.pi)
    keep = ((turns - 1.0) / 3.0).clamp(0, 1)
    return (f * keep + f / factor * (1 - keep)).float().to(device)


def _keys(gen, shape, outliers):
    k = torch.randn(shape, generator=gen, device=DEVICE)
    return (k * outliers).half()


def _outliers(gen, Hkv):
    """[Hkv][1][128]: four channels of each kv head with ten times the magnitude of the others."""
    at = torch.rand((Hkv, D), generator=gen, device=DEVICE).argsort(1) < 4
    return torch.where(at, 10.0, 1.0).unsqueeze(1)


def _pool(gen, n_pages, case, outliers):
    kb, vb = _bits(case)
    pool = torch.empty((n_pages, case["Hkv"], _record_words(case)), dtype=torch.int32, device=DEVICE)
    some = min(n_pages, max(1, 4096 // case["Hkv"]))      # distinct pages; further ones repeat them in another order
    k = _keys(gen, (some, case["Hkv"], TILE, D), outliers)
    v = torch.randn(k.shape, generator=gen, device=DEVICE).half()
    rec = _records(k.view(-1, TILE, D), v.view(-1, TILE, D), kb, vb).view(some, case["Hkv"], -1)
    pick = torch.randint(0, some, (n_pages,), generator=gen, device=DEVICE)
    torch.index_select(rec, 0, pick, out=pool)
    return pool


def _rings(gen, S, case, outliers):
    k = _keys(gen, (S, case["Hkv"], _ring(case), D), outliers)
    return k, torch.randn(k.shape, generator=gen, device=DEVICE).half()


def _ids(gen, lens, W, max_tiles, n_pages, slots):
    """Page ids of the slots' tiles, in no order; -1 behind them."""
    table = torch.full((slots, max_tiles), -1, dtype=torch.int32, device=DEVICE)
    tiles = torch.tensor([_packed_tiles(n, W) for n in lens], device=DEVICE)
    mask = torch.arange(max_tiles, device=DEVICE) < tiles.unsqueeze(1)
    table[mask] = torch.randperm(n_pages, generator=gen, device=DEVICE)[:int(mask.sum())].int()
    return table


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEVICE)


def _used(refs):
    n = (refs.numel() + 31) // 32 * 32
    bits = torch.zeros(n, dtype=torch.int64, device=refs.device)
    bits[:refs.numel()] = (refs > 0).long()
    words = (bits.view(-1, 32) << torch.arange(32, device=refs.device)).sum(1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int()


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    st = dict(case=case)
    if case["kind"] == "rope":
        N, Hq, Hkv, t = case["N"], case["Hq"], case["Hkv"], DTYPES[case["dtype"]]
        # one projection's output, rows of query, Key and Value heads one after the other
        x = torch.randn((N, Hq + 2 * Hkv, D), generator=gen, device=DEVICE) * 1.5
        x[:, Hq:Hq + Hkv] *= _outliers(gen, Hkv).transpose(0, 1)
        x = x.to(t)
        start = torch.randint(0, case["far"], (1,), generator=gen, device=DEVICE)
        pos = torch.randint(0, case["far"], (N,), generator=gen, device=DEVICE) if N <= 64 else start + torch.arange(N, device=DEVICE)
        st.update(q=x[:, :Hq], k=x[:, Hq:Hq + Hkv], v=x[:, Hq + Hkv:], positions=pos.int(), freqs=_frequencies(case["rot"], case["factor"], DEVICE),
                  amplitude=1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0, qw=None, kw=None)
        if case["norm"]:
            st["qw"], st["kw"] = ((1.0 + 0.2 * torch.randn(D, generator=gen, device=DEVICE)).to(t) for _ in range(2))
        st.update(q_out=torch.zeros((N, Hq, D), dtype=torch.float16, device=DEVICE), k_out=torch.zeros((N, Hkv, D), dtype=torch.float16, device=DEVICE),
                  v_out=torch.zeros((N, Hkv, D), dtype=torch.float16, device=DEVICE))
        return st
    p, W = _plan(case), case["W"]
    lens = p["lens"]
    outl = _outliers(gen, case["Hkv"])
    tiles = [_packed_tiles(n, W) for n in lens]
    if case["kind"] in ("append", "attn"):
        B = case["B"]
        slots, max_tiles = B + 2, max(tiles) + 3
        n_pages = sum(tiles) + 5
        where = torch.randperm(slots, generator=gen, device=DEVICE)[:B]
        table = _ids(gen, lens, W, max_tiles, n_pages, B)
        st["table"] = torch.full((slots, max_tiles), -1, dtype=torch.int32, device=DEVICE)
        st["table"][where] = table
        st["lens"] = torch.zeros(slots, dtype=torch.int32, device=DEVICE)
        st["lens"][where] = _ints(lens)
        st["k_win"], st["v_win"] = _rings(gen, slots, case, outl)
        st["rows"] = where.int()
        if case["kind"] == "attn":
            st["pool"] = _pool(gen, n_pages, case, outl)
            st["rows"] = torch.cat([st["rows"], torch.full((case["pad"],), -1, dtype=torch.int32, device=DEVICE)])
            st["q"] = torch.randn((B + case["pad"], case["Hq"], D), generator=gen, device=DEVICE).half()
            st["out"] = torch.zeros_like(st["q"])
            st["max_len"] = max(lens)
        else:
            st["pool"] = torch.zeros((n_pages, case["Hkv"], _record_words(case)), dtype=torch.int32, device=DEVICE)
            cu = [0]
            for n in p["new"]:
                cu.append(cu[-1] + n)
            st["cu"], st["max_new"] = (None if case["new"] == 1 else _ints(cu)), max(p["new"])
            st["grown"] = torch.zeros(slots, dtype=torch.int32, device=DEVICE)
            st["grown"][where] = _ints(p["new"])
            # K as the rotation leaves it, V a slice of the projection's rows
            st["k"] = _keys(gen, (case["Hkv"], cu[-1], D), outl).transpose(0, 1).contiguous()
            st["v"] = torch.randn((cu[-1], 2 * case["Hkv"], D), generator=gen, device=DEVICE).half()[:, case["Hkv"]:]
            # what falls due and what stays, as the plain form's program knows from the lengths it keeps
            due = [(b, t) for b, (a, n) in enumerate(zip(p["old"], lens)) for t in range(_packed_tiles(a, W), _packed_tiles(n, W))]
            stay = [(b, t) for b, (a, n) in enumerate(zip(p["old"], lens)) for t in range(max(a, TILE * _packed_tiles(n, W)), n)]
            st["due"] = torch.tensor(due, dtype=torch.int64, device=DEVICE).view(-1, 2)
            st["stay"] = torch.tensor(stay, dtype=torch.int64, device=DEVICE).view(-1, 2)
            st["old"], st["first"] = torch.tensor(p["old"], device=DEVICE), torch.tensor(cu[:-1], device=DEVICE)
        return st
    S = case["S"]
    n_pages = sum(tiles) + 64
    max_tiles = max(tiles) + 1
    if case["op"] == "children":
        parents = S - case["n"]
        table = _ids(gen, lens[:parents], W, max_tiles, n_pages, parents)
        st["table"] = torch.cat([table, table[_ints(p["src"]).long()]])
        st["src"], st["dst"] = _ints(p["src"]), _ints(p["dst"])
        st["k_win"], st["v_win"] = _rings(gen, S, case, outl)
    else:
        st["table"] = _ids(gen, lens, W, max_tiles, n_pages, S)
        st["rows"], st["turn"] = [_ints(r) for r in p["rows"]], 0
        st["cu"] = [_ints([0] + [sum(lens[s] for s in r[:i + 1]) for i in range(len(r))]) for r in p["rows"]]
        if case["op"] == "turnover":
            st["pool"] = _pool(gen, n_pages, case, outl)
    st["lens"] = _ints(lens)
    st["grown"] = torch.zeros(S, dtype=torch.int32, device=DEVICE)
    ids = st["table"][torch.arange(max_tiles, device=DEVICE) < _ints(tiles).unsqueeze(1)].long()
    st["refs"] = torch.bincount(ids, minlength=n_pages).int()
    st["used"] = _used(st["refs"])
    st["status"] = torch.zeros(1, dtype=torch.int32, device=DEVICE)
    return st


# ---------------------------------------------------------------------------------------------------------------- the plain forms
def _turn(x, cos, sin, rot, pairs):
    """x [N][H][128] in 32 bits, cos and sin [N][1][rot / 2]."""
    y = x.clone()
    if pairs == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    return y


def _rope(st):
    c = st["case"]
    angle = st["positions"].double().view(-1, 1, 1) * st["freqs"].double()          # far positions lose their angle in 32 bits
    cos, sin = (angle.cos() * st["amplitude"]).float(), (angle.sin() * st["amplitude"]).float()
    out = []
    for x, w in ((st["q"], st["qw"]), (st["k"], st["kw"])):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        out.append(_turn(x, cos, sin, c["rot"], c["pairs"]).half())
    return out + [st["v"].half()]


def _append(st):
    c = st["case"]
    (kb, vb), cap, pool, rows = _bits(c), _ring(c), st["pool"], st["rows"].long()
    b, t = st["due"].unbind(1)
    tok = t.unsqueeze(1) * TILE + torch.arange(TILE, device=t.device)               # [due][32]
    is_new = (tok >= st["old"][b].unsqueeze(1)).view(-1, TILE, 1, 1)
    at = (st["first"][b].unsqueeze(1) + tok - st["old"][b].unsqueeze(1)).clamp(min=0, max=max(0, st["k"].shape[0] - 1))
    slot = rows[b].unsqueeze(1)
    k = torch.where(is_new, st["k"][at], st["k_win"][slot, :, tok % cap])           # [due][32][Hkv][128]
    v = torch.where(is_new, st["v"][at], st["v_win"][slot, :, tok % cap])
    n = b.shape[0] * c["Hkv"]
    rec = _records(k.transpose(1, 2).reshape(n, TILE, D), v.transpose(1, 2).reshape(n, TILE, D), kb, vb)
    pool[st["table"][rows[b], t].long()] = rec.view(b.shape[0], c["Hkv"], rec.shape[1])
    b, t = st["stay"].unbind(1)
    at = st["first"][b] + t - st["old"][b]
    st["k_win"][rows[b], :, t % cap] = st["k"][at]
    st["v_win"][rows[b], :, t % cap] = st["v"][at]
    return pool, st["k_win"], st["v_win"]


def _tiles_of(lens, W):
    return torch.where(lens < W + TILE, torch.zeros_like(lens), (lens - W) // TILE)


def _attn(st):
    c = st["case"]
    (kb, vb), W, cap = _bits(c), c["W"], _ring(c)
    rows = st["rows"].long().clamp(min=0)
    lens = torch.where(st["rows"] < 0, 0, st["lens"][rows])                         # [B]
    B, Hkv, G = lens.shape[0], c["Hkv"], c["Hq"] // c["Hkv"]
    T = _packed_tiles(st["max_len"], W)
    t = torch.arange(T, device=lens.device)
    tiles = _tiles_of(lens, W)
    in_page = t < tiles.unsqueeze(1)                                                # [B][T]
    rec = st["pool"][st["table"][rows, :T].clamp(min=0).long()]                     # [B][T][Hkv][words]
    k, v = _dequantize(rec, kb, vb)
    k, v = (x.transpose(1, 2).reshape(B, Hkv, T * TILE, D) for x in (k, v))
    w = torch.arange(min(W + TILE - 1, st["max_len"]), device=lens.device)
    tok = tiles.unsqueeze(1) * TILE + w                                             # ring tokens [B][R]
    slot = (tok % cap).long()
    kw, vw = (x[rows.unsqueeze(1), :, slot].transpose(1, 2).float() for x in (st["k_win"], st["v_win"]))
    live = torch.cat([in_page.repeat_interleave(TILE, 1), tok < lens.unsqueeze(1)], 1).view(B, 1, 1, -1)
    q = st["q"].float().view(B, Hkv, G, D)
    s = torch.matmul(q, torch.cat([k, kw], 2).transpose(2, 3).contiguous()) / math.sqrt(D)
    s = s.masked_fill(~live, -math.inf)
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    v = torch.cat([v, vw], 2).masked_fill(~live.view(B, 1, -1, 1), 0.0)
    o = torch.matmul(e, v) / torch.where(total == 0, 1.0, total)
    return torch.where((st["rows"] < 0).view(B, 1, 1), st["out"], o.view(B, c["Hq"], D).half())


def _free(st, rows):
    table, refs, W = st["table"], st["refs"], st["case"]["W"]
    rows = rows.long()
    held = torch.arange(table.shape[1], device=rows.device) < _tiles_of(st["lens"][rows], W).unsqueeze(1)
    refs.index_add_(0, table[rows].clamp(min=0).long().view(-1), -held.int().view(-1))
    st["lens"][rows] = 0
    st["grown"][rows] = 0


def _grow(st, rows, cu):
    """One more stretch of each row: the lowest free pages, in the order of the rows. (The cases have pages enough.)"""
    table, refs, W = st["table"], st["refs"], st["case"]["W"]
    rows = rows.long()
    n = cu[1:] - cu[:-1]
    before, after = _tiles_of(st["lens"][rows], W), _tiles_of(st["lens"][rows] + n, W)
    need = after - before
    first = torch.cumsum(need, 0) - need
    free = torch.argsort((refs > 0).int(), stable=True)
    col = torch.arange(table.shape[1], device=rows.device)
    mine = (col >= before.unsqueeze(1)) & (col < after.unsqueeze(1))
    ids = free[(first.unsqueeze(1) + col - before.unsqueeze(1)).clamp(min=0, max=refs.numel() - 1)].int()
    table[rows] = torch.where(mine, ids, table[rows])
    refs.index_add_(0, ids.long().view(-1), mine.int().view(-1))
    st["lens"][rows] += n
    st["grown"][rows] = n


def _fork(st, src, dst):
    table, W = st["table"], st["case"]["W"]
    src, dst = src.long(), dst.long()
    held = torch.arange(table.shape[1], device=src.device) < _tiles_of(st["lens"][src], W).unsqueeze(1)
    table[dst] = torch.where(held, table[src], table[dst])
    st["refs"].index_add_(0, table[src].clamp(min=0).long().view(-1), held.int().view(-1))
    st["lens"][dst] = st["lens"][src]
    st["grown"][dst] = 0


def _compact(st):
    """The live pages above the new end move into the gaps below it, in order; the records with them."""
    table, refs, W = st["table"], st["refs"], st["case"]["W"]
    live = refs > 0
    low = torch.arange(refs.numel(), device=refs.device) < live.sum()
    src, dst = torch.nonzero(live & ~low).view(-1), torch.nonzero(~live & low).view(-1)
    to = torch.arange(refs.numel(), device=refs.device, dtype=torch.int32)
    to[src] = dst.int()
    refs[dst] = refs[src]
    refs[src] = 0
    held = torch.arange(table.shape[1], device=refs.device) < _tiles_of(st["lens"], W).unsqueeze(1)
    table.copy_(torch.where(held, to[table.clamp(min=0).long()], table))
    st["pool"][dst] = st["pool"][src]


def _pages(st):
    op = st["case"]["op"]
    if op == "children":
        _free(st, st["dst"])
        _fork(st, st["src"], st["dst"])
        src, dst = st["src"].long(), st["dst"].long()
        st["k_win"][dst], st["v_win"][dst] = st["k_win"][src], st["v_win"][src]
        more = [st["k_win"], st["v_win"]]
    else:
        turn = st["turn"]
        st["turn"] = 1 - turn
        _free(st, st["rows"][turn])
        if op == "turnover":
            _compact(st)
        _grow(st, st["rows"][turn], st["cu"][turn])
        more = [st["pool"]] if op == "turnover" else []
    st["used"].copy_(_used(st["refs"]))
    return [st["table"], st["lens"], st["grown"], st["refs"], st["used"]] + more


# ---------------------------------------------------------------------------------------------------------------- the framework's calls
def _own_handles(st):
    """What a serving program builds once around its buffers."""
    import paper_2506_08018_amd as kv
    c = st["case"]
    h = dict(kv=kv, shape=kv.Shape(st["rows"].shape[0] if c["kind"] in ("append", "attn") else c.get("S", 1), c.get("Hq", c["Hkv"]), c["Hkv"]))
    if c["kind"] == "rope":
        return h
    kb, vb = _bits(c)
    S, max_tiles = st["table"].shape
    h["cfg"] = kv.LayerCfg(kb, vb, c["W"])
    n_pages = st["pool"].shape[0] if "pool" in st else st["refs"].numel()
    h["pages"] = kv.Pages(S, n_pages, max_tiles, c["W"], device=DEVICE, buffers={k: st[k] for k in ("table", "lens", "grown", "refs", "used", "status") if k in st})
    if c["kind"] != "pages" or c["op"] != "admit":
        h["cache"] = kv.PagedCache(h["shape"], h["cfg"], n_pages, S, _ring(c), device=DEVICE,
                                   buffers={k: st[k] for k in ("pool", "k_win", "v_win") if k in st})
    if c["kind"] == "attn":
        h["ws"] = torch.zeros(kv.paged_workspace_bytes(h["shape"], st["max_len"]), dtype=torch.uint8, device=DEVICE)
    return h


def _own_run(st):
    if "own" not in st:
        st["own"] = _own_handles(st)
    h, c = st["own"], st["case"]
    kv = h["kv"]
    if c["kind"] == "rope":
        kv.qk_norm_rope(h["shape"], st["q"], st["k"], st["positions"], st["freqs"], st["q_out"], st["k_out"], v=st["v"], v_out=st["v_out"],
                        q_weight=st["qw"], k_weight=st["kw"], eps=1e-6, interleaved=c["pairs"] == "next", amplitude=st["amplitude"])
        return [st["q_out"], st["k_out"], st["v_out"]]
    if c["kind"] == "append":
        kv.paged_append(h["shape"], h["cfg"], st["k"], st["v"], h["cache"], h["pages"], rows=st["rows"], cu=st["cu"], max_new=st["max_new"])
        return st["pool"], st["k_win"], st["v_win"]
    if c["kind"] == "attn":
        return kv.paged_decode_attn(h["shape"], h["cfg"], st["q"], h["cache"], h["pages"], st["out"], h["ws"], rows=st["rows"], max_len=st["max_len"])
    if c["op"] == "children":
        kv.pages_free(h["pages"], st["dst"])
        kv.pages_fork(h["pages"], st["src"], st["dst"])
        kv.copy_windows(h["shape"], h["cfg"], h["cache"], st["src"], st["dst"])
        more = [st["k_win"], st["v_win"]]
    else:
        turn = st["turn"]
        st["turn"] = 1 - turn
        kv.pages_free(h["pages"], st["rows"][turn])
        if c["op"] == "turnover":
            kv.pages_compact(h["pages"])
            kv.move_records(h["shape"], h["cfg"], h["cache"], h["pages"])
        kv.pages_grow(h["pages"], st["rows"][turn], st["cu"][turn])
        more = [st["pool"]] if c["op"] == "turnover" else []
    return [st["table"], st["lens"], st["grown"], st["refs"], st["used"]] + more


def run(state):
    if own:
        return _own_run(state)
    return dict(rope=_rope, append=_append, attn=_attn, pages=_pages)[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------------------------------------------- the definition in 64 bits
def _codes64(sec, bits, keys):
    """Codes [n][32][128] of sections [n][words], field by field."""
    n = sec.shape[0]
    out = torch.zeros((n, TILE, D), dtype=torch.float64, device=sec.device)
    for slot in range(8):
        for hh in range(2):
            for j in range(4):
                if bits == 4:
                    x = sec.view(n, 2, 64, 4)[:, slot // 4, :, j] >> (16 * hh + 4 * (slot % 4)) & 15
                elif bits != 1:
                    x = sec[:, :256].view(n, 64, 4)[:, :, j] >> (16 * hh + 2 * slot) & 3
                if bits in (1, 3):
                    y = sec[:, -128:].view(n, 64, 2)[:, :, j // 2] >> (16 * hh + 8 * (j % 2) + 2 * (slot % 4) + slot // 4) & 1
                    x = y if bits == 1 else x + 4 * y
                x = x.view(n, 4, 16).double()                                       # [n][kq][i]
                for kq in range(4):
                    if keys:         # tokens 8 a + 4 m + b of i = 4 a + b
                        out[:, :, 32 * (slot % 4) + 8 * kq + 2 * j + hh].view(n, 4, 2, 4)[:, :, slot // 4] = x[:, kq].view(n, 4, 4)
                    else:
                        out[:, 8 * kq + 2 * j + hh, 16 * slot:16 * slot + 16] = x[:, kq]
    return out


def _tiles64(rec, kb, vb):
    n = rec.shape[0]
    m = rec[:, :256].contiguous().view(torch.float16).double().view(n, 64, 4, 2)    # [n][column][field][half]
    ks, kz = (m[:, :, f].reshape(n, 1, D) for f in (0, 1))
    vs, vz = (m[:, :, 2 + f].reshape(n, 4, TILE).transpose(1, 2).unsqueeze(-1) for f in (0, 1))
    k, v = _codes64(rec[:, 256:256 + 128 * kb], kb, True), _codes64(rec[:, 256 + 128 * kb:], vb, False)
    if kb == 3:
        k[:, [10, 21]] *= 7.0 / 3.0
    if vb == 3:
        v.view(n, TILE, 4, 32)[..., [10, 21]] *= 7.0 / 3.0
    return k * ks + kz, (v.view(n, TILE, 4, 32) * vs + vz).reshape(n, TILE, D)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "rope":
        N, rot = case["N"], case["rot"]
        angle = st["positions"].double()[:, None, None] * st["freqs"].double()
        turn = torch.polar(torch.full_like(angle, st["amplitude"]), angle)
        out = []
        for x, w in ((st["q"], st["qw"]), (st["k"], st["kw"])):
            x = x.double()
            if w is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / D + 1e-6).sqrt() * w.double()
            head, tail = x[..., :rot], x[..., rot:]
            pair = head.unflatten(-1, (rot // 2, 2)) if case["pairs"] == "next" else head.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            z = z.flatten(-2) if case["pairs"] == "next" else z.transpose(-1, -2).flatten(-2)
            out.append(torch.cat([z, tail], -1))
        return out + [st["v"].double()]
    (kb, vb), W, cap, Hkv = _bits(case), case["W"], _ring(case), case["Hkv"]
    if case["kind"] == "append":       # records are whole words; a ring row is a copy
        p, at = _plan(case), 0
        for b, (old, n) in enumerate(zip(p["old"], p["lens"])):
            t = torch.arange(max(old, TILE * _packed_tiles(n, W)), n, device=DEVICE)
            for ring, x in ((st["k_win"], st["k"]), (st["v_win"], st["v"])):
                ring[int(st["rows"][b])][:, t % cap] = x[at + t - old].transpose(0, 1)
            at += n - old
        return [None, st["k_win"].double(), st["v_win"].double()]
    if case["kind"] == "pages":
        if case["op"] == "children":
            for a, b in zip(*(st[k].tolist() for k in ("src", "dst"))):
                st["k_win"][b], st["v_win"][b] = st["k_win"][a], st["v_win"][a]
            return [None] * 5 + [st["k_win"].double(), st["v_win"].double()]
        return None                    # whole numbers all
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(_plan(case)["lens"]):
        if n == 0:
            continue
        s, T = int(st["rows"][b]), _packed_tiles(n, W)
        ring = torch.arange(TILE * T, n, device=DEVICE) % cap
        rec = st["pool"][st["table"][s, :T].long()].transpose(0, 1).reshape(Hkv * T, _record_words(case))
        k, v = (torch.cat([x.view(Hkv, T * TILE, D), w[s][:, ring].double()], 1) for x, w in zip(_tiles64(rec, kb, vb), (st["k_win"], st["v_win"])))
        q = st["q"][b].double().view(Hkv, -1, D)
        out[b] = (torch.softmax(q @ k.transpose(1, 2).contiguous() / math.sqrt(D), -1) @ v).view(-1, D)
    return out
