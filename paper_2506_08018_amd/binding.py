"""ctypes marshalling for include/kvmix.h. No arithmetic of the method lives here."""
import ctypes as C
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libkvmix.so")
_lib = None


class KVMixError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


class Shape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "Hq", "Hkv", "D", "group")]

    def __init__(self, B, Hq, Hkv, D=128, group=32):
        super().__init__(B, Hq, Hkv, D, group)

    @property
    def units(self):
        return self.B * self.Hkv


class LayerCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("k_bits", "v_bits", "window")]


class _CacheStruct(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("packed", "k_win", "v_win")] + \
               [(n, C.c_int32) for n in ("T_cap", "W_cap", "n_q", "n_w", "w0", "v_lead")]


def lib():
    """Load libkvmix.so (built in-tree by paper_2506_08018_amd/build.py). Fails loudly when it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2506_08018_amd.build` "
                              "(there is no CPU fallback)")
        # PyTorch first: it brings its own copy of the HIP runtime, and the buffers handed to this library are torch's.
        # Loaded the other way round, the library binds to another copy of the runtime, to which torch's pointers
        # mean nothing (every launch then fails with a HIP error).
        import torch  # noqa: F401
        L = C.CDLL(_LIB_PATH)
        P, I, I64, SZ = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
        L.kvmix_version.restype = I
        L.kvmix_strerror.restype = C.c_char_p
        L.kvmix_strerror.argtypes = [I]
        L.kvmix_last_hip_error.restype = I
        L.kvmix_cache_bytes.restype = I
        L.kvmix_cache_bytes.argtypes = [P, P, I, I, P, P]
        L.kvmix_workspace_bytes.restype = I
        L.kvmix_workspace_bytes.argtypes = [P, I, P]
        L.kvmix_quantize_pack.restype = I
        L.kvmix_quantize_pack.argtypes = [P, P, P, P, I64, I64, I64, I, I, P, P]
        L.kvmix_append.restype = I
        L.kvmix_append.argtypes = [P, P, P, P, P, P]
        L.kvmix_append_tokens.restype = I
        L.kvmix_append_tokens.argtypes = [P, P, P, P, I64, I64, I64, I, P, P]
        L.kvmix_decode_attn.restype = I
        L.kvmix_decode_attn.argtypes = [P, P, P, P, C.c_float, P, P, SZ, I, P]
        L.kvmix_decode_attn_static.restype = I
        L.kvmix_decode_attn_static.argtypes = [P, P, P, P, C.c_float, P, I, P]
        L.kvmix_decode_step.restype = I
        L.kvmix_decode_step.argtypes = [P, P, P, P, P, P, C.c_float, P, P, SZ, I, P]
        L.kvmix_stream_read.restype = I
        L.kvmix_stream_read.argtypes = [P, SZ, I, I, P, P]
        L.kvmix_rpc_next.restype = I
        L.kvmix_rpc_next.argtypes = [C.c_double, C.c_double, I, I, P, P]
        L.kvmix_flush.restype = I
        L.kvmix_flush.argtypes = [P, P, P, I, I, P]
        for name, args in (("kvmix_pages_grow", [P, P, P, I, P]), ("kvmix_pages_free", [P, P, I, P]), ("kvmix_pages_fork", [P, P, P, I, P]),
                           ("kvmix_pages_compact", [P, P]), ("kvmix_move_records", [P] * 5), ("kvmix_copy_windows", [P] * 5 + [I, P]),
                           ("kvmix_paged_append", [P, P] + [P, I64, I64] * 2 + [I] + [P] * 4 + [I, P]), ("kvmix_paged_workspace_bytes", [P, I, P]),
                           ("kvmix_paged_decode_attn", [P] * 6 + [I, C.c_float, P, P, SZ, P]),
                           ("kvmix_rope_frequencies", [I, C.c_double, I, C.c_double, I, C.c_double, C.c_double, P, P]),
                           ("kvmix_qk_norm_rope", [P, P, I, I, P, P])):
            getattr(L, name).restype = I
            getattr(L, name).argtypes = args
        L.kvmix_dequant.restype = I
        L.kvmix_dequant.argtypes = [P, P, P, I, P, P]
        _lib = L
    return _lib


def version():
    return lib().kvmix_version()


def strerror(status):
    return lib().kvmix_strerror(int(status)).decode()


def _check(status, where):
    if status != 0:
        raise KVMixError(status, where)


_raw_stream = None      # torch's lookup of the current stream's handle, without a Stream object around it


def _stream(stream=None):
    """hipStream_t of torch's current stream, or of the given torch stream / raw handle."""
    if stream is None:
        global _raw_stream
        import torch
        if _raw_stream is None:
            _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
        return _raw_stream(torch.cuda.current_device())
    return stream if isinstance(stream, int) else stream.cuda_stream


def cache_bytes(shape, cfg, T_cap, W_cap):
    """-> dict of byte sizes: packed (the tile records), win (each of the two window arrays)."""
    out = [C.c_size_t(0) for _ in range(2)]
    _check(lib().kvmix_cache_bytes(C.byref(shape), C.byref(cfg), T_cap, W_cap, *[C.byref(o) for o in out]), "kvmix_cache_bytes")
    return dict(zip(("packed", "win"), (o.value for o in out)))


def workspace_bytes(shape, T_max):
    n = C.c_size_t(0)
    _check(lib().kvmix_workspace_bytes(C.byref(shape), T_max, C.byref(n)), "kvmix_workspace_bytes")
    return n.value


class LayerCache:
    """One layer's cache: device buffers (torch uint8/int16 tensors) plus the host-side struct."""

    def __init__(self, shape, cfg, T_cap, W_cap, device="cuda"):
        import torch
        self.shape, self.cfg = shape, cfg
        sz = cache_bytes(shape, cfg, T_cap, W_cap)
        z = lambda n: torch.zeros(max(n, 16), dtype=torch.uint8, device=device)
        self.packed = z(sz["packed"])
        self.k_win, self.v_win = z(sz["win"]), z(sz["win"])
        self.c = _CacheStruct(self.packed.data_ptr(), self.k_win.data_ptr(), self.v_win.data_ptr(), T_cap, W_cap, 0, 0, 0, 0)

    v_lead = property(lambda self: self.c.v_lead)
    n_qv = property(lambda self: self.c.n_q + self.c.v_lead)
    n = property(lambda self: self.c.n_q + self.c.n_w)
    n_q = property(lambda self: self.c.n_q)
    n_w = property(lambda self: self.c.n_w)
    w0 = property(lambda self: self.c.w0)
    T_cap = property(lambda self: self.c.T_cap)
    W_cap = property(lambda self: self.c.W_cap)

    def nbytes(self):
        return sum(t.numel() for t in (self.packed, self.k_win, self.v_win))

    def set_window(self, k, v):
        """k, v: fp16 tensors [B][Hkv][n_w][128] (oldest first); plain copies into the ring, start slot 0."""
        import torch
        units, W = self.shape.units, self.c.W_cap
        n = k.shape[2]
        assert n <= W
        kw = self.k_win.view(torch.float16).view(units, W, 128)
        vw = self.v_win.view(torch.float16).view(units, W, 128)
        kw[:, :n, :] = k.reshape(units, n, 128)
        vw[:, :n, :] = v.reshape(units, n, 128)
        self.c.n_w = n
        self.c.w0 = 0


def quantize_pack(shape, cfg, k, v, cache, t0=None):
    """k, v: fp16 CUDA tensors [B][Hkv][n_tokens][128] (last dim contiguous). Writes at token offset t0
    (default n_q) and advances cache.n_q."""
    assert k.dtype == v.dtype and k.element_size() == 2 and k.stride(3) == 1 and v.stride() == k.stride()
    n = k.shape[2]
    if t0 is None:
        t0 = cache.c.n_q
    st = lib().kvmix_quantize_pack(C.byref(shape), C.byref(cfg), k.data_ptr(), v.data_ptr(), k.stride(2), k.stride(1),
                                   k.stride(0), n, t0, C.byref(cache.c), _stream())
    _check(st, "kvmix_quantize_pack")
    cache.c.n_q = max(cache.c.n_q, t0 + n)


def append(shape, cfg, k_new, v_new, cache):
    """k_new, v_new: fp16 CUDA tensors [B][Hkv][128], contiguous."""
    assert k_new.is_contiguous() and v_new.is_contiguous()
    _check(lib().kvmix_append(C.byref(shape), C.byref(cfg), k_new.data_ptr(), v_new.data_ptr(), C.byref(cache.c), _stream()),
           "kvmix_append")


def append_tokens(shape, cfg, k_new, v_new, cache):
    """k_new, v_new: fp16 CUDA tensors [B][Hkv][n][128] (last dim contiguous, any strides otherwise)."""
    strides, size = k_new.stride(), k_new.shape
    assert k_new.element_size() == 2 and strides[3] == 1 and v_new.stride() == strides and v_new.shape == size
    st = lib().kvmix_append_tokens(C.byref(shape), C.byref(cfg), k_new.data_ptr(), v_new.data_ptr(), strides[2],
                                   strides[1], strides[0], size[2], C.byref(cache.c), _stream())
    _check(st, "kvmix_append_tokens")


def decode_attn(shape, cfg, q, cache, out, workspace=None, softmax_scale=0.0, n_splits=0, stream=None):
    """q, out: fp16 CUDA tensors [B][Hq][128], contiguous. workspace: uint8 CUDA tensor (zeroed once, and again for another shape) or None.
    stream: torch stream or raw hipStream_t handle (default: torch's current stream)."""
    assert q.is_contiguous() and out.is_contiguous()
    wp, wn = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (None, 0)
    st = lib().kvmix_decode_attn(C.byref(shape), C.byref(cfg), q.data_ptr(), C.byref(cache.c), C.c_float(softmax_scale),
                                 out.data_ptr(), wp, wn, n_splits, _stream(stream))
    _check(st, "kvmix_decode_attn")
    return out


def decode_attn_static(shape, cfg, q, cache, out, softmax_scale=0.0, n_splits=0, stream=None):
    """decode_attn without a workspace argument: the split partials live in the library's own fixed device array."""
    assert q.is_contiguous() and out.is_contiguous()
    st = lib().kvmix_decode_attn_static(C.byref(shape), C.byref(cfg), q.data_ptr(), C.byref(cache.c), C.c_float(softmax_scale),
                                        out.data_ptr(), n_splits, _stream(stream))
    _check(st, "kvmix_decode_attn_static")
    return out


def decode_step(shape, cfg, k_new, v_new, q, cache, out, workspace=None, softmax_scale=0.0, n_splits=0, stream=None):
    """append(k_new, v_new) followed by decode_attn(q), in one launch unless the window overflows."""
    assert k_new.is_contiguous() and v_new.is_contiguous() and q.is_contiguous() and out.is_contiguous()
    wp, wn = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (None, 0)
    st = lib().kvmix_decode_step(C.byref(shape), C.byref(cfg), k_new.data_ptr(), v_new.data_ptr(), q.data_ptr(),
                                 C.byref(cache.c), C.c_float(softmax_scale), out.data_ptr(), wp, wn, n_splits, _stream(stream))
    _check(st, "kvmix_decode_step")
    return out


def rpc_next(r_k, r_v, current_k, current_v):
    """(num_k, num_v) = floor(r * current) for a layer's Keys and Values."""
    nk, nv = C.c_int(0), C.c_int(0)
    _check(lib().kvmix_rpc_next(float(r_k), float(r_v), int(current_k), int(current_v), C.byref(nk), C.byref(nv)), "kvmix_rpc_next")
    return nk.value, nv.value


def flush(shape, cfg, cache, keep_k, keep_v, stream=None):
    """Quantize the Keys / Values that are no longer among the keep_k / keep_v most recent ones."""
    _check(lib().kvmix_flush(C.byref(shape), C.byref(cfg), C.byref(cache.c), int(keep_k), int(keep_v), _stream(stream)), "kvmix_flush")


def stream_read(buf, workgroups, threads=768, nbytes=None, sink=None, stream=None):
    """Load-only pass over the first nbytes (default: all) of the CUDA tensor `buf` in the attention kernel's launch shape."""
    n = buf.numel() * buf.element_size() if nbytes is None else int(nbytes)
    st = lib().kvmix_stream_read(buf.data_ptr(), n, workgroups, threads, sink.data_ptr() if sink is not None else None, _stream(stream))
    _check(st, "kvmix_stream_read")


def dequant(shape, cfg, cache, which, out):
    """out: fp32 CUDA tensor [units][n_q (Keys) or n_q + v_lead (Values)][128]."""
    _check(lib().kvmix_dequant(C.byref(shape), C.byref(cfg), C.byref(cache.c), which, out.data_ptr(), _stream()), "kvmix_dequant")
    return out


# ---- the paged cache
class _PagesStruct(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("table", "lens", "grown", "refs", "used", "status", "moves")] + \
               [(n, C.c_int32) for n in ("n_slots", "n_pages", "max_tiles", "window")]


class _PagedCacheStruct(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("pool", "k_win", "v_win")] + [(n, C.c_int32) for n in ("n_pages", "n_slots", "W_cap")]


# Host time per call, a launch included, is as long as the smaller kernels: tensors are asked for as little as their checks need, structures that a
# program keeps have their reference made once (one token of qk_norm_rope 9.7 -> 7.3 us a pass).
_types = None


def _torch_types():
    """(int32, fp16, fp32, {type: kvmix_dtype}) of torch, which is imported when it is first needed."""
    global _types
    if _types is None:
        import torch
        _types = (torch.int32, torch.float16, torch.float32, {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2})
    return _types


def _int32(t, n, what):
    """Device address of a contiguous int32 tensor of at least n elements; None stays None."""
    if t is None:
        return None
    assert t.dtype is (_types or _torch_types())[0] and t.is_contiguous() and t.numel() >= n, f"{what}: contiguous int32, {n} elements at least"
    return t.data_ptr()


class Pages:
    """Which sequence holds which pages, for all layers: int32 tensors table [n_slots][max_tiles], lens, grown [n_slots], refs [n_pages],
    used [(n_pages + 31) // 32], status [1], moves [4 + 3 n_pages]. buffers: some of them, where the caller has them already (the others
    are made, empty; `moves` only when pages_compact is first called)."""

    def __init__(self, n_slots, n_pages, max_tiles, window, device="cuda", buffers=None):
        import torch
        sizes = dict(table=n_slots * max_tiles, lens=n_slots, grown=n_slots, refs=n_pages, used=(n_pages + 31) // 32, status=1)
        shapes = dict(table=(n_slots, max_tiles))
        self.n_slots, self.n_pages, self.max_tiles, self.window, self.device = n_slots, n_pages, max_tiles, window, device
        given = dict(buffers or {})
        for name, n in sizes.items():
            t = given.pop(name, None)
            if t is None:
                t = torch.zeros(shapes.get(name, (n,)), dtype=torch.int32, device=device)
            setattr(self, name, t)
        self.moves = given.pop("moves", None)
        assert not given, f"unknown buffers {sorted(given)}"
        self.c = _PagesStruct(*[_int32(getattr(self, name), n, name) for name, n in sizes.items()], _int32(self.moves, 4 + 3 * n_pages, "moves"),
                              n_slots, n_pages, max_tiles, window)
        self.ref = C.byref(self.c)

    def _with_moves(self):
        if self.moves is None:
            import torch
            self.moves = torch.zeros(4 + 3 * self.n_pages, dtype=torch.int32, device=self.device)
            self.c.moves = self.moves.data_ptr()
        return self.ref


class PagedCache:
    """One layer of a paged cache: pool int32 [n_pages][Hkv][record words], k_win and v_win fp16 [n_slots][Hkv][W_cap][128]. buffers: as for
    Pages (a layer whose rings alone, or whose pool alone, a call touches may have the rest left out: buffers names those that are there)."""

    def __init__(self, shape, cfg, n_pages, n_slots, W_cap, device="cuda", buffers=None):
        import torch
        words = cache_bytes(shape, cfg, 32, max(W_cap, 32))["packed"] // (4 * shape.units)
        made = dict(pool=lambda: torch.zeros((n_pages, shape.Hkv, words), dtype=torch.int32, device=device),
                    k_win=lambda: torch.zeros((n_slots, shape.Hkv, W_cap, 128), dtype=torch.float16, device=device))
        made["v_win"] = made["k_win"]
        sizes = dict(pool=n_pages * shape.Hkv * words * 4, k_win=n_slots * shape.Hkv * W_cap * 256, v_win=n_slots * shape.Hkv * W_cap * 256)
        for name, make in made.items():
            t = make() if buffers is None else buffers.get(name)
            assert t is None or (t.is_contiguous() and t.numel() * t.element_size() >= sizes[name]), f"{name}: {sizes[name]} contiguous bytes expected"
            setattr(self, name, t)
        self.n_pages, self.n_slots, self.W_cap = n_pages, n_slots, W_cap
        self.c = _PagedCacheStruct(*[None if t is None else t.data_ptr() for t in (self.pool, self.k_win, self.v_win)], n_pages, n_slots, W_cap)
        self.ref = C.byref(self.c)


def pages_grow(pages, rows=None, cu=None, n_rows=None, stream=None):
    """Rows (slots; None: row b is slot b) get room for cu[b + 1] - cu[b] more tokens each (None: one). n_rows: as many as rows or cu name,
    every slot if neither is given."""
    n = n_rows if n_rows is not None else rows.numel() if rows is not None else cu.numel() - 1 if cu is not None else pages.n_slots
    _check(lib().kvmix_pages_grow(pages.ref, _int32(rows, n, "rows"), _int32(cu, n + 1, "cu"), n, _stream(stream)), "kvmix_pages_grow")


def pages_free(pages, rows, stream=None):
    """The slots in `rows` are empty again, pages that nobody else holds are free."""
    _check(lib().kvmix_pages_free(pages.ref, _int32(rows, 0, "rows"), rows.numel(), _stream(stream)), "kvmix_pages_free")


def pages_fork(pages, src, dst, stream=None):
    """Slot dst[i], empty, becomes a second holder of the pages of src[i] (rings: copy_windows, per layer)."""
    n = src.numel()
    _check(lib().kvmix_pages_fork(pages.ref, _int32(src, n, "src"), _int32(dst, n, "dst"), n, _stream(stream)), "kvmix_pages_fork")


def pages_compact(pages, stream=None):
    """Pages in use move to the lowest ids; every layer's records follow by move_records."""
    _check(lib().kvmix_pages_compact(pages._with_moves(), _stream(stream)), "kvmix_pages_compact")


def move_records(shape, cfg, cache, pages, stream=None):
    """One layer's records after pages_compact."""
    _check(lib().kvmix_move_records(C.byref(shape), C.byref(cfg), cache.ref, pages.ref, _stream(stream)), "kvmix_move_records")


def copy_windows(shape, cfg, cache, src, dst, stream=None):
    """Both fp16 rings of slot src[i] to slot dst[i]."""
    n = src.numel()
    st = lib().kvmix_copy_windows(C.byref(shape), C.byref(cfg), cache.ref, _int32(src, n, "src"), _int32(dst, n, "dst"), n, _stream(stream))
    _check(st, "kvmix_copy_windows")


def paged_append(shape, cfg, k_new, v_new, cache, pages, rows=None, cu=None, max_new=1, stream=None):
    """k_new, v_new: fp16 CUDA tensors [tokens][Hkv][128] (last dim contiguous, any strides otherwise), the tokens [cu[b], cu[b + 1]) of batch row b, at most max_new
    each (cu None: token b), for which pages_grow has made room."""
    half, ks, vs, size = (_types or _torch_types())[1], k_new.stride(), v_new.stride(), k_new.shape
    assert k_new.dtype is half and v_new.dtype is half and ks[2] == vs[2] == 1 and v_new.shape == size and size[1:] == (shape.Hkv, 128)
    st = lib().kvmix_paged_append(C.addressof(shape), C.addressof(cfg), k_new.data_ptr(), ks[0], ks[1], v_new.data_ptr(), vs[0], vs[1], size[0], cache.ref,
                                  pages.ref, _int32(rows, shape.B, "rows"), _int32(cu, shape.B + 1, "cu"), max_new, _stream(stream))
    _check(st, "kvmix_paged_append")


def paged_workspace_bytes(shape, max_len):
    n = C.c_size_t(0)
    _check(lib().kvmix_paged_workspace_bytes(C.byref(shape), max_len, C.byref(n)), "kvmix_paged_workspace_bytes")
    return n.value


def paged_decode_attn(shape, cfg, q, cache, pages, out, workspace=None, rows=None, max_len=0, softmax_scale=0.0, stream=None):
    """q, out: fp16 CUDA tensors [B][Hq][128], contiguous; row b attends to slot rows[b]'s tokens, max_len at most (0: what a table row holds).
    workspace: uint8 CUDA tensor of paged_workspace_bytes, zeroed once."""
    assert q.is_contiguous() and out.is_contiguous()
    wp, wn = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (None, 0)
    st = lib().kvmix_paged_decode_attn(C.addressof(shape), C.addressof(cfg), q.data_ptr(), cache.ref, pages.ref, _int32(rows, shape.B, "rows"),
                                       max_len, softmax_scale, out.data_ptr(), wp, wn, _stream(stream))
    _check(st, "kvmix_paged_decode_attn")
    return out


_rope_struct = struct.Struct("PiiffPP" + "PPqq" * 3).pack      # kvmix_rope


ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "turns": 3, "index": 4}


def rope_frequencies(rotary_dim, base=10000.0, scaling="plain", factor=1.0, original_len=0, low=1.0, high=32.0):
    """-> (rotary_dim // 2 floats: radians per position of each pair, factor for cosine and sine). Scalings: include/kvmix.h."""
    out, amplitude = (C.c_float * 64)(), C.c_float(0.0)
    _check(lib().kvmix_rope_frequencies(rotary_dim, base, ROPE_SCALINGS.get(scaling, -1), factor, original_len, low, high, out, C.byref(amplitude)),
           "kvmix_rope_frequencies")
    return list(out[:rotary_dim // 2]), amplitude.value


def qk_norm_rope(shape, q, k, positions, frequencies, q_out, k_out, v=None, v_out=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False,
                 amplitude=1.0, stream=None):
    """q [tokens][Hq][128], k, v [tokens][Hkv][128]: fp16, bf16 or fp32 CUDA tensors of one type (last dim contiguous, any strides otherwise);
    outputs fp16, contiguous. Heads are normed where a weight [128] is given, and the first 2 * len(frequencies) channels rotated (frequencies
    None: none); v is converted only. Any of q, k, v may be None."""
    _, half, single, codes = _types or _torch_types()
    some = q if q is not None else k if k is not None else v
    if some is None:
        return
    n, dtype = some.shape[0], some.dtype
    sides = []
    for x, o, heads in ((q, q_out, shape.Hq), (k, k_out, shape.Hkv), (v, v_out, shape.Hkv)):
        if x is None:
            sides += (0, 0, 0, 0)
            continue
        strides = x.stride()
        assert x.dtype is dtype and x.shape == (n, heads, 128) and strides[2] == 1
        assert o.dtype is half and o.numel() == n * heads * 128 and o.is_contiguous()
        sides += (x.data_ptr(), o.data_ptr(), strides[0], strides[1])
    qw = kw = at = pairs = 0
    if q_weight is not None:
        assert q_weight.dtype is dtype and q_weight.numel() == 128 and q_weight.is_contiguous()
        qw = q_weight.data_ptr()
    if k_weight is not None:
        assert k_weight.dtype is dtype and k_weight.numel() == 128 and k_weight.is_contiguous()
        kw = k_weight.data_ptr()
    if frequencies is not None:
        assert frequencies.dtype is single and frequencies.is_contiguous()
        at, pairs = frequencies.data_ptr(), frequencies.numel()
    rope = _rope_struct(at, 2 * pairs, interleaved, amplitude, eps, qw, kw, *sides)
    st = lib().kvmix_qk_norm_rope(C.addressof(shape), rope, codes.get(dtype, -1), n, _int32(positions, n, "positions"), _stream(stream))
    if st:
        _check(st, "kvmix_qk_norm_rope")
