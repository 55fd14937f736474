"""KVmix hot path on MI355X: thin Python binding over the C-ABI library libkvmix.so.

Every step of the path runs in the HIP kernels of csrc/; this package only marshals arguments.
PyTorch is used for device memory and streams.
"""
from .binding import (KVMixError, LayerCache, LayerCfg, PagedCache, Pages, Shape, append, append_tokens, cache_bytes, copy_windows, decode_attn,
                      decode_attn_static, decode_step, dequant, flush, lib, move_records, paged_append, paged_decode_attn,
                      paged_workspace_bytes, pages_compact, pages_fork, pages_free, pages_grow, qk_norm_rope, quantize_pack,
                      rope_frequencies, rpc_next, stream_read, strerror, version, workspace_bytes)

__all__ = ["KVMixError", "LayerCache", "LayerCfg", "PagedCache", "Pages", "Shape", "append", "append_tokens", "cache_bytes", "copy_windows",
           "decode_attn", "decode_attn_static", "decode_step", "dequant", "flush", "lib", "move_records", "paged_append",
           "paged_decode_attn", "paged_workspace_bytes", "pages_compact", "pages_fork", "pages_free", "pages_grow",
           "qk_norm_rope", "quantize_pack", "rope_frequencies", "rpc_next", "stream_read", "strerror", "version",
           "workspace_bytes"]
