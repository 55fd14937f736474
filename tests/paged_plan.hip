// The host side of kvmix_paged_decode_attn without a GPU: as a shared library in which the launch is taken down instead of made.
#include "../paper_2506_08018_amd/csrc/kvmix_api.hip"
#include "../paper_2506_08018_amd/csrc/kvmix_paged_api.hip"

namespace kvmix {
hipError_t launch_quantize_pack(QuantArgs, int, int, int, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_quantize_fronts(const QuantArgs&, int, int, int, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_append(const AppendArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_dequant(const DequantArgs&, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_stream_read(const void*, size_t, int, int, uint32_t*, hipStream_t) { return hipErrorUnknown; }
template <> hipError_t launch_decode_attn<8, false>(const AttnArgs&, int, int, int, int, hipStream_t) { return hipErrorUnknown; }
template <> hipError_t launch_decode_attn<12, false>(const AttnArgs&, int, int, int, int, hipStream_t) { return hipErrorUnknown; }
template <> hipError_t launch_decode_attn<12, true>(const AttnArgs&, int, int, int, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_paged_append(const PagedAppendArgs&, int, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_rope(const RopeArgs&, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_pages_grow(const kvmix_pages&, const int32_t*, const int32_t*, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_pages_free(const kvmix_pages&, const int32_t*, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_pages_fork(const kvmix_pages&, const int32_t*, const int32_t*, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_pages_compact(const kvmix_pages&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_copy(const CopyArgs&, hipStream_t) { return hipErrorUnknown; }
long long seen[6];
template <int W>
hipError_t note_paged(const PagedAttnArgs& a, const kvmix_pages&, const int32_t*, int n_rows, int pieces, int, int, int block, hipStream_t) {
  seen[0] = pieces; seen[1] = n_rows; seen[2] = block;
  seen[4] = a.share;
  seen[3] = a.part ? reinterpret_cast<char*>(a.part) - reinterpret_cast<char*>(a.counters) : 0;
  seen[5] = W;
  return hipSuccess;
}
template <> hipError_t launch_paged_attn<8>(const PagedAttnArgs& a, const kvmix_pages& p, const int32_t* r, int n, int pieces, int k, int v, int block, hipStream_t s) { return note_paged<8>(a, p, r, n, pieces, k, v, block, s); }
template <> hipError_t launch_paged_attn<12>(const PagedAttnArgs& a, const kvmix_pages& p, const int32_t* r, int n, int pieces, int k, int v, int block, hipStream_t s) { return note_paged<12>(a, p, r, n, pieces, k, v, block, s); }
}  // namespace kvmix

// One call; taken, of its last launch: pieces, batch rows, heads per block, bytes of counters, tiles of a share of one sequence, waves
extern "C" int paged_plan(int B, int Hkv, int G, int v_bits, int W, int max_len, size_t workspace_bytes, long long* taken) {
  const kvmix_shape sh{B, Hkv * G, Hkv, kD, kTile};
  const kvmix_layer_cfg cfg{2, v_bits, W};
  uint16_t* p = reinterpret_cast<uint16_t*>(4096);      // never followed
  int32_t* i = reinterpret_cast<int32_t*>(4096);
  const kvmix_paged_cache c{reinterpret_cast<uint32_t*>(p), p, p, 100, B, W + kTile};
  const kvmix_pages pages{i, i, i, i, reinterpret_cast<uint32_t*>(i), i, i, B, 100, 1 << 20, W};
  const int st = kvmix_paged_decode_attn(&sh, &cfg, p, &c, &pages, i, max_len, 0.0f, p, workspace_bytes ? p : nullptr, workspace_bytes, nullptr);
  for (int k = 0; k < 6; k++) taken[k] = seen[k];
  return st;
}
