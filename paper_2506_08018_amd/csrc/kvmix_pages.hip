// Bookkeeping of the paged cache (gfx950): lengths, page ids and page counts of sequences that come, fork and go, and the copies that
// moving pages and forked rings take. Integers only; contract: include/kvmix.h.
//
// What is free is one bit per page, and allocation takes the lowest free ids: frees and forks are then nothing but atomic
// additions and bit operations, whose order does not change what they leave, and the next grow finds its pages from the bits alone. (A
// stack of free ids would make the ids depend on the order in which frees of one call arrive.) All of these launches are bound by a
// launch and two or three dependent reads of memory, not by their bytes.
#include "kvmix_common.hpp"

namespace kvmix {

namespace {

constexpr int kGrowThreads = 1024;
constexpr int kMaxRows = 4096;                        // of one call of grow or fork
constexpr int kRowsEach = kMaxRows / kGrowThreads;
constexpr int kChunk = 4096;                          // page ids that are looked at together: four bits to a thread
constexpr int kMaxChunks = 1024;                      // 4 M pages

// sum over the workgroup's threads before this one; total: over all of them (all threads call it)
template <typename T>
__device__ T scan_before(T v, T* s_wave, T& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  T x = v;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const T y = __shfl_up(x, d);
    x += lane >= d ? y : 0;
  }
  __syncthreads();                                    // (s_wave may still be read)
  if (lane == kWave - 1) s_wave[wave] = x;
  __syncthreads();
  T before = 0, all = 0;
  for (int w = 0; w < waves; w++) {
    before += w < wave ? s_wave[w] : 0;
    all += s_wave[w];
  }
  total = all;
  return before + x - v;
}

__device__ __forceinline__ uint32_t valid_bits(int word, int n_pages) {
  const int left = n_pages - 32 * word;
  return left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u;
}

// One workgroup: rows first (what each needs, in their order), then as many of the lowest free ids as are granted, a chunk of 4096 pages at
// a time, chunks without a free page skipped. Ranks of free ids meet rows by binary search over the rows' first ranks.
__global__ __launch_bounds__(kGrowThreads) void pages_grow_kernel(kvmix_pages p, const int32_t* rows, const int32_t* cu, int n) {
  __shared__ int s_row[kMaxRows], s_first[kMaxRows], s_before[kMaxRows];
  __shared__ int s_id[kChunk];
  __shared__ int s_free[kMaxChunks];
  __shared__ int s_wave[kGrowThreads / kWave];
  __shared__ long long s_wave_needs[kGrowThreads / kWave];
  __shared__ int s_granted, s_status;
  const int tid = threadIdx.x, words = (p.n_pages + 31) / 32, chunks = (p.n_pages + kChunk - 1) / kChunk;
  if (tid == 0) { s_granted = 0; s_status = 0; }
  for (int c = tid; c < chunks; c += kGrowThreads) s_free[c] = 0;
  for (int i = tid; i < kMaxRows; i += kGrowThreads) s_row[i] = i < n ? (rows ? rows[i] : i) : -1;
  __syncthreads();
  int free_here = 0;
  for (int w = tid; w < words; w += kGrowThreads) {
    const int f = __popc(~p.used[w] & valid_bits(w, p.n_pages));
    free_here += f;
    if (f) atomicAdd(&s_free[w / (kChunk / 32)], f);
  }
  int status = 0, need[kRowsEach], len[kRowsEach], fresh[kRowsEach], tiles[kRowsEach];
  long long sum = 0;
  bool ok[kRowsEach];
#pragma unroll
  for (int e = 0; e < kRowsEach; e++) {
    const int i = tid * kRowsEach + e, row = s_row[i];
    ok[e] = false; need[e] = 0; len[e] = 0; fresh[e] = 0; tiles[e] = 0;
    if (i < n && row >= 0) {
      bool good = row < p.n_slots;
      for (int j = 0; j < i && good; j++) good = s_row[j] != row;
      if (good) {
        len[e] = p.lens[row];
        const int64_t add = cu ? (int64_t)cu[i + 1] - cu[i] : 1;
        good = len[e] >= 0 && add >= 0 && add + len[e] <= 0x7fffffff;
        fresh[e] = (int)add;
      }
      if (!good) status |= KVMIX_PAGES_BAD_ROW;
      if (good) {
        tiles[e] = packed_tiles(len[e], p.window);
        const int after = packed_tiles(len[e] + fresh[e], p.window);
        ok[e] = after <= p.max_tiles;
        if (ok[e]) need[e] = after - tiles[e];
        else { status |= KVMIX_PAGES_EXHAUSTED; p.grown[row] = 0; }
      }
    }
    sum += need[e];
  }
  int n_free;
  long long all;
  scan_before(free_here, s_wave, n_free);
  long long at = scan_before(sum, s_wave_needs, all);
#pragma unroll
  for (int e = 0; e < kRowsEach; e++) {
    const int i = tid * kRowsEach + e;
    s_first[i] = at < 0x7fffffff ? (int)at : 0x7fffffff; s_before[i] = tiles[e];
    at += need[e];
    const bool granted = ok[e] && (need[e] == 0 || at <= n_free);
    if (granted && need[e]) atomicMax(&s_granted, (int)at);
    if (granted) { p.lens[s_row[i]] = len[e] + fresh[e]; p.grown[s_row[i]] = fresh[e]; }
    else if (ok[e]) { p.grown[s_row[i]] = 0; status |= KVMIX_PAGES_EXHAUSTED; }
  }
  if (status) atomicOr(&s_status, status);
  __syncthreads();
  const int granted = s_granted;
  int base = 0;
  for (int c = 0; c < chunks && base < granted; c++) {
    if (s_free[c] == 0) continue;
    const int w = c * (kChunk / 32) + tid / 8, shift = 4 * (tid & 7);
    uint32_t free_bits = 0;
    if (w < words) free_bits = (~p.used[w] & valid_bits(w, p.n_pages)) >> shift & 15u;
    int in_chunk;
    int r = scan_before((int)__popc(free_bits), s_wave, in_chunk);
    uint32_t taken = 0;
#pragma unroll
    for (int b = 0; b < 4; b++)
      if (free_bits >> b & 1u) {
        if (base + r < granted) { s_id[r] = 32 * w + shift + b; taken |= 1u << b; }
        r++;
      }
    if (taken) atomicOr(&p.used[w], taken << shift);
    __syncthreads();
    const int here = in_chunk < granted - base ? in_chunk : granted - base;
    for (int k = tid; k < here; k += kGrowThreads) {
      int lo = 0, hi = n - 1;                          // the last row whose first rank is not past this one
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_first[mid] <= base + k) lo = mid;
        else hi = mid - 1;
      }
      p.table[(size_t)s_row[lo] * p.max_tiles + s_before[lo] + (base + k - s_first[lo])] = s_id[k];
      p.refs[s_id[k]] = 1;
    }
    base += here;
    __syncthreads();
  }
  if (tid == 0 && s_status) atomicOr(p.status, s_status);
}

// A workgroup per row. The length is taken out by an exchange, so that a slot that is named twice is freed once.
constexpr int kRowThreads = 256;
constexpr int kEach = 4;              // table entries of a thread under way together
__global__ __launch_bounds__(kRowThreads) void pages_free_kernel(kvmix_pages p, const int32_t* rows) {
  __shared__ int s_len;
  const int row = rows ? rows[blockIdx.x] : (int)blockIdx.x;
  if (row < 0) return;
  int status = 0;
  if (row >= p.n_slots) {
    status = KVMIX_PAGES_BAD_ROW;
  } else {
    if (threadIdx.x == 0) { s_len = atomicExch(&p.lens[row], 0); p.grown[row] = 0; }
    __syncthreads();
    int tiles = s_len > 0 ? packed_tiles(s_len, p.window) : 0;
    if (s_len < 0 || tiles > p.max_tiles) { status = KVMIX_PAGES_BAD_ROW; tiles = tiles > p.max_tiles ? p.max_tiles : 0; }
    const int32_t* ids = p.table + (size_t)row * p.max_tiles;
    for (int c0 = threadIdx.x; c0 < tiles; c0 += kEach * kRowThreads) {
      int id[kEach], old[kEach];
#pragma unroll
      for (int e = 0; e < kEach; e++) id[e] = c0 + e * kRowThreads < tiles ? ids[c0 + e * kRowThreads] : -1;
#pragma unroll
      for (int e = 0; e < kEach; e++) {
        old[e] = 2;
        if ((uint32_t)id[e] < (uint32_t)p.n_pages) old[e] = atomicSub(&p.refs[id[e]], 1);
        else if (c0 + e * kRowThreads < tiles) status |= KVMIX_PAGES_BAD_ID;
      }
#pragma unroll
      for (int e = 0; e < kEach; e++)
        if (old[e] == 1) atomicAnd(&p.used[id[e] >> 5], ~(1u << (id[e] & 31)));
    }
  }
  if (status) atomicOr(p.status, status);
}

// A workgroup per pair; it looks the other pairs over for its destination.
__global__ __launch_bounds__(kRowThreads) void pages_fork_kernel(kvmix_pages p, const int32_t* src, const int32_t* dst, int n) {
  const int i = blockIdx.x, from = src[i], to = dst[i];
  if (from < 0 || to < 0) return;
  int status = 0;
  if (from >= p.n_slots || to >= p.n_slots) {
    status = KVMIX_PAGES_BAD_ROW;
  } else {
    const int len = p.lens[from], held = p.lens[to];
    bool clash = held != 0 || from == to;
    // a source that is somebody's destination, a destination that is somebody's source or an earlier pair's destination
    for (int j = threadIdx.x; j < n; j += kRowThreads) {
      const int s = src[j], d = dst[j];
      if (s < 0 || d < 0) continue;
      clash |= d == from || s == to || (d == to && j != i);
    }
    if (__syncthreads_or(clash)) {
      status = KVMIX_PAGES_OCCUPIED;
    } else {
      int tiles = len > 0 ? packed_tiles(len, p.window) : 0;
      if (len < 0 || tiles > p.max_tiles) {
        status = KVMIX_PAGES_BAD_ROW;
      } else {
        const int32_t* ids = p.table + (size_t)from * p.max_tiles;
        int32_t* to_ids = p.table + (size_t)to * p.max_tiles;
        for (int c0 = threadIdx.x; c0 < tiles; c0 += kEach * kRowThreads) {
          int id[kEach];
#pragma unroll
          for (int e = 0; e < kEach; e++) id[e] = c0 + e * kRowThreads < tiles ? ids[c0 + e * kRowThreads] : -1;
#pragma unroll
          for (int e = 0; e < kEach; e++) {
            if (c0 + e * kRowThreads >= tiles) break;
            to_ids[c0 + e * kRowThreads] = id[e];
            if ((uint32_t)id[e] < (uint32_t)p.n_pages) atomicAdd(&p.refs[id[e]], 1);
            else status |= KVMIX_PAGES_BAD_ID;
          }
        }
        if (threadIdx.x == 0) { p.lens[to] = len; p.grown[to] = 0; }
      }
    }
  }
  if (status) atomicOr(p.status, status);
}

// One workgroup: pages in use are counted, then gaps below that number and pages above it are listed in order, a word of bits to a thread.
__global__ __launch_bounds__(kGrowThreads) void pages_compact_kernel(kvmix_pages p) {
  __shared__ int s_wave[kGrowThreads / kWave];
  const int tid = threadIdx.x, words = (p.n_pages + 31) / 32;
  int32_t* src = p.moves + 4;
  int32_t* dst = src + p.n_pages;
  int32_t* to = dst + p.n_pages;
  int used = 0, live;
  for (int w = tid; w < words; w += kGrowThreads) used += __popc(p.used[w] & valid_bits(w, p.n_pages));
  scan_before(used, s_wave, live);
  int gaps = 0, above = 0;
  for (int w0 = 0; w0 < words; w0 += kGrowThreads) {
    const int w = w0 + tid;
    uint32_t gap = 0, move = 0;
    if (w < words) {
      const uint32_t u = p.used[w] & valid_bits(w, p.n_pages), low = valid_bits(w, live);
      gap = ~u & low;
      move = u & ~low;
      if (u != low) p.used[w] = low;
    }
    int n_gap, n_move;
    int g = gaps + scan_before((int)__popc(gap), s_wave, n_gap), m = above + scan_before((int)__popc(move), s_wave, n_move);
    for (; gap; gap &= gap - 1u) dst[g++] = 32 * w + __ffs(gap) - 1;
    for (; move; move &= move - 1u) src[m++] = 32 * w + __ffs(move) - 1;
    gaps += n_gap;
    above += n_move;
  }
  __syncthreads();
  for (int i = tid; i < above; i += kGrowThreads) {
    const int s = src[i], d = dst[i];
    p.refs[d] = p.refs[s];
    p.refs[s] = 0;
    to[s] = d;
  }
  if (tid == 0) { p.moves[0] = above; p.moves[1] = live; }
}

__global__ __launch_bounds__(kRowThreads) void pages_rename_kernel(kvmix_pages p) {
  const int row = blockIdx.x, len = p.lens[row], live = p.moves[1];
  const int32_t* to = p.moves + 4 + 2 * (size_t)p.n_pages;
  int tiles = len > 0 ? packed_tiles(len, p.window) : 0;
  if (tiles > p.max_tiles) tiles = p.max_tiles;
  int32_t* ids = p.table + (size_t)row * p.max_tiles;
  for (int c = threadIdx.x; c < tiles; c += kRowThreads) {
    const int id = ids[c];
    if (id < live) continue;
    if (id < p.n_pages) ids[c] = to[id];
    else atomicOr(p.status, KVMIX_PAGES_BAD_ID);
  }
}

// Pieces of 16 KB, four 16-byte loads of a thread under way together; workgroups stay and take every gridDim-th piece.
constexpr int kPiece = 16384;
__global__ __launch_bounds__(256) void copy_kernel(CopyArgs a) {
  const int n = a.count ? *a.count : a.n;
  const uint32_t pieces = (uint32_t)((a.bytes + kPiece - 1) / kPiece), each = pieces * (uint32_t)a.n_base;
  const uint64_t total = (uint64_t)(n > 0 ? n : 0) * each;
  for (uint64_t at = blockIdx.x; at < total; at += gridDim.x) {
    const uint32_t i = (uint32_t)(at / each), rest = (uint32_t)(at % each);
    const int from = a.src[i], to = a.dst[i];
    if ((uint32_t)from >= (uint32_t)a.limit || (uint32_t)to >= (uint32_t)a.limit) {
      if (a.status && threadIdx.x == 0) atomicOr(a.status, KVMIX_PAGES_BAD_ID);
      continue;
    }
    char* base = a.base[rest >= pieces];
    const int64_t off = (int64_t)(rest >= pieces ? rest - pieces : rest) * kPiece + 16 * threadIdx.x, left = a.bytes - off;
    const char* s = base + (int64_t)from * a.bytes + off;
    char* d = base + (int64_t)to * a.bytes + off;
    u32x4_t x[4];
#pragma unroll
    for (int e = 0; e < 4; e++)
      if (4096 * e < left) x[e] = *reinterpret_cast<const u32x4_t*>(s + 4096 * e);
#pragma unroll
    for (int e = 0; e < 4; e++)
      if (4096 * e < left) *reinterpret_cast<u32x4_t*>(d + 4096 * e) = x[e];
  }
}

}  // namespace

hipError_t launch_pages_grow(const kvmix_pages& p, const int32_t* rows, const int32_t* cu, int n, hipStream_t s) {
  return launch(pages_grow_kernel, dim3(1), kGrowThreads, s, p, rows, cu, n);
}
hipError_t launch_pages_free(const kvmix_pages& p, const int32_t* rows, int n, hipStream_t s) {
  return launch(pages_free_kernel, dim3(n), kRowThreads, s, p, rows);
}
hipError_t launch_pages_fork(const kvmix_pages& p, const int32_t* src, const int32_t* dst, int n, hipStream_t s) {
  return launch(pages_fork_kernel, dim3(n), kRowThreads, s, p, src, dst, n);
}
hipError_t launch_pages_compact(const kvmix_pages& p, hipStream_t s) {
  const hipError_t e = launch(pages_compact_kernel, dim3(1), kGrowThreads, s, p);
  return e != hipSuccess ? e : launch(pages_rename_kernel, dim3(p.n_slots), kRowThreads, s, p);
}
hipError_t launch_copy(const CopyArgs& a, hipStream_t s) {
  const int64_t pieces = (a.bytes + kPiece - 1) / kPiece * a.n_base, most = a.n * pieces;
  return launch(copy_kernel, dim3((unsigned)(most < 4096 ? most : 4096)), 256, s, a);
}

}  // namespace kvmix
