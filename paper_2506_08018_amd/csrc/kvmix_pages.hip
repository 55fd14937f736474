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

constexpr int kGrowThreads = 1024, kGrowWaves = kGrowThreads / kWave;
constexpr int kMaxRows = 4096;                        // of one call of grow or fork
constexpr int kMostPages = (1 << 22) - 1;

template <int CTRL, int ROW_MASK = 0xf>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROW_MASK, 0xf, false); }
// sum over the wave's lanes up to this one
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v += dpp<0x111>(v);          // row_shr
  v += dpp<0x112>(v);
  v += dpp<0x114>(v);
  v += dpp<0x118>(v);
  v += dpp<0x142, 0xA>(v);     // row_bcast:15, :31
  v += dpp<0x143, 0xC>(v);
  return v;
}
// Sums over the workgroup's threads before this one, of two numbers at once; totals over all of them. s_wave is the call's own (no barrier
// in front of its first use, one behind).
struct Two { uint32_t a, b; };
__device__ __forceinline__ Two scan_before(Two v, Two (&s_wave)[kGrowWaves], Two& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Two x = {wave_scan(v.a), wave_scan(v.b)};
  if (lane == kWave - 1) s_wave[wave] = x;
  __syncthreads();
  const Two w = s_wave[lane % kGrowWaves], upto = {wave_scan(lane < kGrowWaves ? w.a : 0), wave_scan(lane < kGrowWaves ? w.b : 0)};
  auto at = [](uint32_t y, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)y, l); };
  total = {at(upto.a, kGrowWaves - 1), at(upto.b, kGrowWaves - 1)};
  const int before = __builtin_amdgcn_readfirstlane(wave) - 1;
  Two r = {x.a - v.a, x.b - v.b};
  if (before >= 0) { r.a += at(upto.a, before); r.b += at(upto.b, before); }
  return r;
}

__device__ __forceinline__ uint32_t valid_bits(int word, int n_pages) {
  const int left = n_pages - 32 * word;
  return left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u;
}

// One workgroup: what each row needs, in the rows' order, and how much there is, in one scan; then the lowest free ids that are granted, 32768 pages
// at a time, a word of bits to a thread. Ranks of free ids meet rows by binary search over the rows' first ranks. A slot that is named
// twice is looked for only if two rows meet in a table of 32768 bits. 32 rows with 1000 pages to take from 10 000: 16 us with
// chunks of 4096 ids, cross-lane sums through LDS and a comparison of every two rows, 4.3 now.
// EACH: rows of a thread, in a row.
constexpr int kBits = 32768, kIds = 4096;
template <int EACH>
__global__ __launch_bounds__(kGrowThreads) void pages_grow_kernel(kvmix_pages p, const int32_t* rows, const int32_t* cu, int n) {
  constexpr int kRows = EACH * kGrowThreads;
  __shared__ int s_row[kRows], s_first[kRows], s_before[kRows];
  __shared__ int s_id[kIds], s_rank[kGrowThreads];
  __shared__ uint32_t s_free[kGrowThreads];
  __shared__ uint32_t s_bits[kBits / 32];
  __shared__ Two s_wave[2][kGrowWaves];
  __shared__ int s_granted, s_status, s_twice;
  const int tid = threadIdx.x, words = (p.n_pages + 31) / 32;
  // (in flight together: the first words of bits, the rows, the counts)
  const uint32_t first_bits = tid < words ? ~p.used[tid] & valid_bits(tid, p.n_pages) : 0u;
  int row[EACH], status = 0, need[EACH], len[EACH], fresh[EACH], tiles[EACH];
  bool ok[EACH];
#pragma unroll
  for (int e = 0; e < EACH; e++) {
    const int i = tid * EACH + e;
    row[e] = i < n ? (rows ? rows[i] : i) : -1;
    s_row[i] = row[e];
    ok[e] = row[e] >= 0 && row[e] < p.n_slots;
    if (row[e] >= p.n_slots) status = KVMIX_PAGES_BAD_ROW;
    fresh[e] = 1;
    if (cu && i < n) {
      const int64_t add = (int64_t)cu[i + 1] - cu[i];
      fresh[e] = add >= 0 && add <= 0x7fffffff ? (int)add : -1;
    }
  }
  s_bits[tid] = 0;
  if (tid == 0) { s_granted = 0; s_status = 0; s_twice = 0; }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < EACH; e++) {
    len[e] = ok[e] ? p.lens[row[e]] : 0;
    if (ok[e]) {
      const uint32_t bit = 1u << (row[e] & 31);
      if (atomicOr(&s_bits[row[e] / 32 % (kBits / 32)], bit) & bit) s_twice = 1;
    }
  }
  uint32_t free_here = __popc(first_bits), sum = 0;
  for (int w = tid + kGrowThreads; w < words; w += kGrowThreads) free_here += __popc(~p.used[w] & valid_bits(w, p.n_pages));
  __syncthreads();
  if (s_twice) {
#pragma unroll
    for (int e = 0; e < EACH; e++) {
      bool again = false;
      for (int j = 0; j < tid * EACH + e; j++) again |= s_row[j] == row[e];
      if (again && ok[e]) { ok[e] = false; status |= KVMIX_PAGES_BAD_ROW; }
    }
  }
#pragma unroll
  for (int e = 0; e < EACH; e++) {
    need[e] = 0; tiles[e] = 0;
    if (ok[e] && (len[e] < 0 || fresh[e] < 0 || fresh[e] > 0x7fffffff - len[e])) { ok[e] = false; status |= KVMIX_PAGES_BAD_ROW; p.grown[row[e]] = 0; }
    if (ok[e]) {
      tiles[e] = packed_tiles(len[e], p.window);
      const int after = packed_tiles(len[e] + fresh[e], p.window);
      if (after <= p.max_tiles) need[e] = after - tiles[e];
      else { ok[e] = false; status |= KVMIX_PAGES_EXHAUSTED; p.grown[row[e]] = 0; }
    }
    sum += (uint32_t)need[e];
  }
  // (a thread's needs count up to kMostPages: what is more is more than there is, and 1024 of them fit 32 bits)
  Two all;
  const Two before = scan_before({free_here, sum < (uint32_t)kMostPages ? sum : (uint32_t)kMostPages}, s_wave[0], all);
  const int n_free = (int)all.a;
  int at = before.b < (1u << 24) ? (int)before.b : 1 << 24;
#pragma unroll
  for (int e = 0; e < EACH; e++) {
    const int i = tid * EACH + e;
    s_first[i] = at; s_before[i] = tiles[e];
    at += need[e];
    const bool granted = ok[e] && (need[e] == 0 || at <= n_free);
    if (granted && need[e]) atomicMax(&s_granted, at);
    if (granted) { p.lens[row[e]] = len[e] + fresh[e]; p.grown[row[e]] = fresh[e]; }
    else if (ok[e]) { p.grown[row[e]] = 0; status |= KVMIX_PAGES_EXHAUSTED; }
  }
  if (status) atomicOr(&s_status, status);
  __syncthreads();
  const int granted = s_granted;
  int base = 0;                        // free pages before the words in hand
  for (int w0 = 0; w0 < words && base < granted; w0 += kGrowThreads) {
    const int w = w0 + tid;
    const uint32_t bits = w0 == 0 ? first_bits : w < words ? ~p.used[w] & valid_bits(w, p.n_pages) : 0u;
    int r = (int)before.a, here = n_free;
    if (words > kGrowThreads) {        // (otherwise the first scan has said it)
      Two t;
      if (w0) __syncthreads();         // (s_wave has been read)
      r = base + (int)scan_before({(uint32_t)__popc(bits), 0}, s_wave[1], t).a;
      here = (int)t.a;
    }
    const int end = base + here < granted ? base + here : granted;
    s_rank[tid] = r; s_free[tid] = bits;
    const int bytes = 4 * (words - w0 < kGrowThreads ? words - w0 : kGrowThreads);
    __syncthreads();
    for (int lo = base; lo < end; lo += kIds) {
      const int many = end - lo < kIds ? end - lo : kIds;
      // a byte of bits to a thread (with a word to each, 32 times round the loop where all are free: 16 rows with 1100 pages 5.6 us, 4.4 now)
      for (int t = tid; t < bytes; t += kGrowThreads) {
        const uint32_t word = s_free[t >> 2];
        const int from = 8 * (t & 3);
        int k = s_rank[t >> 2] + __popc(word & ((1u << from) - 1u)) - lo;
        if (k >= many) continue;
        for (uint32_t left = word >> from & 255u; left; left &= left - 1u, k++)
          if (k >= 0 && k < many) s_id[k] = 32 * (w0 + (t >> 2)) + from + __ffs(left) - 1;
      }
      __syncthreads();
      for (int m = tid; m < many; m += kGrowThreads) {
        int a = 0, b = n - 1;          // the last row whose first rank is not past this one
        while (a < b) {
          const int mid = (a + b + 1) >> 1;
          if (s_first[mid] <= lo + m) a = mid;
          else b = mid - 1;
        }
        const int id = s_id[m];
        p.table[(size_t)s_row[a] * p.max_tiles + s_before[a] + (lo + m - s_first[a])] = id;
        p.refs[id] = 1;
      }
      __syncthreads();
    }
    uint32_t taken = bits;             // the lowest of them that are granted
    if (r >= end) taken = 0;
    else if (r + __popc(bits) > end) {
      for (int k = r; k < end; k++) taken &= taken - 1u;
      taken ^= bits;
    }
    if (taken) atomicOr(&p.used[w], taken);
    base += here;
  }
  if (tid == 0 && s_status) atomicOr(p.status, s_status);
}

// A workgroup per row. The length is taken out by an exchange, so that a slot that is named twice is freed once.
constexpr int kRowThreads = 256;
constexpr int kEach = 4;              // table entries of a thread under way together
// A thread's entries of a table row, the first of them on their way before the row's length is known (free of 32 rows with
// 2000 pages 3.88 -> 3.67 us, of 16 with 1100, out of the caches, 5.17 -> 5.04).
struct Ids {
  const int32_t* row;
  int max_tiles, id[kEach];
  __device__ __forceinline__ Ids(const kvmix_pages& p, int slot) : row(p.table + (size_t)slot * p.max_tiles), max_tiles(p.max_tiles) { load(threadIdx.x); }
  __device__ __forceinline__ void load(int c0) {
#pragma unroll
    for (int e = 0; e < kEach; e++) id[e] = c0 + e * kRowThreads < max_tiles ? row[c0 + e * kRowThreads] : -1;
  }
  __device__ __forceinline__ int (&at(int c0))[kEach] {
    if (c0 >= kRowThreads) load(c0);
    return id;
  }
};
__global__ __launch_bounds__(kRowThreads) void pages_free_kernel(kvmix_pages p, const int32_t* rows) {
  __shared__ int s_len;
  const int row = rows ? rows[blockIdx.x] : (int)blockIdx.x;
  if (row < 0) return;
  int status = 0;
  if (row >= p.n_slots) {
    status = KVMIX_PAGES_BAD_ROW;
  } else {
    if (threadIdx.x == 0) { s_len = atomicExch(&p.lens[row], 0); p.grown[row] = 0; }
    Ids ids(p, row);
    __syncthreads();
    int tiles = s_len > 0 ? packed_tiles(s_len, p.window) : 0;
    if (s_len < 0 || tiles > p.max_tiles) { status = KVMIX_PAGES_BAD_ROW; tiles = tiles > p.max_tiles ? p.max_tiles : 0; }
    for (int c0 = threadIdx.x; c0 < tiles; c0 += kEach * kRowThreads) {
      int (&id)[kEach] = ids.at(c0), old[kEach];
#pragma unroll
      for (int e = 0; e < kEach; e++) {
        old[e] = 2;
        if (c0 + e * kRowThreads >= tiles) continue;
        if ((uint32_t)id[e] < (uint32_t)p.n_pages) old[e] = atomicSub(&p.refs[id[e]], 1);
        else status |= KVMIX_PAGES_BAD_ID;
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
    Ids ids(p, from);
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
        int32_t* to_ids = p.table + (size_t)to * p.max_tiles;
        for (int c0 = threadIdx.x; c0 < tiles; c0 += kEach * kRowThreads) {
          const int (&id)[kEach] = ids.at(c0);
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
  __shared__ Two s_wave[2][kGrowWaves];
  const int tid = threadIdx.x, words = (p.n_pages + 31) / 32;
  int32_t* src = p.moves + 4;
  int32_t* dst = src + p.n_pages;
  int32_t* to = dst + p.n_pages;
  const uint32_t first_bits = tid < words ? p.used[tid] & valid_bits(tid, p.n_pages) : 0u;
  uint32_t used = __popc(first_bits);
  for (int w = tid + kGrowThreads; w < words; w += kGrowThreads) used += __popc(p.used[w] & valid_bits(w, p.n_pages));
  Two all;
  scan_before({used, 0}, s_wave[0], all);
  const int live = (int)all.a;
  int gaps = 0, above = 0;
  for (int w0 = 0; w0 < words; w0 += kGrowThreads) {
    const int w = w0 + tid;
    uint32_t gap = 0, move = 0;
    if (w < words) {
      const uint32_t u = w0 == 0 ? first_bits : p.used[w] & valid_bits(w, p.n_pages), low = valid_bits(w, live);
      gap = ~u & low;
      move = u & ~low;
      if (u != low) p.used[w] = low;
    }
    Two many;
    if (w0) __syncthreads();           // (s_wave has been read)
    const Two at = scan_before({(uint32_t)__popc(gap), (uint32_t)__popc(move)}, s_wave[1], many);
    int g = gaps + (int)at.a, m = above + (int)at.b;
    for (; gap; gap &= gap - 1u) dst[g++] = 32 * w + __ffs(gap) - 1;
    for (; move; move &= move - 1u) src[m++] = 32 * w + __ffs(move) - 1;
    gaps += (int)many.a;
    above += (int)many.b;
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

// Pieces of 8 KB, two 16-byte loads of a thread under way together; workgroups stay and take every gridDim-th piece. (300 pages of 32 KB 7.7 us, 8.2 in
// pieces of 16 KB for 4096 workgroups; rings of 32 slots x 8 heads, 50 MB read and written, 7.5 and 7.7.)
constexpr int kPiece = 8192;
__global__ __launch_bounds__(256) void copy_kernel(CopyArgs a) {
  const int n = a.count && *a.count < a.n ? *a.count : a.n;      // (a.n: the most there can be)
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
    u32x4_t x[2];
#pragma unroll
    for (int e = 0; e < 2; e++)
      if (4096 * e < left) x[e] = *reinterpret_cast<const u32x4_t*>(s + 4096 * e);
#pragma unroll
    for (int e = 0; e < 2; e++)
      if (4096 * e < left) *reinterpret_cast<u32x4_t*>(d + 4096 * e) = x[e];
  }
}

}  // namespace

hipError_t launch_pages_grow(const kvmix_pages& p, const int32_t* rows, const int32_t* cu, int n, hipStream_t s) {
  return n <= kGrowThreads ? launch(pages_grow_kernel<1>, dim3(1), kGrowThreads, s, p, rows, cu, n)
                           : launch(pages_grow_kernel<kMaxRows / kGrowThreads>, dim3(1), kGrowThreads, s, p, rows, cu, n);
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
  return launch(copy_kernel, dim3((unsigned)(most < 2048 ? most : 2048)), 256, s, a);
}

}  // namespace kvmix
