// C-ABI entry points of the paged cache and of what stands in front of it: host-side validation and launch plumbing only.
// Contract: include/kvmix.h.
#include <cmath>
#include "kvmix_common.hpp"

using namespace kvmix;

namespace {

constexpr int kMostWorkgroups = 1 << 24;  // of 256 threads along one axis: threads are counted in 32 bits
constexpr int kMostWindow = 1 << 30;      // (with what the largest table holds, lengths stay below 2^31)

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int check_pages(const kvmix_pages* p) {
  if (!p || !p->table || !p->lens || !p->grown || !p->refs || !p->used || !p->status) return KVMIX_ERR_NULL;
  if (!aligned4(p->table) || !aligned4(p->lens) || !aligned4(p->grown)) return KVMIX_ERR_ALIGN;
  if (!aligned4(p->refs) || !aligned4(p->used) || !aligned4(p->status)) return KVMIX_ERR_ALIGN;
  // (fewer than 4 M pages: sums over the workgroup of the grow kernel fit 32 bits)
  if (p->n_slots < 1 || p->n_slots > (1 << 20) || p->n_pages < 1 || p->n_pages >= (1 << 22) || p->max_tiles < 1 || p->max_tiles > (1 << 23)) return KVMIX_ERR_BAD_SHAPE;
  if (p->window < 0 || p->window > kMostWindow || p->window % kTile) return KVMIX_ERR_BAD_SHAPE;
  return KVMIX_OK;
}

int check_paged_cfg(const kvmix_shape* sh, const kvmix_layer_cfg* cfg) {
  const int st = check_shape_cfg(sh, cfg);
  if (st) return st;
  if (cfg->k_bits == 16) return KVMIX_ERR_BAD_BITS;
  return cfg->window < 0 || cfg->window > kMostWindow ? KVMIX_ERR_BAD_SHAPE : KVMIX_OK;
}

// `pool`, `rings`: what the call touches
int check_paged_cache(const kvmix_layer_cfg* cfg, const kvmix_paged_cache* c, bool pool, bool rings) {
  if (!c || (pool && !c->pool) || (rings && (!c->k_win || !c->v_win))) return KVMIX_ERR_NULL;
  if ((pool && !aligned16(c->pool)) || (rings && (!aligned16(c->k_win) || !aligned16(c->v_win)))) return KVMIX_ERR_ALIGN;
  if (c->n_pages < 1 || c->n_slots < 1 || c->W_cap % kTile || c->W_cap < cfg->window + kTile) return KVMIX_ERR_BAD_SHAPE;
  return KVMIX_OK;
}

int check_together(const kvmix_shape* sh, const kvmix_layer_cfg* cfg, const kvmix_paged_cache* c, const kvmix_pages* p) {
  if (c->n_pages != p->n_pages || c->n_slots != p->n_slots || cfg->window != p->window) return KVMIX_ERR_BAD_SHAPE;
  // tile % ring tiles goes by a product with a reciprocal; (slot, head) pairs are counted in 32 bits
  if ((long long)p->max_tiles * (c->W_cap / kTile) >= (1LL << 32) || (long long)p->n_slots * sh->Hkv > 0x7fffffffLL) return KVMIX_ERR_BAD_SHAPE;
  return KVMIX_OK;
}

uint32_t ring_magic(int ring_tiles) { return ring_tiles == 1 ? 0u : (uint32_t)((1ULL << 32) / (uint32_t)ring_tiles + 1); }

// A ragged launch: batch rows in launches of at most kRows, each with a workgroup per piece of a context, kv head and block of heads.
// Pieces are made on the device (find_piece in kvmix_attn.hip): from the tiles of the whole batch a share for each of the kPlaces
// workgroups that the chip holds at once (8 waves, two to a compute unit), or somewhat more. The grid has as many pieces as the chip holds while the rows
// are no more than half of that: in shares of 2.2 (kShares) they always fit. For more rows it has the rows and what shares of 2.2 cut off besides: where
// workgroups queue, few large pieces are better (48 x 8 units of 4 heads, 512 to 8192 tokens 35.4 -> 32.9 us, 64 x 8 of 1 to 4096 20.4 -> 18.6 against a
// grid for every piece that shares of 1.1 make), and each workgroup that finds no piece takes 2 us at the end.
constexpr int kRows = 512, kCus = 256, kPlaces = 2 * kCus;
constexpr float kAloneInTwelve = 0.55f;       // kAlone of a workgroup of 12 waves
struct PagedPlan { int block, head_blocks, rows, pieces, share, waves; size_t counters, bytes; };
PagedPlan plan_paged(const kvmix_shape* sh, int window, int max_len, int v_bits) {
  PagedPlan p;
  const int G = sh->Hq / sh->Hkv;
  // 8 heads with 3- or 4-bit Values do not fit the registers of 8 waves as a block of 8: half a block of 16 (see plan_attention)
  p.block = G <= 4 || (G == 8 && v_bits < 3) ? G : 16;
  p.head_blocks = (G + p.block - 1) / p.block;
  p.rows = sh->B < kRows ? sh->B : kRows;
  const int tiles = packed_tiles(max_len, window), held = max_len - window < kTile ? max_len : window + kTile - 1;
  const long long most = tiles + (long long)kWindowTiles * (((long long)held + kTile - 1) / kTile);
  const long long each = most <= kMinShare ? 1 : (most + kMinShare - 1) / kMinShare;
  const long long units = (long long)sh->B * sh->Hkv;
  const bool few_long = sh->B > 1 && G <= 8 && units <= (G == 8 && v_bits >= 3 ? 64 : 32) && units * tiles > 31 * kCus;
  p.share = 1; p.waves = 8;
  if (few_long) {
    // A few long contexts: one workgroup of 12 waves to a compute unit, as for one sequence (2 x 8 units of 4 heads, 32k tokens 19.5 -> 18.1 us, of 32k
    // and 32 tokens at 3/4 bit 18.3 -> 16.7, 4 x 8 of 512 to 32k 19.0 -> 18.2, 4 x 8 of 8 heads, 16k 22.5 -> 19.9, 8 x 8 of 8 heads with 4-bit
    // Values, 512 to 16k 25.0 -> 20.7). Not with more of them or shorter ones: 8 x 8 of 512 to 32k 21.5 and 25.3, 16 x 8 of 8k 25.4 and 28.4, 4 x 8
    // of 8k 13.2 both, 2 x 8 of 8k 11.1 and 11.9, 4 x 32 of 1 head, 256 to 8k 16.4 and 17.5.
    p.waves = 12;
    p.block = G;
  }
  const int held_at_once = (p.waves == 12 ? kCus : kPlaces) / (sh->Hkv * p.head_blocks);
  const long long by_places = p.rows <= held_at_once / 2 ? held_at_once : p.rows + held_at_once * 5 / 11 + 1, by_length = p.rows * each;
  p.pieces = (int)(by_places < by_length ? by_places : by_length);
  p.counters = ((size_t)p.rows * sh->Hkv * (G > 8 ? G / 8 : 1) * 4 + 255) / 256 * 256;
  p.bytes = p.counters + (size_t)p.pieces * sh->Hkv * G * (kD + 2) * sizeof(float);
  if (sh->B == 1) {
    // One sequence: unsplit, one workgroup or two to a compute unit, at most 64 pieces (1 x 8 heads over 32k tokens: 64 pieces 13.0 us, 256
    // 17.0), by the model of a batch's launch. One to a compute unit has 12 waves where there are more than 20 tiles for it: 8 x 4 heads over
    // 32k tokens 12.5 us (2/2 bit; 3/4 bit 13.3), 8 waves 13.4 (14.6), two of 8 waves 15.7 (16.5); over 120k tokens 23.9, 28.4, 25.2; 8 x 8
    // heads at 2/4 bit over 32k 14.5, 17.1, 22.5; 8 x 2 heads over 16k, 16 tiles each, 9.85, 9.75, 11.8.
    const int groups = sh->Hkv * p.head_blocks;
    float best = INFINITY;
    int splits = 1;
    for (int places = 0; places <= kPlaces; places += kCus) {
      int n = places / groups < 64 ? places / groups : 64;
      if (n > p.pieces) n = p.pieces;
      if (n < 1) n = 1;
      const float largest = (float)((most + n - 1) / n);
      const bool twelve = G <= 8 && (long long)n * groups <= kCus && tiles > 20 * n;
      const float time = (n > 1 ? kMergeTiles * (float)n : 0.0f) + (twelve ? kAloneInTwelve / kAlone : 1.0f) *
                         model_time((float)(n * groups), largest, (float)most * groups / kPlaces, kPlaces, 1.0f / kPlaces);
      if (time < best) { best = time; splits = n; p.waves = twelve ? 12 : 8; }
    }
    if (p.waves == 12) p.block = G;
    p.share = tiles > splits ? (tiles + splits - 1) / splits : 1;
    p.pieces = tiles > 0 ? (tiles + p.share - 1) / p.share : 1;
  }
  return p;
}

}  // namespace

extern "C" {

int kvmix_pages_grow(const kvmix_pages* p, const int32_t* rows, const int32_t* cu, int n_rows, void* stream) {
  const int st = check_pages(p);
  if (st) return st;
  if (n_rows < 0 || n_rows > 4096) return KVMIX_ERR_BAD_SHAPE;
  if (!aligned4(rows) || !aligned4(cu)) return KVMIX_ERR_ALIGN;
  if (n_rows == 0) return KVMIX_OK;
  const hipError_t e = launch_pages_grow(*p, rows, cu, n_rows, (hipStream_t)stream);
  return e == hipSuccess ? KVMIX_OK : hip_fail(e);
}

int kvmix_pages_free(const kvmix_pages* p, const int32_t* rows, int n_rows, void* stream) {
  const int st = check_pages(p);
  if (st) return st;
  if (n_rows < 0 || n_rows > (1 << 20)) return KVMIX_ERR_BAD_SHAPE;
  if (!aligned4(rows)) return KVMIX_ERR_ALIGN;
  if (n_rows == 0) return KVMIX_OK;
  const hipError_t e = launch_pages_free(*p, rows, n_rows, (hipStream_t)stream);
  return e == hipSuccess ? KVMIX_OK : hip_fail(e);
}

int kvmix_pages_fork(const kvmix_pages* p, const int32_t* src, const int32_t* dst, int n_pairs, void* stream) {
  const int st = check_pages(p);
  if (st) return st;
  if (n_pairs < 0 || n_pairs > 4096) return KVMIX_ERR_BAD_SHAPE;
  if (n_pairs == 0) return KVMIX_OK;
  if (!src || !dst) return KVMIX_ERR_NULL;
  if (!aligned4(src) || !aligned4(dst)) return KVMIX_ERR_ALIGN;
  const hipError_t e = launch_pages_fork(*p, src, dst, n_pairs, (hipStream_t)stream);
  return e == hipSuccess ? KVMIX_OK : hip_fail(e);
}

int kvmix_pages_compact(const kvmix_pages* p, void* stream) {
  const int st = check_pages(p);
  if (st) return st;
  if (!p->moves) return KVMIX_ERR_NULL;
  if (!aligned16(p->moves)) return KVMIX_ERR_ALIGN;
  const hipError_t e = launch_pages_compact(*p, (hipStream_t)stream);
  return e == hipSuccess ? KVMIX_OK : hip_fail(e);
}

int kvmix_move_records(const kvmix_shape* sh, const kvmix_layer_cfg* cfg, const kvmix_paged_cache* c, const kvmix_pages* p, void* stream) {
  int st = check_paged_cfg(sh, cfg);
  if (st) return st;
  st = check_paged_cache(cfg, c, true, false);
  if (st) return st;
  st = check_pages(p);
  if (st) return st;
  st = check_together(sh, cfg, c, p);
  if (st) return st;
  if (!p->moves) return KVMIX_ERR_NULL;
  if (!aligned16(p->moves)) return KVMIX_ERR_ALIGN;
  CopyArgs a{};
  a.base[0] = reinterpret_cast<char*>(c->pool);
  a.n_base = 1;
  a.bytes = (int64_t)sh->Hkv * record_words(cfg->k_bits, cfg->v_bits) * 4;
  a.src = p->moves + 4; a.dst = a.src + p->n_pages; a.count = p->moves;
  a.n = p->n_pages / 2 + 1;      // no more moves than gaps and no more than pages above them
  a.limit = p->n_pages;
  a.status = p->status;
  const hipError_t e = launch_copy(a, (hipStream_t)stream);
  return e == hipSuccess ? KVMIX_OK : hip_fail(e);
}

int kvmix_copy_windows(const kvmix_shape* sh, const kvmix_layer_cfg* cfg, const kvmix_paged_cache* c, const int32_t* src, const int32_t* dst,
                       int n_pairs, void* stream) {
  int st = check_paged_cfg(sh, cfg);
  if (st) return st;
  st = check_paged_cache(cfg, c, false, true);
  if (st) return st;
  if (n_pairs < 0 || n_pairs > 65535) return KVMIX_ERR_BAD_SHAPE;
  if (n_pairs == 0) return KVMIX_OK;
  if (!src || !dst) return KVMIX_ERR_NULL;
  if (!aligned4(src) || !aligned4(dst)) return KVMIX_ERR_ALIGN;
  CopyArgs a{};
  a.base[0] = reinterpret_cast<char*>(c->k_win);
  a.base[1] = reinterpret_cast<char*>(c->v_win);
  a.n_base = 2;
  a.bytes = (int64_t)sh->Hkv * c->W_cap * kD * 2;
  a.src = src; a.dst = dst;
  a.n = n_pairs; a.limit = c->n_slots;
  const hipError_t e = launch_copy(a, (hipStream_t)stream);
  return e == hipSuccess ? KVMIX_OK : hip_fail(e);
}

int kvmix_paged_append(const kvmix_shape* sh, const kvmix_layer_cfg* cfg, const uint16_t* k_new, int64_t k_token_stride, int64_t k_head_stride,
                       const uint16_t* v_new, int64_t v_token_stride, int64_t v_head_stride, int n_tokens, const kvmix_paged_cache* c,
                       const kvmix_pages* p, const int32_t* rows, const int32_t* cu, int max_new, void* stream) {
  int st = check_paged_cfg(sh, cfg);
  if (st) return st;
  st = check_paged_cache(cfg, c, true, true);
  if (st) return st;
  st = check_pages(p);
  if (st) return st;
  st = check_together(sh, cfg, c, p);
  if (st) return st;
  if (max_new < 0 || n_tokens < 0 || (!cu && (max_new > 1 || n_tokens < sh->B))) return KVMIX_ERR_BAD_SHAPE;
  if (!aligned4(rows) || !aligned4(cu)) return KVMIX_ERR_ALIGN;
  if (max_new == 0 || n_tokens == 0) return KVMIX_OK;
  if (!k_new || !v_new) return KVMIX_ERR_NULL;
  if (!aligned16(k_new) || !aligned16(v_new)) return KVMIX_ERR_ALIGN;
  for (const int64_t x : {k_token_stride, k_head_stride, v_token_stride, v_head_stride})
    if (x % 8 || x < 0) return KVMIX_ERR_ALIGN;
  if (!rows && p->n_slots < sh->B) return KVMIX_ERR_BAD_SHAPE;
  PagedAppendArgs a{};
  a.q.k = k_new; a.q.v = v_new;
  a.q.tok = k_token_stride; a.q.unit_h = k_head_stride;
  a.v_tok = v_token_stride; a.v_head = v_head_stride;
  a.q.k_ring = c->k_win; a.q.v_ring = c->v_win; a.q.k_ring_w = c->k_win; a.q.v_ring_w = c->v_win;
  a.q.W_cap = c->W_cap; a.q.packed = c->pool; a.q.Hkv = sh->Hkv;
  a.rows = rows; a.cu = cu; a.lens = p->lens; a.grown = p->grown; a.table = p->table; a.status = p->status;
  a.n_slots = p->n_slots; a.n_pages = p->n_pages; a.max_tiles = p->max_tiles; a.window = p->window; a.max_new = max_new;
  a.ring_tiles = c->W_cap / kTile;
  a.ring_magic = ring_magic(a.ring_tiles);
  a.B = sh->B; a.n_tokens = n_tokens;
  // rows that stay lie in two ring tiles if they are no more than a tile, and in all of them at worst; one tile for what is due beyond a 32nd
  a.more = 1 + (max_new <= kTile && a.ring_tiles > 2 ? 2 : a.ring_tiles);
  a.head_magic = ring_magic(sh->Hkv);
  const long long tiles = (long long)n_tokens / kTile + (long long)sh->B * a.more + 1;
  if (tiles * sh->Hkv * sh->Hkv >= (1LL << 32) || (tiles + 7) * sh->Hkv >= kMostWorkgroups) return KVMIX_ERR_BAD_SHAPE;
  const hipError_t e = launch_paged_append(a, cfg->k_bits, cfg->v_bits, (hipStream_t)stream);
  return e == hipSuccess ? KVMIX_OK : hip_fail(e);
}

int kvmix_paged_workspace_bytes(const kvmix_shape* sh, int max_len, size_t* bytes) {
  const kvmix_layer_cfg cfg = {2, 2, 0};
  const int st = check_shape_cfg(sh, &cfg);
  if (st) return st;
  if (!bytes) return KVMIX_ERR_NULL;
  if (max_len < 1) return KVMIX_ERR_BAD_SHAPE;
  // (any window and any widths: a token counts for more in a window than in a page, so that one which holds everything has the most pieces)
  *bytes = 0;
  if (max_len > kMostWindow) max_len = kMostWindow;      // (long before that the pieces are as many as the chip holds)
  for (int v_bits = 2; v_bits <= 3; v_bits++) {
    const PagedPlan p = plan_paged(sh, max_len / kTile * kTile, max_len, v_bits);
    if (p.bytes > *bytes) *bytes = p.bytes;
  }
  return KVMIX_OK;
}

int kvmix_paged_decode_attn(const kvmix_shape* sh, const kvmix_layer_cfg* cfg, const uint16_t* q, const kvmix_paged_cache* c, const kvmix_pages* p,
                            const int32_t* rows, int max_len, float softmax_scale, uint16_t* out, void* workspace, size_t workspace_bytes,
                            void* stream) {
  int st = check_paged_cfg(sh, cfg);
  if (st) return st;
  if (!q || !out) return KVMIX_ERR_NULL;
  if (!aligned16(q) || !aligned16(out)) return KVMIX_ERR_ALIGN;
  st = check_paged_cache(cfg, c, true, true);
  if (st) return st;
  st = check_pages(p);
  if (st) return st;
  st = check_together(sh, cfg, c, p);
  if (st) return st;
  if (!aligned4(rows)) return KVMIX_ERR_ALIGN;
  if (!rows && p->n_slots < sh->B) return KVMIX_ERR_BAD_SHAPE;
  const long long most = (long long)p->max_tiles * kTile + p->window + kTile - 1;
  if (max_len <= 0 || max_len > most) max_len = most < 0x7fffffffLL ? (int)most : 0x7fffffff;
  const PagedPlan plan = plan_paged(sh, p->window, max_len, cfg->v_bits);
  const int G = sh->Hq / sh->Hkv;
  PagedAttnArgs a{};
  if (plan.pieces > plan.rows) {
    if (!workspace) return KVMIX_ERR_NULL;
    if (!aligned16(workspace)) return KVMIX_ERR_ALIGN;
    if (workspace_bytes < plan.bytes) return KVMIX_ERR_WORKSPACE;
    a.counters = reinterpret_cast<uint32_t*>(workspace);
    a.part = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + plan.counters);
  }
  const int counted = plan.rows * sh->Hkv * (G > 8 ? G / 8 : 1);
  a.counter_stride = 1;
  while (a.counter_stride * 2 * counted <= 64) a.counter_stride *= 2;
  a.G = G;
  a.packed = c->pool;
  a.k_win = c->k_win; a.v_win = c->v_win;
  a.W_cap = c->W_cap; a.ring_tiles = c->W_cap / kTile;
  a.head_blocks = plan.head_blocks;
  a.n_slots = p->n_slots; a.n_pages = p->n_pages; a.Hkv = sh->Hkv; a.window = p->window; a.max_len = max_len;
  a.groups = (float)(sh->Hkv * plan.head_blocks);
  const int at_once = plan.waves == 12 ? kCus : kPlaces;
  a.places = (float)at_once; a.inv_places = 1.0f / (float)at_once;
  a.most_pieces = plan.pieces;
  a.share = plan.share; a.inv_share = 1.0f / (float)plan.share;
  a.ring_magic = ring_magic(a.ring_tiles);
  const float scale = softmax_scale > 0.0f ? softmax_scale : 1.0f / std::sqrt((float)kD);
  a.scale_log2 = scale * 1.4426950408889634f;
  // (rows dealt out evenly: a launch of one row is another kind)
  const int launches = (sh->B + kRows - 1) / kRows;
  for (int i = 0, b = 0, n; i < launches; i++, b += n) {
    n = sh->B / launches + (i < sh->B % launches ? 1 : 0);
    a.q = q + (size_t)b * sh->Hq * kD; a.out = out + (size_t)b * sh->Hq * kD;
    kvmix_pages here = *p;
    if (!rows) {      // (the launch's rows are slots from 0 on)
      const size_t ring = (size_t)b * sh->Hkv * c->W_cap * kD;
      here.table += (size_t)b * p->max_tiles; here.lens += b;
      a.k_win = c->k_win + ring; a.v_win = c->v_win + ring;
      a.n_slots = p->n_slots - b;
    }
    const auto run = plan.waves == 12 ? launch_paged_attn<12> : launch_paged_attn<8>;
    const hipError_t e = run(a, here, rows ? rows + b : nullptr, n, plan.pieces, cfg->k_bits, cfg->v_bits, plan.block, (hipStream_t)stream);
    if (e != hipSuccess) return hip_fail(e);
  }
  return KVMIX_OK;
}

int kvmix_rope_frequencies(int rotary_dim, double base, int scaling, double factor, int original_len, double low, double high, float* frequencies,
                           float* amplitude) {
  if (!frequencies) return KVMIX_ERR_NULL;
  if (rotary_dim < 2 || rotary_dim > kD || rotary_dim % 2 || !(base > 1.0) || !std::isfinite(base)) return KVMIX_ERR_BAD_SHAPE;
  if (scaling < KVMIX_ROPE_PLAIN || scaling > KVMIX_ROPE_INDEX) return KVMIX_ERR_BAD_SHAPE;
  if (scaling != KVMIX_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return KVMIX_ERR_BAD_SHAPE;
  const bool ramps = scaling == KVMIX_ROPE_TURNS || scaling == KVMIX_ROPE_INDEX;
  if (ramps && (original_len < 1 || !(low > 0.0) || !(high > low) || !std::isfinite(high))) return KVMIX_ERR_BAD_SHAPE;
  if (scaling == KVMIX_ROPE_BASE && rotary_dim == 2) return KVMIX_ERR_BAD_SHAPE;
  const double two_pi = 6.283185307179586477, r = rotary_dim;
  if (scaling == KVMIX_ROPE_BASE) base *= std::pow(factor, r / (r - 2));
  // index at which a pair makes `turns` turns in original_len positions: original_len * base^(-2i / r) = 2 pi turns
  auto index_of = [&](double turns) { return r * std::log(original_len / (two_pi * turns)) / (2.0 * std::log(base)); };
  for (int i = 0; i < rotary_dim / 2; i++) {
    const double f = std::pow(base, -2.0 * i / r);
    double keep = 1.0;               // share of the unscaled frequency
    if (scaling == KVMIX_ROPE_LINEAR) keep = 0.0;
    if (scaling == KVMIX_ROPE_TURNS) keep = (original_len * f / two_pi - low) / (high - low);
    if (scaling == KVMIX_ROPE_INDEX) keep = (index_of(low) - i) / (index_of(low) - index_of(high));
    keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
    frequencies[i] = (float)(scaling == KVMIX_ROPE_PLAIN || scaling == KVMIX_ROPE_BASE ? f : f * keep + f / factor * (1.0 - keep));
  }
  if (amplitude) *amplitude = scaling == KVMIX_ROPE_INDEX ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return KVMIX_OK;
}

int kvmix_qk_norm_rope(const kvmix_shape* sh, const kvmix_rope* rope, int dtype, int n_tokens, const int32_t* positions, void* stream) {
  const kvmix_layer_cfg cfg = {2, 2, 0};
  const int st = check_shape_cfg(sh, &cfg);
  if (st) return st;
  if (!rope) return KVMIX_ERR_NULL;
  if (dtype != KVMIX_F16 && dtype != KVMIX_BF16 && dtype != KVMIX_F32) return KVMIX_ERR_BAD_SHAPE;
  if (rope->rotary_dim < 0 || rope->rotary_dim > kD || rope->rotary_dim % 16 || n_tokens < 0) return KVMIX_ERR_BAD_SHAPE;
  if (!(rope->eps >= 0.0f) || n_tokens >= kMostWorkgroups) return KVMIX_ERR_BAD_SHAPE;
  if (rope->rotary_dim > 0 && !rope->frequencies) return KVMIX_ERR_NULL;
  if (!aligned16(rope->frequencies) || !aligned16(rope->q_weight) || !aligned16(rope->k_weight) || !aligned4(positions)) return KVMIX_ERR_ALIGN;
  const int step = dtype == KVMIX_F32 ? 4 : 8;       // elements of 16 bytes
  RopeArgs a{};
  const kvmix_rope_side* side[3] = {&rope->q, &rope->k, &rope->v};
  const void* weight[3] = {rope->q_weight, rope->k_weight, nullptr};
  for (int i = 0; i < 3; i++) {
    const kvmix_rope_side& s = *side[i];
    if (!s.in != !s.out) return KVMIX_ERR_NULL;
    if (!aligned16(s.in) || !aligned16(s.out) || (s.in && (s.token_stride % step || s.head_stride % step))) return KVMIX_ERR_ALIGN;
    a.side[i] = RopeSide{s.in, s.out, weight[i], s.token_stride, s.head_stride, !s.in ? 0 : i == 0 ? sh->Hq : sh->Hkv};
  }
  const bool turns = rope->q.in || rope->k.in;
  if (n_tokens == 0 || (!turns && !rope->v.in)) return KVMIX_OK;
  a.rotary_dim = turns ? rope->rotary_dim : 0;
  if (!positions && a.rotary_dim > 0) return KVMIX_ERR_NULL;
  a.positions = positions; a.frequencies = rope->frequencies;
  a.n_tokens = n_tokens; a.interleaved = rope->interleaved != 0;
  a.amplitude = rope->amplitude; a.eps = rope->eps;
  const hipError_t e = launch_rope(a, dtype, (hipStream_t)stream);
  return e == hipSuccess ? KVMIX_OK : hip_fail(e);
}

}  // extern "C"
