// Queries, Keys and Values between the projections and the cache (gfx950): norm of each head, rotation by position, conversion to fp16.
//
// y = x / sqrt(mean(x^2) + eps) * w;  pair (a, b) of y and angle t = position * frequency:  (a cos t - b sin t, b cos t + a sin t).
// Memory-bound: 2 or 4 bytes in and 2 out per element. 16 lanes have a row of 128 channels, 8 channels each, so that both
// channels of a pair belong to one lane: 4 consecutive ones of either half of the rotated part (pairs (i, i + r/2)) or 8 consecutive ones
// (neighbours, and what is not rotated). No lane needs another's values but for the sum of squares. Every row of a token turns by the same
// angles: a lane has 4 of them, made once for all the rows that it takes.
// An angle is a fraction of a turn taken in binary64: position * frequency in fp32 is off by up to position * 2^-24 radians, 0.06 at a
// million.
// Measured: a prompt of 8191 tokens x 48 heads in bf16 (201 MB) 39.3 us, what a plain copy of as many bytes takes (38.9); one row of a lane at a
// time 45 us, with the row's pointers read by index from the arguments and sine and cosine by the math library 64 us. One token x 48
// heads 2.3 us, 64 tokens x 80 heads 3.1, a launch that does anything 2.3. With 8 lanes to a row and 16 bytes of either half per lane
// 38.8 and 41 us (two rows and one at a time), 2.5 for one token; with accesses past the caches 43-49 us.
#include <type_traits>
#include "kvmix_common.hpp"

namespace kvmix {

namespace {

struct Bf16 { uint16_t bits; };
constexpr int P = 4;       // consecutive channels of a lane, twice
// as loaded: 8 bytes, or 16 of fp32
template <typename T> struct Group {
  static constexpr int kWords = P * (int)sizeof(T) / 4;
  typedef uint32_t words_t __attribute__((ext_vector_type(kWords)));
  words_t w;
  __device__ __forceinline__ void load(const void* base, int64_t at) { w = *reinterpret_cast<const words_t*>(reinterpret_cast<const T*>(base) + at); }
  __device__ __forceinline__ void get(float (&x)[P]) const {
#pragma unroll
    for (int i = 0; i < kWords; i++) {
      const uint32_t v = w[i];       // (a copy: a bit cast applied to the vector element itself reads element 0)
      if constexpr (std::is_same_v<T, float>) {
        x[i] = __builtin_bit_cast(float, v);
      } else if constexpr (std::is_same_v<T, Bf16>) {
        const uint32_t lo = v << 16, hi = v & 0xFFFF0000u;
        x[2 * i] = __builtin_bit_cast(float, lo); x[2 * i + 1] = __builtin_bit_cast(float, hi);
      } else {
        const half2_t p = __builtin_bit_cast(half2_t, v);
        x[2 * i] = (float)p[0]; x[2 * i + 1] = (float)p[1];
      }
    }
  }
};
__device__ __forceinline__ void store(uint16_t* p, const float (&x)[P]) {
  const half2_t a = {(half_t)x[0], (half_t)x[1]}, b = {(half_t)x[2], (half_t)x[3]};
  *reinterpret_cast<u32x2_t*>(p) = u32x2_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
// sum over the 16 lanes that have a row; every one of them gets it
__device__ __forceinline__ float row_sum(float v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  v += dpp<0x141>(v);
  v += dpp<0x140>(v);
  return v;
}

constexpr int kRopeThreads = 256, kLanes = kD / (2 * P), kRows = kRopeThreads / kLanes;
// Grid (tokens, blocks of kRows * R rows): R rows of a lane are under way together. Tokens of half as many rows or fewer (R == 1): log2_tokens,
// so many share a workgroup.
template <typename T, int R>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(RopeArgs a) {
  const int c = threadIdx.x % kLanes;
  int token = blockIdx.x, row0 = (int)threadIdx.x / kLanes;      // first row of the lane
  if constexpr (R == 1) {
    const int each = kRows >> a.log2_tokens;
    token = (token << a.log2_tokens) + row0 / each;      // (a power of two)
    row0 %= each;
    if (token >= a.n_tokens) return;
  }
  const int turned = a.rotary_dim / (2 * P);           // lanes that have pairs
  // first channels of the lane's two groups
  const bool halves = !a.interleaved && c < turned;
  const int at0 = halves ? P * c : 2 * P * c, at1 = halves ? a.rotary_dim / 2 + P * c : 2 * P * c + P;
  const int n_q = a.side[0].heads, n_qk = n_q + a.side[1].heads, rows = n_qk + a.side[2].heads;
  Group<T> x0[R], x1[R];
  // (a row's side is chosen with the arguments in scalar registers: as an index into them it would be one more way to memory)
  auto side_of = [&](int row, auto field) {
    const auto q = field(a.side[0]), k = field(a.side[1]), v = field(a.side[2]);
    return row < n_q ? q : row < n_qk ? k : v;
  };
  auto row_at = [&](int k) { return ((int)blockIdx.y * R + k) * kRows + row0; };
  auto head_of = [&](int row) { return row - (row < n_q ? 0 : row < n_qk ? n_q : n_qk); };
#pragma unroll
  for (int k = 0; k < R; k++) {
    const int row = row_at(k);
    if (row >= rows) continue;
    const int64_t at = (int64_t)token * side_of(row, [](const RopeSide& s) { return s.tok; }) +
                       (int64_t)head_of(row) * side_of(row, [](const RopeSide& s) { return s.head; });
    const void* in = side_of(row, [](const RopeSide& s) { return s.in; });
    x0[k].load(in, at + at0);
    x1[k].load(in, at + at1);
  }
  Group<T> w[2][2];
#pragma unroll
  for (int s = 0; s < 2; s++)
    if (a.side[s].weight) { w[s][0].load(a.side[s].weight, at0); w[s][1].load(a.side[s].weight, at1); }
  float cs[P], sn[P];
  if (c < turned) {
    const double pos = (double)a.positions[token];
#pragma unroll
    for (int i = 0; i < P; i++) {
      double t = pos * ((double)a.frequencies[P * c + i] * 0.15915494309189533577);
      t -= rint(t);
      // (the hardware's sine and cosine take turns)
      cs[i] = __builtin_amdgcn_cosf((float)t) * a.amplitude;
      sn[i] = __builtin_amdgcn_sinf((float)t) * a.amplitude;
    }
  }
#pragma unroll
  for (int k = 0; k < R; k++) {
    const int row = row_at(k);
    if (row >= rows) continue;
    float x[P], y[P];
    x0[k].get(x);
    x1[k].get(y);
    const bool key = row >= n_q;
    if (row < n_qk && (key ? a.side[1].weight : a.side[0].weight)) {
      float sum = 0.0f, u[P], v[P];
#pragma unroll
      for (int i = 0; i < P; i++) sum += x[i] * x[i] + y[i] * y[i];
      const float r = rsqrtf(row_sum(sum) * (1.0f / kD) + a.eps);
      (key ? w[1][0] : w[0][0]).get(u);
      (key ? w[1][1] : w[0][1]).get(v);
#pragma unroll
      for (int i = 0; i < P; i++) { x[i] = x[i] * r * u[i]; y[i] = y[i] * r * v[i]; }
    }
    if (row < n_qk && c < turned) {
      if (a.interleaved) {
        // pairs 0 .. P/2 - 1 in the first group, the others in the second
#pragma unroll
        for (int i = 0; i < P; i++) {
          float (&g)[P] = i < P / 2 ? x : y;
          const int e = 2 * (i % (P / 2));
          const float p = g[e], q = g[e + 1];
          g[e] = p * cs[i] - q * sn[i];
          g[e + 1] = q * cs[i] + p * sn[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < P; i++) {
          const float p = x[i], q = y[i];
          x[i] = p * cs[i] - q * sn[i];
          y[i] = q * cs[i] + p * sn[i];
        }
      }
    }
    uint16_t* out = side_of(row, [](const RopeSide& s) { return s.out; }) +
                    ((int64_t)token * side_of(row, [](const RopeSide& s) { return s.heads; }) + head_of(row)) * kD;
    store(out + at0, x);
    store(out + at1, y);
  }
}

// Rows of a lane under way together: one while the workgroups are few (256 tokens x 48 heads, 768 of them, 3.48 us with one, 3.51 with two,
// 3.98 with three; 512: 4.84, 4.72, 5.02), two up to twice that and more (1024: 7.55, 6.74, 7.18), three for large ones (2048: 11.4, 10.6,
// 10.3; 4096: 23.4, 21.1, 19.9; in fp32 28.6, 28.7, 30.0).
template <typename T>
hipError_t launch_rope_type(RopeArgs a, hipStream_t s) {
  const int rows = a.side[0].heads + a.side[1].heads + a.side[2].heads, blocks = (rows + kRows - 1) / kRows;
  const int64_t workgroups = (int64_t)a.n_tokens * blocks;
  auto run = [&](auto each) {
    constexpr int R = decltype(each)::value;
    const int tokens = (int)(((int64_t)a.n_tokens + (1 << a.log2_tokens) - 1) >> a.log2_tokens);
    return launch(qk_norm_rope_kernel<T, R>, dim3(tokens, (rows + kRows * R - 1) / (kRows * R)), kRopeThreads, s, a);
  };
  a.log2_tokens = 0;
  if (blocks == 1)
    while (a.log2_tokens < 4 && rows << (a.log2_tokens + 1) <= kRows) a.log2_tokens++;
  if (blocks == 1 || workgroups < 1200) return run(std::integral_constant<int, 1>{});
  if (sizeof(T) == 4 || blocks == 2 || workgroups < 4800) return run(std::integral_constant<int, 2>{});
  return run(std::integral_constant<int, 3>{});
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, int dtype, hipStream_t s) {
  switch (dtype) {
    case KVMIX_F16: return launch_rope_type<half_t>(a, s);
    case KVMIX_BF16: return launch_rope_type<Bf16>(a, s);
    case KVMIX_F32: return launch_rope_type<float>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace kvmix
