// Queries, Keys and Values between the projections and the cache (gfx950): norm of each head, rotation by position, conversion to fp16.
//
// y = x / sqrt(mean(x^2) + eps) * w;  pair (a, b) of y and angle t = position * frequency:  (a cos t - b sin t, b cos t + a sin t).
// Memory-bound: 2 or 4 bytes in and 2 out per element. 16 lanes have a row of 128 channels, 8 channels each, so that both
// channels of a pair belong to one lane: 4 consecutive ones of either half of the rotated part (pairs (i, i + r/2)) or 8 consecutive ones
// (neighbours, and what is not rotated). No lane needs another's values but for the sum of squares. Every row of a token turns by the same
// angles: a lane has 4 of them, made once for all the rows that it takes.
// An angle is a fraction of a turn taken in binary64: position * frequency in fp32 is off by up to position * 2^-24 radians, 0.06 at a
// million.
#include <type_traits>
#include "kvmix_common.hpp"

namespace kvmix {

namespace {

struct Bf16 { uint16_t bits; };
template <typename T> struct Four;          // 4 consecutive elements as loaded
template <> struct Four<half_t> {
  u32x2_t w;
  __device__ __forceinline__ void get(float (&x)[4]) const {
    const uint32_t a = w[0], b = w[1];       // (copies: a bit cast applied to the vector element itself reads element 0)
    const half2_t p = __builtin_bit_cast(half2_t, a), q = __builtin_bit_cast(half2_t, b);
    x[0] = (float)p[0]; x[1] = (float)p[1]; x[2] = (float)q[0]; x[3] = (float)q[1];
  }
};
template <> struct Four<Bf16> {
  u32x2_t w;
  __device__ __forceinline__ void get(float (&x)[4]) const {
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const uint32_t v = w[i], lo = v << 16, hi = v & 0xFFFF0000u;
      x[2 * i] = __builtin_bit_cast(float, lo); x[2 * i + 1] = __builtin_bit_cast(float, hi);
    }
  }
};
template <> struct Four<float> {
  float4_t w;
  __device__ __forceinline__ void get(float (&x)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = w[i];
  }
};
template <typename T> __device__ __forceinline__ Four<T> load4(const void* base, int64_t at) {
  Four<T> r;
  r.w = *reinterpret_cast<const decltype(r.w)*>(reinterpret_cast<const T*>(base) + at);
  return r;
}
__device__ __forceinline__ void store4(uint16_t* p, const float (&x)[4]) {
  const half2_t a = {(half_t)x[0], (half_t)x[1]}, b = {(half_t)x[2], (half_t)x[3]};
  *reinterpret_cast<u32x2_t*>(p) = u32x2_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
// sum over the 16 lanes of each row; every lane of the row gets it
__device__ __forceinline__ float row_sum(float v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  v += dpp<0x141>(v);
  v += dpp<0x140>(v);
  return v;
}

constexpr int kRopeThreads = 256;
// R: rows of a lane under way together; grid (tokens, blocks of 16 R rows)
template <typename T, int R>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(RopeArgs a) {
  const int token = blockIdx.x, c = threadIdx.x & 15;
  const int turned = a.rotary_dim / 8;                 // lanes that have pairs
  // first channels of the lane's two fours
  const bool halves = !a.interleaved && c < turned;
  const int at0 = halves ? 4 * c : 8 * c, at1 = halves ? a.rotary_dim / 2 + 4 * c : 8 * c + 4;
  const int n_q = a.side[0].heads, n_k = a.side[1].heads, rows = n_q + n_k + a.side[2].heads;
  Four<T> x0[R], x1[R], w0[R], w1[R];
  int side[R], head[R];
#pragma unroll
  for (int k = 0; k < R; k++) {
    const int row = (blockIdx.y * R + k) * (kRopeThreads / 16) + (int)(threadIdx.x >> 4);
    side[k] = row >= rows ? -1 : row < n_q ? 0 : row < n_q + n_k ? 1 : 2;
    head[k] = row - (side[k] >= 1 ? n_q : 0) - (side[k] == 2 ? n_k : 0);
    if (side[k] < 0) continue;
    const RopeSide& s = a.side[side[k]];
    const int64_t at = (int64_t)token * s.tok + (int64_t)head[k] * s.head;
    x0[k] = load4<T>(s.in, at + at0);
    x1[k] = load4<T>(s.in, at + at1);
    if (s.weight) { w0[k] = load4<T>(s.weight, at0); w1[k] = load4<T>(s.weight, at1); }
  }
  float cs[4], sn[4];
  if (c < turned) {
    const double pos = (double)a.positions[token];
    const float4_t f = *reinterpret_cast<const float4_t*>(a.frequencies + 4 * c);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      double t = pos * ((double)f[i] * 0.15915494309189533577);
      t -= rint(t);
      float s, co;
      sincospif(2.0f * (float)t, &s, &co);
      cs[i] = co * a.amplitude;
      sn[i] = s * a.amplitude;
    }
  }
#pragma unroll
  for (int k = 0; k < R; k++) {
    if (side[k] < 0) continue;
    const RopeSide& s = a.side[side[k]];
    float x[4], y[4];
    x0[k].get(x);
    x1[k].get(y);
    if (s.weight) {
      float sum = 0.0f, u[4], v[4];
#pragma unroll
      for (int i = 0; i < 4; i++) sum += x[i] * x[i] + y[i] * y[i];
      const float r = rsqrtf(row_sum(sum) * (1.0f / kD) + a.eps);
      w0[k].get(u);
      w1[k].get(v);
#pragma unroll
      for (int i = 0; i < 4; i++) { x[i] = x[i] * r * u[i]; y[i] = y[i] * r * v[i]; }
    }
    if (side[k] < 2 && c < turned) {
      if (a.interleaved) {
        const float p[4] = {x[0], x[2], y[0], y[2]}, q[4] = {x[1], x[3], y[1], y[3]};
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const float even = p[i] * cs[i] - q[i] * sn[i], odd = q[i] * cs[i] + p[i] * sn[i];
          (i < 2 ? x : y)[2 * (i & 1)] = even;
          (i < 2 ? x : y)[2 * (i & 1) + 1] = odd;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const float p = x[i], q = y[i];
          x[i] = p * cs[i] - q * sn[i];
          y[i] = q * cs[i] + p * sn[i];
        }
      }
    }
    uint16_t* out = s.out + ((int64_t)token * s.heads + head[k]) * kD;
    store4(out + at0, x);
    store4(out + at1, y);
  }
}

template <typename T>
hipError_t launch_rope_type(const RopeArgs& a, hipStream_t s) {
  const int rows = a.side[0].heads + a.side[1].heads + a.side[2].heads, each = kRopeThreads / 16;
  return launch(qk_norm_rope_kernel<T, 1>, dim3(a.n_tokens, (rows + each - 1) / each), kRopeThreads, s, a);
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
