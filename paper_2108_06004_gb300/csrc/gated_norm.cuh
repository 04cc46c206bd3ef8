// Shared pieces of the kernels for the norms around a block: rows and groups, the gate, sums.
#pragma once

#include "attention.cuh"
#include "dropout_norm.cuh"

namespace gs {
namespace norm {

// Where row r (of groups) starts, in a tensor whose rows of all groups are `stride` apart; `outer`
// is 1 where the groups of all rows are evenly apart, so that they are rows themselves.
__device__ __forceinline__ int64_t group_start(int64_t r, int outer, int64_t stride, int width) {
  return outer == 1 ? r * stride : r / outer * stride + r % outer * width;
}

// The weights of a group of eight columns of group `g` of a row.  Only a first group's are sure to start at a
// 16-byte boundary where the width is odd.
template <int L>
__device__ __forceinline__ void group_weight8(const float* weight, const Span& s, int lead, int width, int groups,
                                              int64_t r, float (&w)[8]) {
  if (groups == 1) {
    weight8<L>(weight, s, lead, width, w);
  } else {
    weight += r % groups * width;
    if (L == kEven)
      weight8<kEven>(weight, s, 0, width, w);
    else
      unpack8<float, kApart>(fetch8<float, kApart>(weight + s.col, s), s, w);
  }
}

// Two adjacent elements with one instruction.
__device__ __forceinline__ float2 two(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 mul(float2 a, float b) { return __fmul2_rn(a, two(b)); }
__device__ __forceinline__ float2 add(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 fma(float2 a, float b, float2 c) { return __ffma2_rn(a, two(b), c); }
using Eight = float2[4];
template <typename E, int L>
__device__ __forceinline__ void unpack(const Raw8<E>& r, const Span& g, Eight& v) {
  unpack8<E, L>(r, g, reinterpret_cast<float(&)[8]>(v));
}

// act(u), and its slope: with s(u) = 1 / (1 + e^-u), a = act(u) and 1 - s = e^-u s, a (1 - s) + s for u s and s (1 - s) for s.
// For fp32 e^-u is right to a unit in the last place whatever u is. For 16-bit types it comes from the base-two
// exponential of a rounded product, off by |u| 2^-24 of itself, which is far below a rounding of theirs as long as s is not zero (its
// exponent stops where s is zero in fp32), and the approximate reciprocal: 32768x4096 bf16 backward takes 429 us from cold
// with them, 552 with fp32's; fp32 16384x1024 backward 175 us, 163 with the approximate ones.
__device__ __forceinline__ float power(float x) {
  float y;
  asm("{\n .reg .f32 t;\n min.NaN.f32 t, %1, 0f42FE0000;\n ex2.approx.ftz.f32 %0, t;\n}" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float inverse(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <typename E>
struct Gate {
  bool silu;
  __device__ __forceinline__ explicit Gate(int act) : silu(act == GS_GATE_SILU) {}
  // s and 1 - s
  static __device__ __forceinline__ float2 open(float2 u, float2& rest) {
    if constexpr (sizeof(E) == 4) {
      const float2 e = make_float2(expf(-u.x), expf(-u.y));
      const float2 s = make_float2(__frcp_rn(e.x + 1.f), __frcp_rn(e.y + 1.f));
      rest = make_float2(isinf(e.x) ? 1.f : e.x * s.x, isinf(e.y) ? 1.f : e.y * s.y);
      return s;
    } else {
      const float2 x = mul(u, -1.4426950408889634f), e = make_float2(power(x.x), power(x.y)), d = add(e, two(1.f));
      const float2 s = make_float2(inverse(d.x), inverse(d.y));
      rest = mul(e, s);
      return s;
    }
  }
  __device__ __forceinline__ float2 value(float2 u, float2& slope) const {
    float2 rest;
    const float2 s = open(u, rest);
    if (silu) {
      const float2 a = mul(u, s);
      slope = fma(a, rest, s);
      return a;
    }
    slope = mul(s, rest);
    return s;
  }
  __device__ __forceinline__ float2 value(float2 u) const {
    float2 slope;
    return value(u, slope);
  }
};

// N sums at once over the TPR threads of a row; every thread of the CTA takes part.  Two calls in turn use two
// scratch arrays, so one barrier each is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*scratch)[32]) {
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int o = TPR < 32 ? TPR / 2 : 16; o > 0; o >>= 1) v[n] += __shfl_xor_sync(0xFFFFFFFFu, v[n], o);
  if constexpr (TPR > 32) {
    constexpr int W = TPR / 32;
    const int warp = threadIdx.x >> 5, first = warp / W * W;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) scratch[n][warp] = v[n];
    }
    __syncthreads();
    // every warp adds the warps' sums up itself, a lane each, all lanes in the same order
#pragma unroll
    for (int n = 0; n < N; ++n) {
      v[n] = (threadIdx.x & 31) < W ? scratch[n][first + (threadIdx.x & 31)] : 0.f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        if (o < W) v[n] += __shfl_xor_sync(0xFFFFFFFFu, v[n], o);
      v[n] = __shfl_sync(0xFFFFFFFFu, v[n], 0);
    }
  }
}

// Threads a row and groups of eight a thread: one as long as 1024 threads do.
inline Shape gated_shape(int wide) {
  Shape s = {1024, 2, 1, 1024};
  for (int tpr : kThreadsOfRow)
    if (wide <= 8 * tpr) {
      s.tpr = tpr;
      s.per = 1;
      s.rows = tpr > 128 ? 1 : 256 / tpr;
      s.threads = s.rows * tpr;
      break;
    }
  return s;
}
template <typename F>
inline cudaError_t with_gated_shape(const Shape& s, F&& f) {
  using std::integral_constant;
  const integral_constant<int, 1> one;
  switch (s.tpr) {
    case 8: return f(integral_constant<int, 8>(), one);
    case 16: return f(integral_constant<int, 16>(), one);
    case 32: return f(integral_constant<int, 32>(), one);
    case 64: return f(integral_constant<int, 64>(), one);
    case 96: return f(integral_constant<int, 96>(), one);
    case 128: return f(integral_constant<int, 128>(), one);
    case 192: return f(integral_constant<int, 192>(), one);
    case 256: return f(integral_constant<int, 256>(), one);
    case 384: return f(integral_constant<int, 384>(), one);
    case 512: return f(integral_constant<int, 512>(), one);
    case 768: return f(integral_constant<int, 768>(), one);
    default: return s.per == 1 ? f(integral_constant<int, 1024>(), one) : f(integral_constant<int, 1024>(), integral_constant<int, 2>());
  }
}

}  // namespace norm
}  // namespace gs
