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

// act(u), and its slope: 1 - sigmoid is e^-u sigmoid, and one where e^-u is past fp32.
__device__ __forceinline__ float gate_of(int act, float u, float& slope) {
  const float e = __expf(-u), s = __fdividef(1.f, 1.f + e), rest = s > 0.f ? e * s : 1.f;
  slope = act == GS_GATE_SILU ? s * fmaf(u, rest, 1.f) : s * rest;
  return act == GS_GATE_SILU ? u * s : s;
}
__device__ __forceinline__ float gate_of(int act, float u) {
  float slope;
  return gate_of(act, u, slope);
}

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
#pragma unroll
    for (int n = 0; n < N; ++n) {
      v[n] = 0.f;
#pragma unroll
      for (int k = 0; k < W; ++k) v[n] += scratch[n][first + k];
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
