// Shared pieces of the kernels for dropout, residual add and RMS norm: how a row is laid over threads,
// its sums, its weights.
#pragma once

#include "gs_layer.cuh"

namespace gs {
namespace norm {

// Sum over the TPR threads of a row; every thread of the CTA takes part.  Two sums in turn use two
// scratch arrays, so one barrier each is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* scratch) {
#pragma unroll
  for (int o = TPR < 32 ? TPR / 2 : 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  if constexpr (TPR > 32) {
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) scratch[warp] = v;
    __syncthreads();
    constexpr int W = TPR / 32;
    const int first = warp / W * W;
    v = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) v += scratch[first + k];
  }
  return v;
}

// The weights of a group, which start at a 16-byte boundary where the row does not have a lead.
// Otherwise they are taken out of the three words of four that hold them.
template <int L>
__device__ __forceinline__ void weight8(const float* weight, const Span& g, int lead, int cols, float (&w)[8]) {
  if (L == kEven || (L == kTogether && lead == 0 && g.whole())) {
    unpack8<float, kEven>(fetch8<float, kEven>(weight + g.col, g), g, w);
  } else if (L == kTogether && g.whole() && (g.col & ~3) + 12 <= cols) {
    float t[12];
#pragma unroll
    for (int k = 0; k < 3; ++k)
      *reinterpret_cast<float4*>(t + 4 * k) = *reinterpret_cast<const float4*>(weight + (g.col & ~3) + 4 * k);
    const bool one = g.col & 1, two = g.col & 2;
#pragma unroll
    for (int k = 0; k < 11; ++k) t[k] = one ? t[k + 1] : t[k];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = two ? t[k + 2] : t[k];
  } else {
    unpack8<float, kApart>(fetch8<float, kApart>(weight + g.col, g), g, w);
  }
}

// A row has TPR threads; narrow ones share a CTA.
template <int TPR> constexpr int kRowsPerCta = TPR > 128 ? 1 : 256 / TPR;
template <int TPR> constexpr int kCtaThreads = kRowsPerCta<TPR> * TPR;

// Threads a row: with one group of eight a thread up to 256 elements, and for fp32, whose groups take
// twice the registers, as long as 1024 threads do; with two above.  Steps of a half keep most threads
// of any width busy.  Calls f with both numbers as constants.
constexpr int kThreadsOfRow[] = {8, 16, 32, 64, 96, 128, 192, 256, 384, 512, 768, 1024};
struct Shape {
  int tpr, per;       // threads a row, groups a thread
  int rows, threads;  // of a CTA
};
inline Shape shape_of(int wide, bool fp32) {
  Shape s = {1024, 2, 1, 1024};
  for (int tpr : kThreadsOfRow) {
    const int per = tpr < 32 || wide <= 256 || (fp32 && (tpr < 1024 || wide <= 8192)) ? 1 : 2;
    if (wide <= 8 * per * tpr) {
      s.tpr = tpr;
      s.per = per;
      s.rows = tpr > 128 ? 1 : 256 / tpr;
      s.threads = s.rows * tpr;
      break;
    }
  }
  return s;
}
template <bool FP32, typename F>
inline cudaError_t with_shape(const Shape& s, F&& f) {
  using std::integral_constant;
  const auto given = [&](auto tpr) {
    constexpr int TPR = decltype(tpr)::value;
    if constexpr (TPR < 32 || (FP32 && TPR < 1024)) return f(tpr, integral_constant<int, 1>());
    else if constexpr (TPR == 32 || FP32)
      return s.per == 1 ? f(tpr, integral_constant<int, 1>()) : f(tpr, integral_constant<int, 2>());
    else return f(tpr, integral_constant<int, 2>());
  };
  switch (s.tpr) {
    case 8: return given(integral_constant<int, 8>());
    case 16: return given(integral_constant<int, 16>());
    case 32: return given(integral_constant<int, 32>());
    case 64: return given(integral_constant<int, 64>());
    case 96: return given(integral_constant<int, 96>());
    case 128: return given(integral_constant<int, 128>());
    case 192: return given(integral_constant<int, 192>());
    case 256: return given(integral_constant<int, 256>());
    case 384: return given(integral_constant<int, 384>());
    case 512: return given(integral_constant<int, 512>());
    case 768: return given(integral_constant<int, 768>());
    default: return given(integral_constant<int, 1024>());
  }
}

// Elements that a row takes: its first group may start up to seven before it.
inline int width(int cols, Layout layout) { return layout == kTogether ? cols + 7 : cols; }

}  // namespace norm
}  // namespace gs
