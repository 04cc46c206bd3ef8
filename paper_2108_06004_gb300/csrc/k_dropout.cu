// Dropout with a mask that is never stored, with an optional residual add, and its backward
// pass (the same kernel without a residual).
//
//   out[e] = (residual[e] +) (u(e) < t ? 0 : x[e] * 65536 / (65536 - t))
//
// with u(e) 16 bits of Philox4x32-10 at counter (e / 8, offset) and t = round(65536 p).  One
// call of the generator gives eight elements, so a thread owns eight adjacent ones, and issues
// the loads of two such groups before it works on either.
//
// Bound by memory but for bf16 without a residual, where the generator's integer instructions (64 % of
// their pipe) come close: 16384x4096 takes 42 us in bf16 (94 % of the copy rate, 98 % with p = 0), 58 us
// with a residual and 79 us in fp32 (both at the copy rate).  Rows with strides take 51 us (a
// division a group).  Where rows are padded and their width is no multiple of eight, a group lies in two blocks
// of the generator, and all ten rounds are run for both: 16384x4097 71 us, 121 us with rows that differ in
// alignment too (single elements).
#include "gs_layer.cuh"

namespace gs {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 2;  // groups of eight whose loads a thread has under way

// n / d for n below 2^31: with 2^(k-1) < d <= 2^k and m = floor(2^(31+k) / d) + 1, m n / 2^(31+k) exceeds
// n / d by less than n / 2^(31+k) < 1 / d, which does not reach the next whole number.
struct Divisor {
  uint32_t d, m, k;
};
Divisor divisor(uint32_t d) {
  uint32_t k = 0;
  while ((uint64_t(1) << k) < d) ++k;
  return Divisor{d, (uint32_t)(((uint64_t(1) << 31) << k) / d + 1), k};
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const Divisor& v) {
  return (uint32_t)((uint64_t)n * v.m >> 31 >> v.k);
}

// ROWS 0: one row (the tensors are contiguous); 1: rows of `groups` groups, fewer than 2^31 in all;
// 2: any number.
template <typename E, int ROWS, int L, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads)
k_dropout(const __grid_constant__ DropoutParams p, int64_t groups, Divisor by_groups) {
  grid_begin();
  const int64_t total = groups * p.rows, step = (int64_t)gridDim.x * kThreads;
  for (int64_t g0 = (int64_t)blockIdx.x * kThreads + threadIdx.x; g0 < total; g0 += kAhead * step) {
    Raw8<E> x[kAhead], res[kAhead];
    int64_t row[kAhead], col[kAhead];
    Span part[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t g = g0 + u * step;
      row[u] = ROWS == 0 ? 0 : ROWS == 1 ? (int64_t)divide((uint32_t)g, by_groups) : g / groups;
      const int lead = lead_of<L>(row[u], p.x_stride, p.lead);
      col[u] = (g - row[u] * groups) * 8 - lead;
      part[u] = span<L>(g - row[u] * groups, lead, p.cols);
      if (g >= total) part[u].hi = part[u].lo = 0;
      if (!part[u].some()) continue;
      const bool inner = ROWS > 0 && p.spaced && row[u] > 0 && row[u] + 1 < p.rows;
      x[u] = fetch8<E, L>(static_cast<const E*>(p.x) + row[u] * p.x_stride + col[u], part[u], inner);
      if (RESIDUAL)
        res[u] = fetch8<E, L>(static_cast<const E*>(p.residual) + row[u] * p.residual_stride + col[u], part[u], inner);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (!part[u].some()) continue;
      float v[8];
      unpack8<E, L>(x[u], part[u], v);
      drop8<L == kEven>(v, row[u] * p.cols + col[u], p.drop);
      if (RESIDUAL) {
        float w[8];
        unpack8<E, L>(res[u], part[u], w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += w[j];
      }
      store8<E, L>(static_cast<E*>(p.out) + row[u] * p.out_stride + col[u], part[u], v);
    }
  }
}

template <typename E, int ROWS, int L>
cudaError_t run(const DropoutParams& p, int64_t groups, cudaStream_t s) {
  const int64_t ctas = (groups * p.rows + kThreads - 1) / kThreads;
  const int64_t most = (int64_t)kSMs * 64;
  const dim3 grid((unsigned)(ctas < most ? ctas : most));
  const Divisor by = ROWS == 1 ? divisor((uint32_t)groups) : Divisor{};
  return p.residual ? launch(k_dropout<E, ROWS, L, true>, grid, dim3(kThreads), s, p, groups, by)
                    : launch(k_dropout<E, ROWS, L, false>, grid, dim3(kThreads), s, p, groups, by);
}

}  // namespace

cudaError_t launch_dropout(const DropoutParams& p, int dtype, Layout layout, cudaStream_t s) {
  // a row's last group may start up to seven columns earlier than its number says
  const int64_t groups = (p.cols + 7) / 8 + (layout == kTogether ? 1 : 0);
  // groups past the end of the last one are asked for too, before they are found not to exist
  const bool few = groups * p.rows < (int64_t(1) << 31) - kAhead * int64_t(kSMs) * 64 * kThreads;
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return with_layout(layout, [&](auto how) {
      constexpr int L = decltype(how)::value;
      return p.rows == 1 ? run<E, 0, L>(p, groups, s) : few ? run<E, 1, L>(p, groups, s) : run<E, 2, L>(p, groups, s);
    });
  });
}

}  // namespace gs
