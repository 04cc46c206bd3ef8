// Dropout with a mask that is never stored, with an optional residual add, and its backward
// pass (the same kernel without a residual).
//
//   out[e] = (residual[e] +) (u(e) < t ? 0 : x[e] * 65536 / (65536 - t))
//
// with u(e) 16 bits of Philox4x32-10 at counter (e / 8, offset) and t = round(65536 p).  One
// call of the generator gives eight elements, so a thread owns eight adjacent ones.
#include "gs_layer.cuh"

namespace gs {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 2;  // groups of eight whose loads a thread has under way

// FLAT: one row of 8 * groups elements or fewer (the tensors are contiguous).  Otherwise rows
// with strides, `groups` of them a row.  VEC: groups are whole and 16-byte aligned, but for a
// last one of a FLAT row.
template <typename E, bool FLAT, bool VEC, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads) k_dropout(const __grid_constant__ DropoutParams p, int64_t groups) {
  grid_begin();
  const int64_t total = groups * p.rows, step = (int64_t)gridDim.x * kThreads;
  for (int64_t g0 = (int64_t)blockIdx.x * kThreads + threadIdx.x; g0 < total; g0 += kAhead * step) {
    Raw8<E> x[kAhead], res[kAhead];
    int64_t row[kAhead], col[kAhead];
    int n[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t g = g0 + u * step;
      row[u] = FLAT ? 0 : total <= 0xFFFFFFFFll ? (int64_t)((uint32_t)g / (uint32_t)groups) : g / groups;
      col[u] = (g - row[u] * groups) * 8;
      n[u] = g < total ? (int)(p.cols - col[u] < 8 ? p.cols - col[u] : 8) : 0;
      const E* px = static_cast<const E*>(p.x) + row[u] * p.x_stride + col[u];
      const E* pr = static_cast<const E*>(p.residual) + row[u] * p.residual_stride + col[u];
      if (VEC && n[u] == 8) {
        x[u] = fetch8<E, true>(px, 8);
        if (RESIDUAL) res[u] = fetch8<E, true>(pr, 8);
      } else {
        x[u] = fetch8<E, false>(px, n[u]);
        if (RESIDUAL) res[u] = fetch8<E, false>(pr, n[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (n[u] == 0) continue;
      float v[8];
      unpack8(x[u], v);
      drop8<(FLAT || VEC)>(v, (uint64_t)(row[u] * p.cols + col[u]), p.drop);
      if (RESIDUAL) {
        float w[8];
        unpack8(res[u], w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += w[j];
      }
      E* po = static_cast<E*>(p.out) + row[u] * p.out_stride + col[u];
      if (VEC && n[u] == 8)
        store8<E, true>(po, 8, v);
      else
        store8<E, false>(po, n[u], v);
    }
  }
}

template <typename E, bool FLAT, bool VEC>
cudaError_t run(const DropoutParams& p, cudaStream_t s) {
  const int64_t groups = (p.cols + 7) / 8;
  const int64_t ctas = (groups * p.rows + kThreads - 1) / kThreads;
  const int64_t most = (int64_t)kSMs * 64;
  const dim3 grid((unsigned)(ctas < most ? ctas : most));
  return p.residual ? launch(k_dropout<E, FLAT, VEC, true>, grid, dim3(kThreads), s, p, groups)
                    : launch(k_dropout<E, FLAT, VEC, false>, grid, dim3(kThreads), s, p, groups);
}

}  // namespace

cudaError_t launch_dropout(const DropoutParams& p, int dtype, bool vec, cudaStream_t s) {
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    if (p.rows == 1) return vec ? run<E, true, true>(p, s) : run<E, true, false>(p, s);
    return vec ? run<E, false, true>(p, s) : run<E, false, false>(p, s);
  });
}

}  // namespace gs
