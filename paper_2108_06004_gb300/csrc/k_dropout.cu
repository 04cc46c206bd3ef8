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

// FLAT: one row of 8 * groups elements or fewer (the tensors are contiguous).  Otherwise rows
// with strides, `groups` of them a row.  VEC: groups are whole and 16-byte aligned, but for a
// last one of a FLAT row.
template <typename E, bool FLAT, bool VEC>
__global__ void __launch_bounds__(kThreads) k_dropout(const __grid_constant__ DropoutParams p, int64_t groups) {
  grid_begin();
  const E* x = static_cast<const E*>(p.x);
  const E* res = static_cast<const E*>(p.residual);
  E* out = static_cast<E*>(p.out);
  const int64_t total = groups * p.rows;
  for (int64_t g = (int64_t)blockIdx.x * kThreads + threadIdx.x; g < total; g += (int64_t)gridDim.x * kThreads) {
    const int64_t row = FLAT ? 0 : (total <= 0xFFFFFFFFll ? (int64_t)((uint32_t)g / (uint32_t)groups) : g / groups);
    const int64_t col = (g - row * groups) * 8;
    const int n = (int)(p.cols - col < 8 ? p.cols - col : 8);
    const uint32_t bits = keep8<(FLAT || VEC)>((uint64_t)(row * p.cols + col), p.drop);
    const E* px = x + row * p.x_stride + col;
    const E* pr = res + row * p.residual_stride + col;
    E* po = out + row * p.out_stride + col;
    float v[8], w[8];
    if (VEC && n == 8) {
      load8<E, true>(px, 8, v);
      if (res) load8<E, true>(pr, 8, w);
    } else {
      load8<E, false>(px, n, v);
      if (res) load8<E, false>(pr, n, w);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = drop(v[j], bits, j, p.drop.scale) + (res ? w[j] : 0.f);
    if (VEC && n == 8)
      store8<E, true>(po, 8, v);
    else
      store8<E, false>(po, n, v);
  }
}

template <typename E, bool FLAT, bool VEC>
cudaError_t run(const DropoutParams& p, cudaStream_t s) {
  const int64_t groups = (p.cols + 7) / 8;
  const int64_t ctas = (groups * p.rows + kThreads - 1) / kThreads;
  const int64_t most = (int64_t)device_info().sms * 64;
  return launch(k_dropout<E, FLAT, VEC>, dim3((unsigned)(ctas < most ? ctas : most)), dim3(kThreads), s, p, groups);
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
