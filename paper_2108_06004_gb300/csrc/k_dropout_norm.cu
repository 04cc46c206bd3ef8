// Dropout, residual add and RMS norm in one pass over a row.
//
//   y = residual + dropout(x),  rstd = (mean(y^2) + eps)^(-1/2),  z = y rstd w
//
// A row is held in the registers of its threads, one or two groups of eight elements each, so every
// tensor is read and written once.  Bound by memory: 32768x4096 takes 158 us in bf16 and 302 us in fp32 (both at
// the copy rate), 131072x64 13 us (76 %), 4096x1024 7.8 us (63 %: one wave of CTAs, whose rows pass
// from load to store once).  Rows that start anywhere: 16384x4097 129 us (61 %), 32768x1001 66 us (59 %),
// 131072x65 40 us (25 %); tensors whose rows differ in alignment, or a weight that does not start at a
// 16-byte boundary, make all elements move one by one: 32768x1024 138 us (43 with an aligned weight).
#include "dropout_norm.cuh"

namespace gs {
namespace {

using namespace norm;

// Few enough registers that 1792 threads stay resident: 4096x1024 bf16 takes 7.8 us with seven CTAs
// of 256 threads an SM, 9.4 us with the five that the compiler's own choice leaves room for.  Rows of 2-byte
// types that start anywhere spill up to 176 bytes a thread for it (their groups take more registers), and are
// faster all the same where they are wide (16384x4097 129 us, 183 without the cap; 16384x2047 70, 81;
// 131072x65 40, 42) or within 7 % (65536x257 65, 61); 300x1001, a call of 3 us, is 0.5 us slower.
template <typename E, int TPR, int V, int L>
__global__ void __launch_bounds__(kCtaThreads<TPR>, 1792 / kCtaThreads<TPR>)
k_norm_forward(const __grid_constant__ NormForwardParams p) {
  grid_begin();
  __shared__ float scratch[32];
  constexpr int RPC = kRowsPerCta<TPR>;
  const int lane = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * RPC + threadIdx.x / TPR;
  const bool live = row < p.rows;
  const int lead = lead_of<L>(row, p.x_stride, p.lead);
  float t[V][8];
  float sum = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const Span g = span<L>(v * TPR + lane, lead, p.cols);
    if (!live || !g.some()) continue;
    float res[8];
    const bool inner = p.spaced && row > 0 && row + 1 < p.rows;
    const Raw8<E> raw_x = fetch8<E, L>(static_cast<const E*>(p.x) + row * p.x_stride + g.col, g, inner);
    const Raw8<E> raw_res = fetch8<E, L>(static_cast<const E*>(p.residual) + row * p.residual_stride + g.col, g, inner);
    unpack8<E, L>(raw_x, g, t[v]);
    unpack8<E, L>(raw_res, g, res);
    drop8<L == kEven>(t[v], row * p.cols + g.col, p.drop);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      t[v][j] += res[j];  // zero where there is no element
      sum += t[v][j] * t[v][j];
    }
    store8<E, L>(static_cast<E*>(p.y) + row * p.y_stride + g.col, g, t[v]);
  }
  sum = row_sum<TPR>(sum, scratch);
  const float rstd = rsqrtf(sum / (float)p.cols + p.eps);
  if (!live) return;
  if (lane == 0) p.rstd[row] = rstd;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const Span g = span<L>(v * TPR + lane, lead, p.cols);
    if (!g.some()) continue;
    float w[8];
    weight8<L>(p.weight, g, lead, p.cols, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] *= t[v][j] * rstd;
    store8<E, L>(static_cast<E*>(p.z) + row * p.z_stride + g.col, g, w);
  }
}

}  // namespace

cudaError_t launch_norm_forward(const NormForwardParams& p, int dtype, Layout layout, cudaStream_t s) {
  if (width(p.cols, layout) > kNormMaxCols) layout = kApart;  // the row with its lead does not fit
  const Shape shape = shape_of(width(p.cols, layout), dtype == GS_F32);
  const int64_t ctas = (p.rows + shape.rows - 1) / shape.rows;
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return with_shape<sizeof(E) == 4>(shape, [&](auto tpr, auto v) {
      return with_layout(layout, [&](auto how) {
        return launch(k_norm_forward<E, decltype(tpr)::value, decltype(v)::value, decltype(how)::value>, dim3((unsigned)ctas),
                      dim3(shape.threads), s, p);
      });
    });
  });
}

}  // namespace gs
