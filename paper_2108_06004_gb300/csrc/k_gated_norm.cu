// The norm after a block, its gate and residual scale, and the norm before the next block, in one
// pass over a row.
//
//   rstd = (mean(x^2) + eps)^(-1/2),  y = residual + scale act(gate) x rstd w,
//   next_rstd = (mean(y^2) + eps)^(-1/2),  z = y next_rstd w_next
//
// A row (or a group of its columns, where there is no next norm) is held in the registers of its threads, so
// every tensor is read and written once.  Bound by memory; 4096x1024 bf16 takes 11 us on the device, 54 % of the copy rate
// (two sums over a row one after the other, in 1.4 waves of CTAs).
#include "gated_norm.cuh"

namespace gs {
namespace {

using namespace norm;

template <typename E, int TPR, int V, int L>
// Registers for 1536 threads of an SM: those of 2-byte types with no more than 128 threads a row have 46 without the cap.
__global__ void __launch_bounds__(kCtaThreads<TPR>, V == 1 && sizeof(E) == 2 && TPR <= 768 ? 1536 / kCtaThreads<TPR> : 1)
k_gated_norm(const __grid_constant__ GatedNormParams p, int outer) {
  grid_begin();
  __shared__ float scratch[2][32];
  constexpr int RPC = kRowsPerCta<TPR>;
  const int lane = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * RPC + threadIdx.x / TPR;
  const bool live = row < p.rows, inner = p.spaced && row > 0 && row + 1 < p.rows;
  const int lead = lead_of<L>(row, p.x_stride, p.lead);
  const auto from = [&](const void* t, int64_t stride) { return static_cast<const E*>(t) + group_start(row, outer, stride, p.width); };
  const Gate<E> gate(p.act);
  Eight t[V];
  Raw8<E> gates[V], residual[V];
  float2 sum = two(0.f);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const Span s = span<L>(v * TPR + lane, lead, p.width);
    if (!live || !s.some()) continue;
    const Raw8<E> x = fetch8<E, L>(from(p.x, p.x_stride) + s.col, s, inner);
    if (p.gate) gates[v] = fetch8<E, L>(from(p.gate, p.gate_stride) + s.col, s, inner);
    if (p.residual) residual[v] = fetch8<E, L>(from(p.residual, p.residual_stride) + s.col, s, inner);
    unpack<E, L>(x, s, t[v]);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = fma(t[v][j], t[v][j], sum);
  }
  const float rstd = rsqrtf(row_sum<TPR>(sum.x + sum.y, scratch[0]) / (float)p.width + p.eps);
  if (live && lane == 0) p.rstd[row] = rstd;
  sum = two(0.f);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const Span s = span<L>(v * TPR + lane, lead, p.width);
    if (!live || !s.some()) continue;
    Eight w;
    group_weight8<L>(p.weight, s, lead, p.width, p.groups, row, reinterpret_cast<float(&)[8]>(w));
#pragma unroll
    for (int j = 0; j < 4; ++j) t[v][j] = mul(t[v][j], mul(w[j], rstd * p.scale));
    if (p.gate) {
      unpack<E, L>(gates[v], s, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) t[v][j] = mul(t[v][j], gate.value(w[j]));
    }
    if (p.residual) {
      unpack<E, L>(residual[v], s, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) t[v][j] = add(t[v][j], w[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = fma(t[v][j], t[v][j], sum);  // zero where there is no element
    store8<E, L>(static_cast<E*>(p.y) + group_start(row, outer, p.y_stride, p.width) + s.col, s, reinterpret_cast<float(&)[8]>(t[v]));
  }
  if (!p.next_weight) return;
  const float next = rsqrtf(row_sum<TPR>(sum.x + sum.y, scratch[1]) / (float)p.width + p.eps);
  if (!live) return;
  if (lane == 0) p.next_rstd[row] = next;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const Span s = span<L>(v * TPR + lane, lead, p.width);
    if (!s.some()) continue;
    Eight w;
    weight8<L>(p.next_weight, s, lead, p.width, reinterpret_cast<float(&)[8]>(w));
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = mul(w[j], mul(t[v][j], next));
    store8<E, L>(static_cast<E*>(p.z) + row * p.z_stride + s.col, s, reinterpret_cast<float(&)[8]>(w));
  }
}

}  // namespace

cudaError_t launch_gated_norm(const GatedNormParams& p, int outer, int dtype, Layout layout, cudaStream_t s) {
  if (width(p.width, layout) > kNormMaxCols) layout = kApart;
  const Shape shape = gated_shape(width(p.width, layout));
  const int64_t ctas = (p.rows + shape.rows - 1) / shape.rows;
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return with_gated_shape(shape, [&](auto tpr, auto v) {
      return with_layout(layout, [&](auto how) {
        return launch(k_gated_norm<E, decltype(tpr)::value, decltype(v)::value, decltype(how)::value>, dim3((unsigned)ctas),
                      dim3(shape.threads), s, p, outer);
      });
    });
  });
}

}  // namespace gs
