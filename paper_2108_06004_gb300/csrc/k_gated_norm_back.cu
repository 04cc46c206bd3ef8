// Backward pass of the norms around a block:
//
//   m = y next_rstd,  u = dz w_next,  t = next_rstd (u - m mean(u m)) + dy,   dresidual = t
//   n = x rstd,  e = scale t,  dgate = e n w act'(gate),  p = e act(gate) w,
//   dx = rstd (p - n mean(p n)),  dw = sum over rows of e act(gate) n,  dw_next = sum over rows of dz m
//
// Every tensor is read and written once.  A CTA takes rows in turn; the weights' gradients are summed by
// each thread over its rows, whose columns and group are the same, then over the CTAs by a last kernel, in a fixed
// order.  Bound by memory.
#include <numeric>

#include "gated_norm.cuh"

namespace gs {
namespace {

using namespace norm;

template <typename E, int TPR, int V, int L>
__global__ void __launch_bounds__(kCtaThreads<TPR>, kCtaThreads<TPR> <= 256 ? 2 : 1)
k_gated_norm_back(const __grid_constant__ GatedNormBackParams p, int outer) {
  grid_begin();
  __shared__ float scratch[2][2][32];
  constexpr int RPC = kRowsPerCta<TPR>;
  extern __shared__ float fold[];  // RPC > 1 and one group a row: [RPC][width]
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  // a thread's rows, `step` apart, have the same lead and the same group
  const int64_t step = (int64_t)gridDim.x * RPC, first = (int64_t)blockIdx.x * RPC;
  const int lead = lead_of<L>(first + sub, p.x_stride, p.lead);
  float dw[V][8], dnext[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[v][j] = dnext[v][j] = 0.f;
  constexpr bool AHEAD = V == 1 && sizeof(E) == 2 && TPR <= 512;
  struct Row {
    Raw8<E> x[V], gate[V], dy[V], dz[V], y[V];
    float rstd, next_rstd;
  };
  const auto fetch = [&](int64_t row, Row& r) {
    if (row >= p.rows) return;
    const bool inner = p.spaced && row > 0 && row + 1 < p.rows;
    r.rstd = p.rstd[row];
    if (p.dz) r.next_rstd = p.next_rstd[row];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Span s = span<L>(v * TPR + lane, lead, p.width);
      if (!s.some()) continue;
      const auto get = [&](const void* t, int64_t stride) {
        return fetch8<E, L>(static_cast<const E*>(t) + group_start(row, outer, stride, p.width) + s.col, s, inner);
      };
      r.x[v] = get(p.x, p.x_stride);
      if (p.gate) r.gate[v] = get(p.gate, p.gate_stride);
      if (p.dy) r.dy[v] = get(p.dy, p.dy_stride);
      if (p.dz) {
        r.dz[v] = get(p.dz, p.dz_stride);
        r.y[v] = get(p.y, p.y_stride);
      }
    }
  };
  Row now;
  if (AHEAD) fetch(first + sub, now);
  int turn = 0;
  for (int64_t row0 = first; row0 < p.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + sub;
    const bool live = row < p.rows;
    Row next;
    if (AHEAD)
      fetch(row + step, next);
    else
      fetch(row, now);
    const auto put = [&](void* t, int64_t stride, const Span& s, const float(&v)[8]) {
      store8<E, L>(static_cast<E*>(t) + group_start(row, outer, stride, p.width) + s.col, s, v);
    };
    float sum = 0.f;
    if (p.dz) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Span s = span<L>(v * TPR + lane, lead, p.width);
        if (!live || !s.some()) continue;
        float dz[8], m[8], w[8];
        weight8<L>(p.next_weight, s, lead, p.width, w);
        unpack8<E, L>(now.dz[v], s, dz);
        unpack8<E, L>(now.y[v], s, m);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float a = dz[j] * (m[j] * now.next_rstd);  // zero where there is no element
          dnext[v][j] += a;
          sum += a * w[j];
        }
      }
      sum = row_sum<TPR>(sum, scratch[0][turn]) / (float)p.width;
    }
    float dn[V][8], inside = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Span s = span<L>(v * TPR + lane, lead, p.width);
      if (!live || !s.some()) continue;
      float t[8], a[8], w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) t[j] = 0.f;
      if (p.dy) unpack8<E, L>(now.dy[v], s, t);
      if (p.dz) {
        float m[8];
        weight8<L>(p.next_weight, s, lead, p.width, w);
        unpack8<E, L>(now.dz[v], s, a);
        unpack8<E, L>(now.y[v], s, m);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] += now.next_rstd * (a[j] * w[j] - m[j] * now.next_rstd * sum);
      }
      if (p.dresidual) put(p.dresidual, p.dresidual_stride, s, t);
      float n[8];
      group_weight8<L>(p.weight, s, lead, p.width, p.groups, row, w);
      unpack8<E, L>(now.x[v], s, n);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        n[j] *= now.rstd;
        t[j] *= p.scale;
      }
      if (p.gate) {
        float u[8], slope[8];
        unpack8<E, L>(now.gate[v], s, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = gate_of(p.act, u[j], slope[j]);
        if (p.dgate) {
#pragma unroll
          for (int j = 0; j < 8; ++j) slope[j] *= t[j] * n[j] * w[j];
          put(p.dgate, p.dgate_stride, s, slope);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] *= u[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = t[j] * n[j];
        dw[v][j] += a;
        dn[v][j] = t[j] * w[j];
        inside += a * w[j];
      }
    }
    inside = row_sum<TPR>(inside, scratch[1][turn]) / (float)p.width;
    if (live && p.dx) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Span s = span<L>(v * TPR + lane, lead, p.width);
        if (!s.some()) continue;
        float n[8];
        unpack8<E, L>(now.x[v], s, n);
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] = now.rstd * (dn[v][j] - n[j] * now.rstd * inside);
        put(p.dx, p.dx_stride, s, n);
      }
    }
    if (AHEAD) now = next;
  }
  const int64_t n = (int64_t)gridDim.x * p.width;
  for (int which = 0; which < (p.next_weight ? 2 : 1); ++which) {
    // rows of sums: one of each CTA, or, where rows have several groups, of each of its rows
    const bool apart = p.groups > 1;
    float* part = p.partial + which * n + (int64_t)blockIdx.x * (apart ? RPC : 1) * p.width;
    float* to = RPC > 1 && !apart ? fold + sub * p.width : part + (apart ? sub * p.width : 0);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Span s = span<L>(v * TPR + lane, lead, p.width);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j >= s.lo && j < s.hi) to[s.col + j] = which ? dnext[v][j] : dw[v][j];
    }
    if (RPC > 1 && !apart) {
      __syncthreads();
      for (int col = threadIdx.x; col < p.width; col += blockDim.x) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < RPC; ++k) sum += fold[k * p.width + col];
        part[col] = sum;
      }
      __syncthreads();
    }
  }
}

// CTAs: as many as stay resident, the rows dealt round robin, so that a thread's rows share their group and (rows
// of a thread being a multiple of eight apart) their lead.
int64_t ctas_of(int64_t rows, int groups, const Shape& shape) {
  const int64_t need = (rows + shape.rows - 1) / shape.rows;
  const int64_t even = groups / std::gcd(groups, shape.rows);  // CTAs whose rows hold whole sets of groups
  int64_t most = (int64_t)kSMs * (shape.threads <= 512 ? 512 / shape.threads : 1);
  const int64_t unit = std::lcm(even, (int64_t)8);
  most = (most + unit - 1) / unit * unit;
  return need < most ? (need + even - 1) / even * even : most;
}

}  // namespace

// CTAs times the sums that each writes, for any alignment of the rows.
int64_t gated_norm_most_sums(int64_t rows, int groups, int wide_cols) {
  int64_t most = 0;
  for (int wide : {wide_cols, wide_cols + 7 <= kNormMaxCols ? wide_cols + 7 : wide_cols}) {
    const Shape shape = gated_shape(wide);
    const int64_t n = ctas_of(rows, groups, shape) * (groups > 1 ? shape.rows : 1);
    most = n > most ? n : most;
  }
  return most;
}

cudaError_t launch_gated_norm_backward(const GatedNormBackParams& p, int outer, float* dweight, float* dnext_weight,
                                       int dtype, Layout layout, cudaStream_t s) {
  if (width(p.width, layout) > kNormMaxCols) layout = kApart;
  const Shape shape = gated_shape(width(p.width, layout));
  const int64_t ctas = ctas_of(p.rows, p.groups, shape);
  if (ctas > 0) {
    const size_t smem = shape.rows > 1 && p.groups == 1 ? (size_t)shape.rows * p.width * sizeof(float) : 0;
    const cudaError_t err = with_type(dtype, [&](auto e) {
      using E = decltype(e);
      return with_gated_shape(shape, [&](auto tpr, auto v) {
        return with_layout(layout, [&](auto how) {
          return launch_cluster(k_gated_norm_back<E, decltype(tpr)::value, decltype(v)::value, decltype(how)::value>,
                                dim3((unsigned)ctas), dim3(shape.threads), smem, 1, s, p, outer);
        });
      });
    });
    if (err != cudaSuccess) return err;
  }
  const int64_t sums = p.groups > 1 ? ctas * shape.rows / p.groups : ctas;
  const cudaError_t err = launch_column_sums(p.partial, sums, (int64_t)p.groups * p.width, nullptr, 0.f, dweight, s);
  if (err != cudaSuccess || !p.next_weight) return err;
  return launch_column_sums(p.partial + ctas * p.width, ctas, p.width, nullptr, 0.f, dnext_weight, s);
}

}  // namespace gs
