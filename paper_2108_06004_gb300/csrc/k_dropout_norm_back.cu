// Backward pass of dropout, residual add and RMS norm, from dz, dy (the gradient that reaches y past
// the norm) and the stored y:
//
//   n = y rstd,  u = dz w,  dt = rstd (u - n mean(u n)) + dy
//   dresidual = dt,  dx = mask dt scale,  dw = sum over rows of dz n
//
// Every tensor is read and written once.  A CTA takes rows in turn, the next one's loads under way while
// it works on one; dw is summed by each thread over the rows of its CTA, then over the CTAs by a
// last kernel, in a fixed order.  Bound by memory: 32768x4096 takes 205 us in bf16 (97 % of the copy
// rate; 511 us when a row's loads waited for the row before), 65536x1024 105 us (95 %), fp32 16384x4096
// 205 us (97 %).  What is in flight goes by threads and registers: past 4096 columns of a 2-byte type a row
// takes 384 threads, of which one CTA fits an SM where two of 256 did, and bf16 16384x4104 takes 137 us (73 %),
// 16384x5120 151 us (82 %), 16384x6144 170 us (88 %).  Rows that start anywhere pay for single elements at both ends
// and weights out of step with the groups on top: 16384x4097 211 us (47 %), 32768x1001 85 us (57 %).  Above
// 8192 columns (fp32 4096) the next row is not loaded ahead: 16384x12288 412 us (72 %), 16384x16384 572 us (69 %).
// Single elements throughout (see the forward pass): 32768x1024 180 us, 56 with an aligned weight.
#include "dropout_norm.cuh"

namespace gs {
namespace {

using namespace norm;

template <typename E, int TPR, int V, int L>
__global__ void __launch_bounds__(kCtaThreads<TPR>, kCtaThreads<TPR> <= 256 ? 2 : 1)
k_norm_backward(const __grid_constant__ NormBackwardParams p) {
  grid_begin();
  __shared__ float scratch[2][32];
  constexpr int RPC = kRowsPerCta<TPR>;
  extern __shared__ float fold[];  // RPC > 1: [RPC][cols]
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  // a thread's rows, `step` apart, all have the same lead: step is a multiple of eight where a thread
  // has more than one
  const int64_t step = (int64_t)gridDim.x * RPC, first = (int64_t)blockIdx.x * RPC;
  const int lead = lead_of<L>(first + sub, p.dz_stride, p.lead);
  float dw[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[v][j] = 0.f;
  // A row's inputs stay as they are in memory and are unpacked once for the sums and again for the
  // results: half the registers that fp32 values take.  The next row's are loaded meanwhile, but in the
  // widest rows, whose 768 threads and more have registers for one row only.
  constexpr bool AHEAD = TPR < 768;
  Raw8<E> dz[V], y[V], dy[V];
  float rstd = 0.f;
  auto fetch = [&](int64_t row, Raw8<E>(&dz)[V], Raw8<E>(&y)[V], Raw8<E>(&dy)[V], float& rstd) {
    if (row >= p.rows) return;
    rstd = p.rstd[row];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Span g = span<L>(v * TPR + lane, lead, p.cols);
      if (!g.some()) continue;
      const bool inner = p.spaced && row > 0 && row + 1 < p.rows;
      dz[v] = fetch8<E, L>(static_cast<const E*>(p.dz) + row * p.dz_stride + g.col, g, inner);
      y[v] = fetch8<E, L>(static_cast<const E*>(p.y) + row * p.y_stride + g.col, g, inner);
      if (p.dy) dy[v] = fetch8<E, L>(static_cast<const E*>(p.dy) + row * p.dy_stride + g.col, g, inner);
    }
  };
  float weight[AHEAD ? V : 1][8];  // a thread's columns are the same in all its rows
  if (AHEAD) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Span g = span<L>(v * TPR + lane, lead, p.cols);
      if (g.some()) weight8<L>(p.weight, g, lead, p.cols, weight[AHEAD ? v : 0]);
    }
    fetch(first + sub, dz, y, dy, rstd);
  }
  int turn = 0;
  for (int64_t row0 = first; row0 < p.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + sub;
    const bool live = row < p.rows;
    Raw8<E> next_dz[V], next_y[V], next_dy[V];
    float next_rstd = 0.f;
    if (AHEAD)
      fetch(row + step, next_dz, next_y, next_dy, next_rstd);
    else
      fetch(row, dz, y, dy, rstd);
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Span g = span<L>(v * TPR + lane, lead, p.cols);
      if (!live || !g.some()) continue;
      float u[8], n[8];
      float(&w)[8] = weight[AHEAD ? v : 0];
      unpack8<E, L>(dz[v], g, u);
      unpack8<E, L>(y[v], g, n);
      if (!AHEAD) weight8<L>(p.weight, g, lead, p.cols, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float t = u[j] * (n[j] * rstd);  // zero where there is no element
        dw[v][j] += t;
        sum += t * w[j];
      }
    }
    sum = row_sum<TPR>(sum, scratch[turn]) / (float)p.cols;
    if (live) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Span g = span<L>(v * TPR + lane, lead, p.cols);
        if (!g.some()) continue;
        float u[8], n[8], d[8];
        float(&w)[8] = weight[AHEAD ? v : 0];
        unpack8<E, L>(dz[v], g, u);
        unpack8<E, L>(y[v], g, n);
        if (!AHEAD) weight8<L>(p.weight, g, lead, p.cols, w);
        if (p.dy) {
          unpack8<E, L>(dy[v], g, d);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) d[j] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] += rstd * (u[j] * w[j] - n[j] * rstd * sum);
        if (p.dresidual) store8<E, L>(static_cast<E*>(p.dresidual) + row * p.dresidual_stride + g.col, g, d);
        if (p.dx) {
          drop8<L == kEven>(d, row * p.cols + g.col, p.drop);
          store8<E, L>(static_cast<E*>(p.dx) + row * p.dx_stride + g.col, g, d);
        }
      }
    }
    if (AHEAD) {
      rstd = next_rstd;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        dz[v] = next_dz[v];
        y[v] = next_y[v];
        dy[v] = next_dy[v];
      }
    }
  }
  float* part = p.partial + (int64_t)blockIdx.x * p.cols;
  float* to = RPC > 1 ? fold + sub * p.cols : part;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const Span g = span<L>(v * TPR + lane, lead, p.cols);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= g.lo && j < g.hi) to[g.col + j] = dw[v][j];
  }
  if constexpr (RPC > 1) {
    __syncthreads();
    for (int col = threadIdx.x; col < p.cols; col += blockDim.x) {
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < RPC; ++k) sum += fold[k * p.cols + col];
      part[col] = sum;
    }
  }
}

}  // namespace

// CTAs of the backward pass: as many as stay resident with 128 registers a thread, each with its rows
// dealt round robin.  (The most is a multiple of eight, and so are the rows from one of a thread's
// to its next.)
int norm_backward_ctas(int64_t rows, int wide, int dtype) {
  static_assert(kSMs % 8 == 0, "rows of a thread must share their lead");
  const Shape shape = shape_of(wide, dtype == GS_F32);
  const int64_t need = (rows + shape.rows - 1) / shape.rows;
  const int64_t most = (int64_t)kSMs * (shape.threads <= 512 ? 512 / shape.threads : 1);
  return (int)(need < most ? need : most);
}

// The same for any type and any alignment of the rows.
int norm_backward_most_ctas(int64_t rows, int cols) {
  int most = 0;
  for (int dtype : {GS_F32, GS_BF16})
    for (int wide : {cols, cols + 7 <= kNormMaxCols ? cols + 7 : cols}) {
      const int n = norm_backward_ctas(rows, wide, dtype);
      most = n > most ? n : most;
    }
  return most;
}

cudaError_t launch_norm_backward(const NormBackwardParams& p, float* dweight, int dtype, Layout layout, cudaStream_t s) {
  if (width(p.cols, layout) > kNormMaxCols) layout = kApart;
  const int wide = width(p.cols, layout), ctas = norm_backward_ctas(p.rows, wide, dtype);
  const Shape shape = shape_of(wide, dtype == GS_F32);
  if (ctas > 0) {
    const size_t smem = shape.rows > 1 ? (size_t)shape.rows * p.cols * sizeof(float) : 0;
    const cudaError_t err = with_type(dtype, [&](auto e) {
      using E = decltype(e);
      return with_shape<sizeof(E) == 4>(shape, [&](auto tpr, auto v) {
        return with_layout(layout, [&](auto how) {
          return launch_cluster(k_norm_backward<E, decltype(tpr)::value, decltype(v)::value, decltype(how)::value>, dim3(ctas),
                                dim3(shape.threads), smem, 1, s, p);
        });
      });
    });
    if (err != cudaSuccess) return err;
  }
  return launch_column_sums(p.partial, ctas, p.cols, nullptr, 0.f, dweight, s);
}

}  // namespace gs
