// Dropout, residual add and RMS norm in one pass over a row, and the backward pass.
//
//   y = residual + dropout(x),  rstd = (mean(y^2) + eps)^(-1/2),  z = y rstd w
//   backward, from dz, dy (the gradient that reaches y past the norm) and the stored y:
//     n = y rstd,  u = dz w,  dt = rstd (u - n mean(u n)) + dy
//     dresidual = dt,  dx = mask dt scale,  dw = sum over rows of dz n
//
// A row is held in the registers of TPR threads, V groups of eight elements each, so every tensor
// is read and written once.  dw is summed by each thread over the rows of its CTA, then over the
// CTAs by a second kernel, in a fixed order.
#include "gs_layer.cuh"

namespace gs {
namespace {

// Sum over the TPR threads of a row; every thread of the CTA takes part.  Two sums in turn use two
// scratch arrays, so one barrier each is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  if (TPR > 32) {
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
    unpack8(fetch8<float, kEven>(weight + g.col, g), w);
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
    unpack8(fetch8<float, kApart>(weight + g.col, g), w);
  }
}

template <int TPR> constexpr int kCtaThreads = TPR > 256 ? TPR : 256;

template <typename E, int TPR, int V, int L>
__global__ void __launch_bounds__(kCtaThreads<TPR>)
k_norm_forward(const __grid_constant__ NormForwardParams p) {
  grid_begin();
  __shared__ float scratch[32];
  constexpr int RPC = kCtaThreads<TPR> / TPR;
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
    unpack8(fetch8<E, L>(static_cast<const E*>(p.x) + row * p.x_stride + g.col, g), t[v]);
    unpack8(fetch8<E, L>(static_cast<const E*>(p.residual) + row * p.residual_stride + g.col, g), res);
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

template <typename E, int TPR, int V, int L>
__global__ void __launch_bounds__(kCtaThreads<TPR>, kCtaThreads<TPR> == 256 ? 2 : 1)
k_norm_backward(const __grid_constant__ NormBackwardParams p) {
  grid_begin();
  __shared__ float scratch[2][32];
  constexpr int RPC = kCtaThreads<TPR> / TPR;
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
  // widest rows, whose 1024 threads have registers for one row only.
  constexpr bool AHEAD = TPR < 1024;
  Raw8<E> dz[V], y[V], dy[V];
  float rstd = 0.f;
  auto fetch = [&](int64_t row, Raw8<E>(&dz)[V], Raw8<E>(&y)[V], Raw8<E>(&dy)[V], float& rstd) {
    if (row >= p.rows) return;
    rstd = p.rstd[row];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Span g = span<L>(v * TPR + lane, lead, p.cols);
      if (!g.some()) continue;
      dz[v] = fetch8<E, L>(static_cast<const E*>(p.dz) + row * p.dz_stride + g.col, g);
      y[v] = fetch8<E, L>(static_cast<const E*>(p.y) + row * p.y_stride + g.col, g);
      if (p.dy) dy[v] = fetch8<E, L>(static_cast<const E*>(p.dy) + row * p.dy_stride + g.col, g);
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
      unpack8(dz[v], u);
      unpack8(y[v], n);
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
        unpack8(dz[v], u);
        unpack8(y[v], n);
        if (!AHEAD) weight8<L>(p.weight, g, lead, p.cols, w);
        if (p.dy) {
          unpack8(dy[v], d);
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

// Threads a row and groups of eight a thread: a row of up to 512 elements is one warp's, wider
// ones have two groups a thread.
template <typename F>
cudaError_t with_shape(int cols, F&& f) {  // cols: with the elements that leads may add
  using std::integral_constant;
  if (cols <= 256) return f(integral_constant<int, 32>(), integral_constant<int, 1>());
  if (cols <= 512) return f(integral_constant<int, 32>(), integral_constant<int, 2>());
  if (cols <= 1024) return f(integral_constant<int, 64>(), integral_constant<int, 2>());
  if (cols <= 2048) return f(integral_constant<int, 128>(), integral_constant<int, 2>());
  if (cols <= 4096) return f(integral_constant<int, 256>(), integral_constant<int, 2>());
  if (cols <= 8192) return f(integral_constant<int, 512>(), integral_constant<int, 2>());
  return f(integral_constant<int, 1024>(), integral_constant<int, 2>());
}

int rows_per_cta(int cols) {
  int tpr = 32;
  while (tpr * 16 < cols) tpr *= 2;
  return tpr >= 256 ? 1 : 256 / tpr;
}

// Elements that a row takes: its first group may start up to seven before it.
int width(int cols, Layout layout) { return layout == kTogether ? cols + 7 : cols; }

}  // namespace

// CTAs of the backward pass: as many as stay resident, each with its rows dealt round robin.  (Both
// numbers are multiples of eight, and so are the rows from one of a thread's to its next.)
int norm_backward_ctas(int64_t rows, int cols) {
  static_assert(kSMs % 8 == 0, "rows of a thread must share their lead");
  const int64_t rpc = rows_per_cta(cols);
  const int64_t need = (rows + rpc - 1) / rpc;
  const int64_t most = cols <= 4096 ? 2 * kSMs : kSMs;
  return (int)(need < most ? need : most);
}

cudaError_t launch_norm_forward(const NormForwardParams& p, int dtype, Layout layout, cudaStream_t s) {
  if (width(p.cols, layout) > kNormMaxCols) layout = kApart;  // the row with its lead does not fit
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return with_shape(width(p.cols, layout), [&](auto tpr, auto v) {
      constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value;
      constexpr int N = kCtaThreads<TPR>;
      const int64_t ctas = (p.rows + N / TPR - 1) / (N / TPR);
      return with_layout(layout, [&](auto how) {
        return launch(k_norm_forward<E, TPR, V, decltype(how)::value>, dim3((unsigned)ctas), dim3(N), s, p);
      });
    });
  });
}

cudaError_t launch_norm_backward(const NormBackwardParams& p, float* dweight, int dtype, Layout layout, cudaStream_t s) {
  if (width(p.cols, layout) > kNormMaxCols) layout = kApart;
  const int wide = width(p.cols, layout), ctas = norm_backward_ctas(p.rows, wide);
  if (ctas > 0) {
    cudaError_t err = with_type(dtype, [&](auto e) {
      using E = decltype(e);
      return with_shape(wide, [&](auto tpr, auto v) {
        constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value;
        constexpr int N = kCtaThreads<TPR>;
        const size_t smem = N > TPR ? (size_t)(N / TPR) * p.cols * sizeof(float) : 0;
        return with_layout(layout, [&](auto how) {
          return launch_cluster(k_norm_backward<E, TPR, V, decltype(how)::value>, dim3(ctas), dim3(N), smem, 1, s, p);
        });
      });
    });
    if (err != cudaSuccess) return err;
  }
  return launch_column_sums(p.partial, ctas, p.cols, nullptr, 0.f, dweight, s);
}

}  // namespace gs
