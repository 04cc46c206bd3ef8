// Dropout, residual add and RMS norm in one pass over a row, and the backward pass.
//
//   y = residual + dropout(x),  rstd = (mean(y^2) + eps)^(-1/2),  z = y rstd w
//   backward, from dz, dy (the gradient that reaches y past the norm) and the stored y:
//     n = y rstd,  u = dz w,  dt = rstd (u - n mean(u n)) + dy
//     dresidual = dt,  dx = mask dt scale,  dw = sum over rows of dz n
//
// A row is held in the registers of TPR threads, 8 * V adjacent-by-8 elements each, so every
// tensor is read and written once.  dw is summed by each thread over the rows of its CTA, then
// over the CTAs by a second kernel, in a fixed order.
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

template <int TPR> constexpr int kCtaThreads = TPR > 256 ? TPR : 256;

template <typename E, int TPR, int V, bool VEC>
__global__ void __launch_bounds__(kCtaThreads<TPR>)
k_norm_forward(const __grid_constant__ NormForwardParams p) {
  grid_begin();
  __shared__ float scratch[32];
  constexpr int RPC = kCtaThreads<TPR> / TPR;
  const int lane = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * RPC + threadIdx.x / TPR;
  const bool live = row < p.rows;
  float t[V][8];
  float sum = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int col = (v * TPR + lane) * 8;
    if (!live || col >= p.cols) continue;
    const int n = p.cols - col;
    float res[8];
    load8<E, VEC>(static_cast<const E*>(p.x) + row * p.x_stride + col, n, t[v]);
    load8<E, VEC>(static_cast<const E*>(p.residual) + row * p.residual_stride + col, n, res);
    drop8<VEC>(t[v], (uint64_t)row * (uint64_t)p.cols + col, p.drop);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      t[v][j] += res[j];
      if (VEC || j < n) sum += t[v][j] * t[v][j];
    }
    store8<E, VEC>(static_cast<E*>(p.y) + row * p.y_stride + col, n, t[v]);
  }
  sum = row_sum<TPR>(sum, scratch);
  const float rstd = rsqrtf(sum / (float)p.cols + p.eps);
  if (!live) return;
  if (lane == 0) p.rstd[row] = rstd;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int col = (v * TPR + lane) * 8;
    if (col >= p.cols) continue;
    const int n = p.cols - col;
    float w[8];
    load8<float, VEC>(p.weight + col, n, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] *= t[v][j] * rstd;
    store8<E, VEC>(static_cast<E*>(p.z) + row * p.z_stride + col, n, w);
  }
}

template <typename E, int TPR, int V, bool VEC>
__global__ void __launch_bounds__(kCtaThreads<TPR>, kCtaThreads<TPR> == 256 ? 2 : 1)
k_norm_backward(const __grid_constant__ NormBackwardParams p) {
  grid_begin();
  __shared__ float scratch[2][32];
  constexpr int RPC = kCtaThreads<TPR> / TPR;
  extern __shared__ float fold[];  // RPC > 1: [RPC][cols]
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const int64_t step = (int64_t)gridDim.x * RPC;
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
      const int col = (v * TPR + lane) * 8;
      if (col >= p.cols) continue;
      const int m = p.cols - col;
      dz[v] = fetch8<E, VEC>(static_cast<const E*>(p.dz) + row * p.dz_stride + col, m);
      y[v] = fetch8<E, VEC>(static_cast<const E*>(p.y) + row * p.y_stride + col, m);
      if (p.dy) dy[v] = fetch8<E, VEC>(static_cast<const E*>(p.dy) + row * p.dy_stride + col, m);
    }
  };
  const int64_t first = (int64_t)blockIdx.x * RPC;
  if (AHEAD) fetch(first + sub, dz, y, dy, rstd);
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
      const int col = (v * TPR + lane) * 8;
      if (!live || col >= p.cols) continue;
      const int m = p.cols - col;
      float u[8], n[8], w[8];
      unpack8(dz[v], u);
      unpack8(y[v], n);
      load8<float, VEC>(p.weight + col, m, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float t = u[j] * (n[j] * rstd);
        if (VEC || j < m) {
          dw[v][j] += t;
          sum += t * w[j];
        }
      }
    }
    sum = row_sum<TPR>(sum, scratch[turn]) / (float)p.cols;
    if (live) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int col = (v * TPR + lane) * 8;
        if (col >= p.cols) continue;
        const int m = p.cols - col;
        float u[8], n[8], d[8], w[8];
        unpack8(dz[v], u);
        unpack8(y[v], n);
        load8<float, VEC>(p.weight + col, m, w);
        if (p.dy) {
          unpack8(dy[v], d);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) d[j] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] += rstd * (u[j] * w[j] - n[j] * rstd * sum);
        if (p.dresidual) store8<E, VEC>(static_cast<E*>(p.dresidual) + row * p.dresidual_stride + col, m, d);
        if (p.dx) {
          drop8<VEC>(d, (uint64_t)row * (uint64_t)p.cols + col, p.drop);
          store8<E, VEC>(static_cast<E*>(p.dx) + row * p.dx_stride + col, m, d);
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
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int col = (v * TPR + lane) * 8 + j;
      if (col < p.cols) to[col] = dw[v][j];
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

// dweight[col] = sum over the CTAs' partial rows, 32 columns a CTA, the rows dealt to 8 warps.
__global__ void __launch_bounds__(256) k_norm_weight(const float* partial, int n, int cols, float* dweight) {
  grid_begin();
  __shared__ float part[8][32];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
  float sum = 0.f;
  if (col < cols)
    for (int k = w; k < n; k += 8) sum += partial[(int64_t)k * cols + col];
  part[w][threadIdx.x & 31] = sum;
  __syncthreads();
  if (w == 0 && col < cols) {
#pragma unroll
    for (int k = 1; k < 8; ++k) sum += part[k][threadIdx.x];
    dweight[col] = sum;
  }
}

// Threads a row and groups of eight a thread: a row of up to 512 elements is one warp's, wider
// ones have two groups a thread.
template <typename F>
cudaError_t with_shape(int cols, F&& f) {
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

}  // namespace

// CTAs of the backward pass: as many as stay resident, each with its rows dealt round robin.
int norm_backward_ctas(int64_t rows, int cols) {
  const int64_t rpc = rows_per_cta(cols);
  const int64_t need = (rows + rpc - 1) / rpc;
  const int64_t most = cols <= 4096 ? 2 * kSMs : kSMs;
  return (int)(need < most ? need : most);
}

cudaError_t launch_norm_forward(const NormForwardParams& p, int dtype, bool vec, cudaStream_t s) {
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return with_shape(p.cols, [&](auto tpr, auto v) {
      constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value;
      constexpr int N = kCtaThreads<TPR>;
      const int64_t ctas = (p.rows + N / TPR - 1) / (N / TPR);
      return vec ? launch(k_norm_forward<E, TPR, V, true>, dim3((unsigned)ctas), dim3(N), s, p)
                 : launch(k_norm_forward<E, TPR, V, false>, dim3((unsigned)ctas), dim3(N), s, p);
    });
  });
}

cudaError_t launch_norm_backward(const NormBackwardParams& p, float* dweight, int dtype, bool vec, cudaStream_t s) {
  const int ctas = norm_backward_ctas(p.rows, p.cols);
  if (ctas > 0) {
    cudaError_t err = with_type(dtype, [&](auto e) {
      using E = decltype(e);
      return with_shape(p.cols, [&](auto tpr, auto v) {
        constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value;
        constexpr int N = kCtaThreads<TPR>;
        const size_t smem = N > TPR ? (size_t)(N / TPR) * p.cols * sizeof(float) : 0;
        return vec ? launch_cluster(k_norm_backward<E, TPR, V, true>, dim3(ctas), dim3(N), smem, 1, s, p)
                   : launch_cluster(k_norm_backward<E, TPR, V, false>, dim3(ctas), dim3(N), smem, 1, s, p);
      });
    });
    if (err != cudaSuccess) return err;
  }
  return launch(k_norm_weight, dim3((p.cols + 31) / 32), dim3(256), s, (const float*)p.partial, ctas, p.cols, dweight);
}

}  // namespace gs
