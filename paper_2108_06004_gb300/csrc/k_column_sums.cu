// Column sums of a tall matrix, the last step of parameter gradients that CTAs have summed in parts.
// Bound by latency: a few hundred rows.  32 columns a CTA; its 32 warps take every 32nd row, four
// loads at a time, and then a column each.  The order of the additions is fixed by the sizes.
#include "gs_layer.cuh"

namespace gs {
namespace {

// out[c] = sum of partial[k][c], times -scale sigmoid(decay[c]) where decay is given.
__global__ void __launch_bounds__(1024)
k_column_sums(const float* partial, int64_t n, int64_t cols, const float* decay, float scale, float* out) {
  grid_begin();
  __shared__ float part[32][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t c0 = (int64_t)blockIdx.x * 32;
  float sum = 0.f;
  if (c0 + lane < cols) {
#pragma unroll 4
    for (int64_t k = w; k < n; k += 32) sum += partial[k * cols + c0 + lane];
  }
  part[w][lane] = sum;
  __syncthreads();
  sum = part[lane][w];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  const int64_t c = c0 + w;
  if (lane == 0 && c < cols) out[c] = decay ? -scale * sum / (1.f + expf(-decay[c])) : sum;
}

}  // namespace

cudaError_t launch_column_sums(const float* partial, int64_t n, int64_t cols, const float* decay, float scale,
                               float* out, cudaStream_t s) {
  return launch(k_column_sums, dim3((unsigned)((cols + 31) / 32)), dim3(1024), s, partial, n, cols, decay, scale, out);
}

}  // namespace gs
