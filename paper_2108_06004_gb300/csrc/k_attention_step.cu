// One token of linear attention with a decay for each head: the state in place, and what is read from it.
//
//   S <- e^g S + k v',  o = scale S' q
//
// Bound by memory: the state is read and written once.  A CTA takes 32 columns of one head's state, 16 rows of
// eight 16-byte words (or 4 rows of single elements) at a time, all loads of a thread ahead of their use; the rows'
// shares of o are summed over the warp and then over the CTA, in a fixed order.  200x16x128 bf16 takes 61 us (91 % of the
// copy rate); 1x16x64 5.5 us on the device, and 10 to 12 us with the call from Python, by the host.
#include "attention.cuh"

namespace gs {
namespace {

constexpr int kStepThreads = 128, kStepCols = 32;

template <typename E>
__device__ __forceinline__ float at(const HeadsIn& t, int64_t b, int head, int d) {
  return to_f32(static_cast<const E*>(t.data)[b * t.batch + head / t.share * t.head + d]);
}

// W: elements of a load.
template <typename E, int W>
__global__ void __launch_bounds__(kStepThreads)
k_attention_step(const __grid_constant__ AttentionStepParams p) {
  grid_begin();
  constexpr int LANES = kStepCols / W, GROUPS = kStepThreads / LANES, AHEAD = 8;
  __shared__ float q[kAttentionMaxHead], k[kAttentionMaxHead], part[4][kStepCols];
  const int slices = (p.Dv + kStepCols - 1) / kStepCols;
  const int slice = blockIdx.x % slices, head = blockIdx.x / slices % p.H;
  const int64_t b = blockIdx.x / slices / p.H;
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, col = slice * kStepCols + lane * W;
  const int64_t slot = p.slots ? p.slots[b] : b;
  E* o = static_cast<E*>(p.o.data) + b * p.o.batch + head * p.o.head;
  if (slot < 0 || slot >= p.n_slots) {
    for (int d = slice * kStepCols + threadIdx.x; d < min(p.Dv, (slice + 1) * kStepCols); d += kStepThreads) o[d] = from_f32<E>(0.f);
    return;
  }
  const bool mine = col < p.Dv;
  float* state = p.state + slot * p.state_stride + (int64_t)head * p.Dk * p.Dv + col;
  float sum[W], v[W];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    sum[j] = 0.f;
    v[j] = mine ? at<E>(p.v, b, head, col + j) : 0.f;
  }
  float S[AHEAD][W];
  const auto load = [&](int r0) {
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int r = r0 + a * GROUPS;
      if (!mine || r >= p.Dk) continue;
      if constexpr (W == 4)
        *reinterpret_cast<float4*>(S[a]) = *reinterpret_cast<const float4*>(state + (int64_t)r * p.Dv);
      else
        S[a][0] = state[(int64_t)r * p.Dv];
    }
  };
  load(group);
  for (int d = threadIdx.x; d < p.Dk; d += kStepThreads) {
    q[d] = at<E>(p.q, b, head, d);
    k[d] = at<E>(p.k, b, head, d);
  }
  __syncthreads();
  const Decay d = decay_of(taken(p.log_decay[head]));
  for (int r0 = group; r0 < p.Dk; r0 += AHEAD * GROUPS) {
    if (r0 != group) load(r0);
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int r = r0 + a * GROUPS;
      if (!mine || r >= p.Dk) continue;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        S[a][j] = decayed(S[a][j], d, k[r] * v[j]);
        sum[j] = fmaf(q[r], S[a][j], sum[j]);
      }
      if constexpr (W == 4)
        *reinterpret_cast<float4*>(state + (int64_t)r * p.Dv) = *reinterpret_cast<const float4*>(S[a]);
      else
        state[(int64_t)r * p.Dv] = S[a][0];
    }
  }
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int x = LANES; x < 32; x *= 2) sum[j] += __shfl_xor_sync(0xFFFFFFFFu, sum[j], x);
  if ((threadIdx.x & 31) < LANES) {
#pragma unroll
    for (int j = 0; j < W; ++j) part[threadIdx.x >> 5][lane * W + j] = sum[j];
  }
  __syncthreads();
  const int c = slice * kStepCols + threadIdx.x;
  if (threadIdx.x < kStepCols && c < p.Dv)
    o[c] = from_f32<E>(p.scale * ((part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x])));
}

}  // namespace

cudaError_t launch_attention_step(const AttentionStepParams& p, int dtype, bool vec, cudaStream_t s) {
  const dim3 grid((unsigned)(p.B * p.H * ((p.Dv + kStepCols - 1) / kStepCols)));
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return vec ? launch(k_attention_step<E, 4>, grid, dim3(kStepThreads), s, p) : launch(k_attention_step<E, 1>, grid, dim3(kStepThreads), s, p);
  });
}

}  // namespace gs
