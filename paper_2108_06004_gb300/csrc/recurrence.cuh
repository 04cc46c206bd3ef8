// Shared pieces of the gated linear recurrence's kernels: the gates' arithmetic, the maps of runs
// of tokens, tile loads, and the exchange of maps over a cluster.
#pragma once

#include <cooperative_groups.h>

#include <atomic>

#include "gs_layer.cuh"

namespace gs {
namespace rec {

namespace cg = cooperative_groups;

constexpr int kSlots = 8;                // warps of a CTA, one run of tokens each
constexpr int kThreads = kSlots * 32;
constexpr int kPairs = 32;               // lanes: two channels each
constexpr int kChannels = 2 * kPairs;
constexpr int kStateEvery = 64;          // tokens between the states kept for the backward pass
constexpr int kMaxCluster = 16;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rsq(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The smaller of the two, NaN when x is.
__device__ __forceinline__ float at_most(float x, float most) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(most));
  return y;
}

// Two channels at a time: one instruction for both.
__device__ __forceinline__ float2 two(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 add(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 choose(bool c, float2 a, float2 b) { return make_float2(c ? a.x : b.x, c ? a.y : b.y); }

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kHuge = 1099511627776.f;  // 2^40
constexpr float kSeries = 0.25f;          // the series serves -q up to here

// softplus without overflow; for very negative arguments it is exp(x) and goes to zero.
__device__ __forceinline__ float softplus(float x) { return x > 20.f ? x : log1pf(expf(x)); }

// c softplus(lambda), kept from underflowing so that rsqrt(X) below stays finite.
__device__ __forceinline__ float2 decay_rate(float2 lam, float c) {
  return make_float2(fmaxf(c * softplus(lam.x), 1e-37f), fmaxf(c * softplus(lam.y), 1e-37f));
}

// What a token's gates give, with rate = c softplus(lambda) and q = log a = -rate sigmoid(r):
//   z = sqrt(sigmoid(r)) = p / sqrt(1 + p^2), p = e^(r/2);   sigmoid(i) = p^2 / (1 + p^2), p = e^(i/2)
//   a = 1 + q s,   s = (e^q - 1) / q,   1 - a^2 = (1 - a)(1 + a) = z^2 X,   X = rate s (1 + a)
// Halving the exponents keeps both gates exact to a few roundings down to the smallest numbers,
// and capping p at 2^40 (where they are 1) keeps them from overflowing.  1 - a is never taken as
// a difference where it is small: s is a series for q > -1/4 (five terms past the first, a
// relative error below 5e-8), and a = 1 + q s is then off by half a rounding, where the
// exponential's own bias would add up over the thousands of tokens that a state lives.
// sqrt(1 - a^2) = z X rsqrt(X), and its derivatives need z rsqrt(X) and no quotient that could
// be 0/0: X is about 2 rate even where the gate is shut.
struct Gate {
  float2 z, sr, si;  // sqrt(sigmoid(r)), sigmoid(r), sigmoid(i)
  float2 a;
  float2 rx;         // rsqrt(X)
  float2 gain;       // sqrt(1 - a^2)
};

// SERIES: rate is at most kSeries in both channels, so q always is in the series' range.
template <bool SERIES>
__device__ __forceinline__ Gate gate(float2 r, float2 i, float2 rate) {
  Gate g;
  const float2 one = two(1.f);
  const float2 hr = mul(r, two(0.5f * kLog2e)), hi = mul(i, two(0.5f * kLog2e));
  const float2 pr = make_float2(at_most(ex2(hr.x), kHuge), at_most(ex2(hr.y), kHuge));
  const float2 pi = make_float2(at_most(ex2(hi.x), kHuge), at_most(ex2(hi.y), kHuge));
  const float2 ur = fma(pr, pr, one);
  g.z = mul(pr, make_float2(rsq(ur.x), rsq(ur.y)));
  g.sr = mul(g.z, g.z);
  const float2 sq = mul(pi, pi), ui = add(sq, one);
  g.si = mul(sq, make_float2(rcp(ui.x), rcp(ui.y)));
  const float2 q = mul(make_float2(-rate.x, -rate.y), g.sr);
  float2 s = fma(q, two(1.f / 720.f), two(1.f / 120.f));
  s = fma(q, s, two(1.f / 24.f));
  s = fma(q, s, two(1.f / 6.f));
  s = fma(q, s, two(0.5f));
  s = fma(q, s, one);
  g.a = fma(q, s, one);
  if (!SERIES) {
    if (q.x < -kSeries) {
      g.a.x = ex2(kLog2e * q.x);
      s.x = (1.f - g.a.x) * rcp(-q.x);
    }
    if (q.y < -kSeries) {
      g.a.y = ex2(kLog2e * q.y);
      s.y = (1.f - g.a.y) * rcp(-q.y);
    }
  }
  const float2 X = mul(mul(rate, s), add(g.a, one));
  g.rx = make_float2(rsq(X.x), rsq(X.y));
  g.gain = mul(mul(g.z, X), g.rx);
  return g;
}

// The map h -> a h + b of a run of tokens.  `cut` beside it: the run holds a reset, so that h
// does not reach its end (not even as an infinity or NaN times zero).
struct Run {
  float2 a, b;
};

__device__ __forceinline__ float2 apply(const Run& m, bool cut, float2 h) {
  const float2 v = fma(m.a, h, m.b);
  return choose(cut, m.b, v);
}
// first, then `next`
__device__ __forceinline__ void extend(Run& m, bool& cut, const Run& next, bool next_cut) {
  m.b = apply(next, next_cut, m.b);
  m.a = mul(m.a, next.a);
  cut = cut || next_cut;
}
__device__ __forceinline__ Run identity() { return Run{two(1.f), two(0.f)}; }
__device__ __forceinline__ Run as_run(float4 v) { return Run{make_float2(v.x, v.y), make_float2(v.z, v.w)}; }
__device__ __forceinline__ float4 as_float4(const Run& m) { return make_float4(m.a.x, m.a.y, m.b.x, m.b.y); }

// Two adjacent channels of an fp32 array and of a result; n of them exist.
__device__ __forceinline__ float2 load_f32(const float* p, int n) {
  return make_float2(p && n > 0 ? p[0] : 0.f, p && n > 1 ? p[1] : 0.f);
}
__device__ __forceinline__ void store_f32(float* p, int n, float2 v) {
  if (n > 0) p[0] = v.x;
  if (n > 1) p[1] = v.y;
}
template <typename E, bool PAIR>
__device__ __forceinline__ void store2(E* p, int n, float2 v) {
  if (PAIR && n == 2) {
    *reinterpret_cast<typename Pack2<E>::type*>(p) = Pack2<E>::down(v);
  } else {
    if (n > 0) p[0] = from_f32<E>(v.x);
    if (n > 1) p[1] = from_f32<E>(v.y);
  }
}

// Where a thread works: its row of the batch, its channels, its place in the CTA and cluster.
struct Place {
  int64_t b, d0, d;      // row, first channel of the CTA, first channel of the thread
  int n;                 // the thread's channels that exist, 0 ... 2
  int pair, slot;
  int rank, cluster;
  int64_t len;           // tokens of the row
};

__device__ __forceinline__ Place place(const RecurrenceParams& p) {
  Place w;
  w.cluster = (int)cg::this_cluster().num_blocks();
  w.rank = (int)cg::this_cluster().block_rank();
  const unsigned column = blockIdx.x / (unsigned)w.cluster;
  w.b = column / (unsigned)p.groups;
  w.pair = threadIdx.x & 31;
  w.slot = threadIdx.x >> 5;
  w.d0 = (int64_t)(column - (unsigned)w.b * (unsigned)p.groups) * kChannels;
  w.d = w.d0 + 2 * w.pair;
  w.n = (int)(p.D - w.d < 0 ? 0 : p.D - w.d < 2 ? p.D - w.d : 2);
  w.len = p.T;
  if (p.lengths) {
    const int64_t l = p.lengths[w.b];
    w.len = l < 0 ? 0 : l < p.T ? l : p.T;
  }
  return w;
}

__device__ __forceinline__ int clamp_int(int64_t v, int most) { return v < 0 ? 0 : v < most ? (int)v : most; }

// Resets among the `live` tokens of a warp from t0 on, one bit each: lane k reads the flag of
// token k (ahead of time), the warp collects them.
__device__ __forceinline__ uint8_t reset_flag(const RecurrenceParams& p, const Place& w, int64_t t0, int live) {
  return w.pair < live ? p.reset[w.b * p.T + t0 + w.pair] : 0;
}

// ---- tile loads -----------------------------------------------------------------------------
// A tile is [TOKENS][kChannels] elements in shared memory: tokens t0 ... t0 + live - 1 of the
// CTA's channels, of which `channels` exist; what does not exist is zero.  UNIT is the size of one
// copy: 16 or 4 bytes asynchronously, or single 2-byte elements through registers, where rows of a
// 2-byte type start at odd elements.
template <int UNIT>
__device__ __forceinline__ void copy_async(void* to, const void* from, int bytes) {
  const uint32_t dst = (uint32_t)__cvta_generic_to_shared(to);
  if (UNIT == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(from), "r"(bytes) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

template <typename E, int UNIT, int TOKENS>
__device__ __forceinline__ void load_tile(E* tile, const E* from, int64_t token_stride, int64_t t0, int live,
                                          int channels) {
  constexpr int PER = UNIT / (int)sizeof(E);      // elements of a copy
  constexpr int U = kChannels / PER;              // copies of a token
  constexpr int R = kThreads / U;                 // tokens at a time
  const int u = threadIdx.x % U, row = threadIdx.x / U;
  const E* src = from + t0 * token_stride + (int64_t)row * token_stride + u * PER;
  E* dst = tile + row * kChannels + u * PER;
  const int have = clamp_int(channels - u * PER, PER);
  if constexpr (UNIT == 2) {
    constexpr int BATCH = 8;
#pragma unroll
    for (int j0 = 0; j0 < TOKENS / R; j0 += BATCH) {
      E v[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
        v[j] = have > 0 && row + (j0 + j) * R < live ? src[(int64_t)(j0 + j) * R * token_stride] : from_f32<E>(0.f);
#pragma unroll
      for (int j = 0; j < BATCH; ++j) dst[(j0 + j) * R * kChannels] = v[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < TOKENS / R; ++j) {
      const bool some = have > 0 && row + j * R < live;
      copy_async<UNIT>(dst + j * R * kChannels, some ? src : from, some ? have * (int)sizeof(E) : 0);
      src += R * token_stride;
    }
  }
}

// ---- exchange over the cluster ----------------------------------------------------------------
// The chunks' maps.  `mine` of this CTA goes into every CTA's table at this rank; warp k writes to
// the CTAs k, k + kSlots, ...  The two halves of the table alternate, so one barrier a step is
// enough: a CTA writes step s + 2 only after all have passed the barrier of s + 1, and so have
// read step s.
struct Totals {
  float4 run[2][kMaxCluster][kPairs];
  uint32_t cut[2][kMaxCluster];
};

__device__ __forceinline__ void exchange(Totals& t, int half, const Place& w, const Run& mine, bool cut) {
  cg::cluster_group cl = cg::this_cluster();
  for (int k = w.slot; k < w.cluster; k += kSlots) {
    Totals* to = cl.map_shared_rank(&t, k);
    to->run[half][w.rank][w.pair] = as_float4(mine);
    if (w.pair == 0) to->cut[half][w.rank] = cut;
  }
  cl.sync();
}

// Shared memory beyond the default and clusters beyond the portable size are asked for once per
// kernel and device.
template <typename K>
cudaError_t prepare_kernel(K kernel, size_t smem, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

}  // namespace rec
}  // namespace gs
