// Gated linear recurrence over time, forward and backward, and its single-token step.
//
//   log a_t = -c softplus(lambda) sigmoid(r_t),   v_t = 1 - a_t^2,
//   h_t = a_t h_{t-1} + sqrt(v_t) sigmoid(i_t) x_t,   y_t = h_t      (at a reset a_t = 0)
//
// A run of tokens acts on the state as h -> A h + B with A the product of its a_t, and such maps
// compose, so time is cut three times: a thread owns kLen tokens of two channels, the kSlots
// warps of a CTA own adjacent runs (a chunk), and where the rows and channels alone do not fill
// the device a cluster of CTAs owns adjacent chunks.  Each thread first works out (A, B) of its
// run, the warps exchange them in shared memory and the CTAs in distributed shared memory behind
// the hardware's cluster barrier, and then the run is walked again from its true starting state.
// Every tensor is read from and written to memory once, and the order of all operations is fixed.
//
// The backward pass walks time from the end: g_t = dy_t + a_{t+1} g_{t+1} is the same kind of map.
// It needs h_{t-1} in full precision; it recomputes it from the state at the start of each chunk,
// which the forward pass leaves in fp32 (4 bytes for kChunk tokens) rather than from y.
#include <cooperative_groups.h>

#include "gs_layer.cuh"

namespace gs {
namespace {

namespace cg = cooperative_groups;

constexpr int kSlots = 8;                // warps of a CTA, one run of tokens each
constexpr int kLen = 16;                 // tokens of a run
constexpr int kChunk = kSlots * kLen;    // tokens of a CTA
constexpr int kPairs = 32;               // lanes: two channels each
constexpr int kChannels = 2 * kPairs;
constexpr int kMaxCluster = 8;
constexpr int kThreads = kSlots * 32;

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

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kHuge = 1099511627776.f;  // 2^40

// softplus without overflow; for very negative arguments it is exp(x) and goes to zero.
__device__ __forceinline__ float softplus(float x) { return x > 20.f ? x : log1pf(expf(x)); }

// What a token's gates give, with rate = c softplus(lambda) and q = log a = -rate sigmoid(r):
//   z = sqrt(sigmoid(r)) = p / sqrt(1 + p^2), p = e^(r/2);   sigmoid(i) = p^2 / (1 + p^2), p = e^(i/2)
//   w = 1 - a = -q s,   s = (1 - e^q) / -q,   1 - a^2 = w (2 - w) = z^2 X,   X = rate s (2 - w)
// Halving the exponents keeps both gates exact to a few roundings down to the smallest numbers,
// and capping p at 2^40 (where they are 1) keeps them from overflowing.  1 - a is never taken as
// a difference where it is small: s is the series of (e^q - 1) / q for q > -1/4 (five terms past
// the first, a relative error below 5e-8), and a = 1 - w is then off by half a rounding, where
// the exponential's own bias would add up over the thousands of tokens that a state lives.
// sqrt(1 - a^2) = z X rsqrt(X), and its derivatives need z rsqrt(X) and no quotient that could
// be 0/0: X is about 2 rate even where the gate is shut.
struct Gate {
  float z, sr, si;  // sqrt(sigmoid(r)), sigmoid(r), sigmoid(i)
  float a;
  float rx;         // rsqrt(X)
  float gain;       // sqrt(1 - a^2)
};

__device__ __forceinline__ Gate gate(float r, float i, float rate) {
  Gate g;
  const float pr = at_most(ex2(0.5f * kLog2e * r), kHuge), pi = at_most(ex2(0.5f * kLog2e * i), kHuge);
  g.z = pr * rsq(fmaf(pr, pr, 1.f));
  g.sr = g.z * g.z;
  g.si = pi * pi * rcp(fmaf(pi, pi, 1.f));
  const float q = -rate * g.sr;
  float s = fmaf(q, 1.f / 720.f, 1.f / 120.f);
  s = fmaf(q, s, 1.f / 24.f);
  s = fmaf(q, s, 1.f / 6.f);
  s = fmaf(q, s, 0.5f);
  s = fmaf(q, s, 1.f);
  float w = -q * s;
  if (q < -0.25f) {
    w = 1.f - ex2(kLog2e * q);
    s = w * rcp(-q);
  }
  g.a = 1.f - w;
  const float X = rate * s * (2.f - w);
  g.rx = rsq(fmaxf(X, 1e-36f));
  g.gain = g.z * X * g.rx;
  return g;
}

// The map h -> a h + b of a run; `cut`: it holds a reset, so that h does not reach its end (not
// even as an infinity or NaN times zero).
struct Run {
  float2 a, b;
};

__device__ __forceinline__ float2 apply(const Run& m, bool cut, float2 h) {
  return cut ? m.b : make_float2(fmaf(m.a.x, h.x, m.b.x), fmaf(m.a.y, h.y, m.b.y));
}

// Two adjacent channels of one token, zero where they do not exist.
template <typename E, bool VEC>
__device__ __forceinline__ float2 load2(const E* p, int n) {
  if (VEC) return n > 0 ? Pack2<E>::up(*reinterpret_cast<const typename Pack2<E>::type*>(p)) : make_float2(0.f, 0.f);
  return make_float2(n > 0 ? to_f32(p[0]) : 0.f, n > 1 ? to_f32(p[1]) : 0.f);
}
template <typename E, bool VEC>
__device__ __forceinline__ void store2(E* p, int n, float2 v) {
  if (VEC) {
    if (n > 0) *reinterpret_cast<typename Pack2<E>::type*>(p) = Pack2<E>::down(v);
  } else {
    if (n > 0) p[0] = from_f32<E>(v.x);
    if (n > 1) p[1] = from_f32<E>(v.y);
  }
}
__device__ __forceinline__ float2 load_f32(const float* p, int n) {
  return make_float2(p && n > 0 ? p[0] : 0.f, p && n > 1 ? p[1] : 0.f);
}
__device__ __forceinline__ void store_f32(float* p, int n, float2 v) {
  if (n > 0) p[0] = v.x;
  if (n > 1) p[1] = v.y;
}

// Where a thread works: its channels, its row of the batch, its place in the CTA and cluster.
struct Place {
  int64_t b, d;
  int n;                 // channels that exist, 0 ... 2
  int pair, slot;
  int rank, cluster;
  int64_t len;           // tokens of the row
};

__device__ __forceinline__ Place place(const RecurrenceParams& p) {
  Place w;
  w.cluster = (int)cg::this_cluster().num_blocks();
  w.rank = (int)cg::this_cluster().block_rank();
  const int64_t column = blockIdx.x / w.cluster;
  w.b = column / p.groups;
  w.pair = threadIdx.x & 31;
  w.slot = threadIdx.x >> 5;
  w.d = (column - w.b * p.groups) * kChannels + 2 * w.pair;
  w.n = (int)(p.D - w.d < 0 ? 0 : p.D - w.d < 2 ? p.D - w.d : 2);
  w.len = p.T;
  if (p.lengths) {
    const int64_t l = p.lengths[w.b];
    w.len = l < 0 ? 0 : l < p.T ? l : p.T;
  }
  return w;
}

template <typename E>
__device__ __forceinline__ const E* at(const Seq<const void*>& t, const Place& w) {
  return static_cast<const E*>(t.data) + w.b * t.batch + w.d;
}
template <typename E>
__device__ __forceinline__ E* at(const Seq<void*>& t, const Place& w) {
  return static_cast<E*>(t.data) + w.b * t.batch + w.d;
}

__device__ __forceinline__ float2 rates(const RecurrenceParams& p, const Place& w) {
  const float2 lam = load_f32(p.decay + w.d, w.n);
  return make_float2(p.c * softplus(lam.x), p.c * softplus(lam.y));
}

// Resets among the tokens t0 ... t0 + n - 1 of a row, one bit each.
__device__ __forceinline__ uint32_t reset_bits(const RecurrenceParams& p, const Place& w, int64_t t0, int n) {
  uint32_t bits = 0;
  if (p.reset) {
    const uint8_t* f = p.reset + w.b * p.T + t0;
#pragma unroll
    for (int k = 0; k < kLen; ++k)
      if (k < n && f[k]) bits |= 1u << k;
  }
  return bits;
}

struct Shared {
  float4 run[kSlots][kPairs];                 // (a, b) of each warp's run
  uint32_t cut[kSlots];
  float4 total[2][kMaxCluster][kPairs];       // (a, b) of each CTA's chunk, two steps' worth
  uint32_t total_cut[2][kMaxCluster];
};

__device__ __forceinline__ Run as_run(float4 v) { return Run{make_float2(v.x, v.y), make_float2(v.z, v.w)}; }

// Exchange the chunks' maps: `mine` of this CTA goes into every CTA's table at this rank.  Warp k
// writes to CTA k.  The two halves of the table alternate, so one barrier a step is enough: a CTA
// writes step s + 2 only after all have passed the barrier of s + 1, and so have read step s.
__device__ __forceinline__ void exchange(Shared& sh, int half, const Place& w, const Run& mine, bool cut) {
  cg::cluster_group cl = cg::this_cluster();
  if (w.slot < w.cluster) {
    Shared* to = cl.map_shared_rank(&sh, w.slot);
    to->total[half][w.rank][w.pair] = make_float4(mine.a.x, mine.a.y, mine.b.x, mine.b.y);
    if (w.pair == 0) to->total_cut[half][w.rank] = cut;
  }
  cl.sync();
}

template <typename E, bool VEC>
__global__ void __launch_bounds__(kThreads) k_recurrence_forward(const __grid_constant__ RecurrenceParams p) {
  grid_begin();
  __shared__ Shared sh;
  const Place w = place(p);
  if (w.cluster > 1) cg::this_cluster().sync();  // every CTA of the cluster runs before its memory is written
  const float2 rate = rates(p, w);
  const E *x = at<E>(p.x, w), *r = at<E>(p.r, w), *i = at<E>(p.i, w);
  E* y = at<E>(p.y, w);
  const int64_t chunks = (p.T + kChunk - 1) / kChunk;
  float2 state = load_f32(p.h0 ? p.h0 + w.b * p.D + w.d : nullptr, w.n);
  const int64_t steps = ((w.len + kChunk - 1) / kChunk + w.cluster - 1) / w.cluster;
  for (int64_t s = 0; s < steps; ++s) {
    const int64_t chunk = s * w.cluster + w.rank;
    const int64_t t0 = chunk * kChunk + w.slot * kLen;
    const int live = (int)(w.len - t0 < 0 ? 0 : w.len - t0 < kLen ? w.len - t0 : kLen);
    const uint32_t resets = reset_bits(p, w, t0, live);
    float2 a[kLen], b[kLen];
    Run run{make_float2(1.f, 1.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int k = 0; k < kLen; ++k) {
      a[k] = make_float2(1.f, 1.f);
      b[k] = make_float2(0.f, 0.f);
      if (k < live) {
        const float2 xv = load2<E, VEC>(x + (t0 + k) * p.x.token, w.n);
        const float2 rv = load2<E, VEC>(r + (t0 + k) * p.r.token, w.n);
        const float2 iv = load2<E, VEC>(i + (t0 + k) * p.i.token, w.n);
        const Gate g0 = gate(rv.x, iv.x, rate.x), g1 = gate(rv.y, iv.y, rate.y);
        const bool cut = resets >> k & 1u;
        a[k] = cut ? make_float2(0.f, 0.f) : make_float2(g0.a, g1.a);
        b[k] = make_float2((cut ? 1.f : g0.gain) * g0.si * xv.x, (cut ? 1.f : g1.gain) * g1.si * xv.y);
        run.a = make_float2(run.a.x * a[k].x, run.a.y * a[k].y);
        run.b = apply(Run{a[k], b[k]}, cut, run.b);
      }
    }
    __syncthreads();  // the table of the step before has been read
    sh.run[w.slot][w.pair] = make_float4(run.a.x, run.a.y, run.b.x, run.b.y);
    if (w.pair == 0) sh.cut[w.slot] = resets;
    __syncthreads();
    float2 h;  // at the start of the chunk, then of the run
    if (w.cluster > 1) {
      Run total = as_run(sh.run[0][w.pair]);
      bool cut = sh.cut[0];
#pragma unroll
      for (int k = 1; k < kSlots; ++k) {
        const Run next = as_run(sh.run[k][w.pair]);
        total.b = apply(next, sh.cut[k], total.b);
        total.a = make_float2(total.a.x * next.a.x, total.a.y * next.a.y);
        cut = cut || sh.cut[k];
      }
      exchange(sh, (int)(s & 1), w, total, cut);
      h = state;
      for (int k = 0; k < w.cluster; ++k) {
        if (k == w.rank) h = state;
        state = apply(as_run(sh.total[s & 1][k][w.pair]), sh.total_cut[s & 1][k], state);
      }
    } else {
      h = state;
#pragma unroll
      for (int k = 0; k < kSlots; ++k) state = apply(as_run(sh.run[k][w.pair]), sh.cut[k], state);
    }
    if (p.states && w.slot == 0 && chunk < chunks) store_f32(p.states + (w.b * chunks + chunk) * p.D + w.d, w.n, h);
    for (int k = 0; k < w.slot; ++k) h = apply(as_run(sh.run[k][w.pair]), sh.cut[k], h);
#pragma unroll
    for (int k = 0; k < kLen; ++k) {
      if (k < live) {
        h = apply(Run{a[k], b[k]}, resets >> k & 1u, h);
        store2<E, VEC>(y + (t0 + k) * p.y.token, w.n, h);
      } else if (t0 + k < p.T) {
        store2<E, VEC>(y + (t0 + k) * p.y.token, w.n, make_float2(0.f, 0.f));
      }
    }
  }
  // past the last step every token is masked
  for (int64_t chunk = steps * w.cluster + w.rank; chunk < chunks; chunk += w.cluster)
    for (int k = 0; k < kLen; ++k) {
      const int64_t t = chunk * kChunk + w.slot * kLen + k;
      if (t < p.T) store2<E, VEC>(y + t * p.y.token, w.n, make_float2(0.f, 0.f));
    }
  if (p.h_last && w.rank == 0 && w.slot == 0) store_f32(p.h_last + w.b * p.D + w.d, w.n, state);
}

template <typename E, bool VEC>
__global__ void __launch_bounds__(kThreads) k_recurrence_backward(const __grid_constant__ RecurrenceParams p) {
  grid_begin();
  __shared__ Shared sh;                    // the maps of h, and of g over a CTA's chunk
  __shared__ float4 back[kSlots][kPairs];  // the maps of g over a warp's run
  const Place w = place(p);
  if (w.cluster > 1) cg::this_cluster().sync();  // every CTA of the cluster runs before its memory is written
  const float2 rate = rates(p, w);
  const E *x = at<E>(p.x, w), *r = at<E>(p.r, w), *i = at<E>(p.i, w), *dy = at<E>(p.dy, w);
  E *dx = at<E>(p.dx, w), *dr = at<E>(p.dr, w), *di = at<E>(p.di, w);
  const int64_t chunks = (p.T + kChunk - 1) / kChunk;
  float2 flow = load_f32(p.dh_last ? p.dh_last + w.b * p.D + w.d : nullptr, w.n);  // a_{t+1} g_{t+1}
  float2 sum = make_float2(0.f, 0.f);    // of dlog a * sigmoid(r)
  const int64_t steps = ((w.len + kChunk - 1) / kChunk + w.cluster - 1) / w.cluster;
  const float2 zero = make_float2(0.f, 0.f);
  for (int64_t s = steps - 1; s >= 0; --s) {
    const int64_t chunk = s * w.cluster + w.rank;
    const int64_t t0 = chunk * kChunk + w.slot * kLen;
    const int live = (int)(w.len - t0 < 0 ? 0 : w.len - t0 < kLen ? w.len - t0 : kLen);
    const uint32_t resets = reset_bits(p, w, t0, live);
    float2 a[kLen], h[kLen];  // h: first b_t, then the state before token t
    Run run{make_float2(1.f, 1.f), zero};
#pragma unroll
    for (int k = 0; k < kLen; ++k) {
      a[k] = make_float2(1.f, 1.f);
      h[k] = zero;
      if (k < live) {
        const float2 xv = load2<E, VEC>(x + (t0 + k) * p.x.token, w.n);
        const float2 rv = load2<E, VEC>(r + (t0 + k) * p.r.token, w.n);
        const float2 iv = load2<E, VEC>(i + (t0 + k) * p.i.token, w.n);
        const Gate g0 = gate(rv.x, iv.x, rate.x), g1 = gate(rv.y, iv.y, rate.y);
        const bool cut = resets >> k & 1u;
        a[k] = cut ? zero : make_float2(g0.a, g1.a);
        h[k] = make_float2((cut ? 1.f : g0.gain) * g0.si * xv.x, (cut ? 1.f : g1.gain) * g1.si * xv.y);
        run.a = make_float2(run.a.x * a[k].x, run.a.y * a[k].y);
        run.b = apply(Run{a[k], h[k]}, cut, run.b);
      }
    }
    Run rev{run.a, zero};
#pragma unroll
    for (int k = kLen - 1; k >= 0; --k)
      if (k < live) {
        const float2 d = load2<E, VEC>(dy + (t0 + k) * p.dy.token, w.n);
        const bool cut = resets >> k & 1u;
        rev.b = cut ? zero : make_float2(a[k].x * (rev.b.x + d.x), a[k].y * (rev.b.y + d.y));
      }
    __syncthreads();
    sh.run[w.slot][w.pair] = make_float4(run.a.x, run.a.y, run.b.x, run.b.y);
    back[w.slot][w.pair] = make_float4(rev.a.x, rev.a.y, rev.b.x, rev.b.y);
    if (w.pair == 0) sh.cut[w.slot] = resets;
    __syncthreads();
    float2 g;  // the flow into the end of the chunk, then of the run
    if (w.cluster > 1) {
      Run total = as_run(back[kSlots - 1][w.pair]);
      bool cut = sh.cut[kSlots - 1];
#pragma unroll
      for (int k = kSlots - 2; k >= 0; --k) {
        const Run next = as_run(back[k][w.pair]);
        total.b = apply(next, sh.cut[k], total.b);
        total.a = make_float2(total.a.x * next.a.x, total.a.y * next.a.y);
        cut = cut || sh.cut[k];
      }
      exchange(sh, (int)(s & 1), w, total, cut);
      g = flow;
      for (int k = w.cluster - 1; k >= 0; --k) {
        if (k == w.rank) g = flow;
        flow = apply(as_run(sh.total[s & 1][k][w.pair]), sh.total_cut[s & 1][k], flow);
      }
    } else {
      g = flow;
#pragma unroll
      for (int k = kSlots - 1; k >= 0; --k) flow = apply(as_run(back[k][w.pair]), sh.cut[k], flow);
    }
    for (int k = kSlots - 1; k > w.slot; --k) g = apply(as_run(back[k][w.pair]), sh.cut[k], g);
    float2 before = chunk < chunks ? load_f32(p.states + (w.b * chunks + chunk) * p.D + w.d, w.n) : zero;
    for (int k = 0; k < w.slot; ++k) before = apply(as_run(sh.run[k][w.pair]), sh.cut[k], before);
#pragma unroll
    for (int k = 0; k < kLen; ++k)
      if (k < live) {
        const float2 next = apply(Run{a[k], h[k]}, resets >> k & 1u, before);
        h[k] = before;
        before = next;
      }
    float2 part = zero;
#pragma unroll
    for (int k = kLen - 1; k >= 0; --k) {
      const int64_t t = t0 + k;
      if (k < live) {
        const float2 xv = load2<E, VEC>(x + t * p.x.token, w.n);
        const float2 rv = load2<E, VEC>(r + t * p.r.token, w.n);
        const float2 iv = load2<E, VEC>(i + t * p.i.token, w.n);
        const float2 dv = load2<E, VEC>(dy + t * p.dy.token, w.n);
        const bool cut = resets >> k & 1u;
        float ox[2], orr[2], oi[2];
        const float xs[2] = {xv.x, xv.y}, rs[2] = {rv.x, rv.y}, is[2] = {iv.x, iv.y};
        const float gs_[2] = {g.x + dv.x, g.y + dv.y}, as[2] = {a[k].x, a[k].y}, hs[2] = {h[k].x, h[k].y};
        const float ra[2] = {rate.x, rate.y};
        float ps[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const Gate e = gate(rs[q], is[q], ra[q]);
          const float gain = cut ? 1.f : e.gain;
          const float gx = gs_[q] * e.si * xs[q];
          ox[q] = gs_[q] * gain * e.si;
          oi[q] = gx * gain * (1.f - e.si);
          const float ga = gs_[q] * as[q] * hs[q], gv = gx * as[q] * as[q] * e.z * e.rx;
          orr[q] = cut ? 0.f : (1.f - e.sr) * ra[q] * (gv - ga * e.sr);
          ps[q] = cut ? 0.f : ga * e.sr - gv;
        }
        store2<E, VEC>(dx + t * p.dx.token, w.n, make_float2(ox[0], ox[1]));
        store2<E, VEC>(dr + t * p.dr.token, w.n, make_float2(orr[0], orr[1]));
        store2<E, VEC>(di + t * p.di.token, w.n, make_float2(oi[0], oi[1]));
        part = make_float2(part.x + ps[0], part.y + ps[1]);
        g = cut ? zero : make_float2(as[0] * gs_[0], as[1] * gs_[1]);
      } else if (t < p.T) {
        store2<E, VEC>(dx + t * p.dx.token, w.n, zero);
        store2<E, VEC>(dr + t * p.dr.token, w.n, zero);
        store2<E, VEC>(di + t * p.di.token, w.n, zero);
      }
    }
    sum = make_float2(sum.x + part.x, sum.y + part.y);
  }
  for (int64_t chunk = steps * w.cluster + w.rank; chunk < chunks; chunk += w.cluster)
    for (int k = 0; k < kLen; ++k) {
      const int64_t t = chunk * kChunk + w.slot * kLen + k;
      if (t < p.T) {
        store2<E, VEC>(dx + t * p.dx.token, w.n, zero);
        store2<E, VEC>(dr + t * p.dr.token, w.n, zero);
        store2<E, VEC>(di + t * p.di.token, w.n, zero);
      }
    }
  if (p.dh0 && w.rank == 0 && w.slot == 0) store_f32(p.dh0 + w.b * p.D + w.d, w.n, flow);
  // the CTA's share of the decay's gradient, its warps in order
  __syncthreads();
  back[w.slot][w.pair] = make_float4(sum.x, sum.y, 0.f, 0.f);
  __syncthreads();
  if (w.slot == 0) {
    for (int k = 1; k < kSlots; ++k) {
      sum.x += back[k][w.pair].x;
      sum.y += back[k][w.pair].y;
    }
    store_f32(p.partial + (w.b * w.cluster + w.rank) * p.D + w.d, w.n, sum);
  }
}

// ddecay[d] = -c sigmoid(lambda) * the sum of the CTAs' shares, in a fixed order.
__global__ void __launch_bounds__(256)
k_recurrence_decay(const float* partial, int64_t n, int64_t D, const float* decay, float c, float* ddecay) {
  grid_begin();
  __shared__ float part[8][32];
  const int64_t d = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
  const int w = threadIdx.x >> 5;
  float sum = 0.f;
  if (d < D)
    for (int64_t k = w; k < n; k += 8) sum += partial[k * D + d];
  part[w][threadIdx.x & 31] = sum;
  __syncthreads();
  if (w == 0 && d < D) {
#pragma unroll
    for (int k = 1; k < 8; ++k) sum += part[k][threadIdx.x];
    ddecay[d] = -c * sum / (1.f + expf(-decay[d]));
  }
}

template <typename E, bool VEC>
__global__ void __launch_bounds__(128) k_recurrence_step(const __grid_constant__ RecurrenceStepParams p) {
  grid_begin();
  const int64_t d = 2 * ((int64_t)blockIdx.x * 128 + threadIdx.x);
  const int n = (int)(p.D - d < 0 ? 0 : p.D - d < 2 ? p.D - d : 2);
  if (n == 0) return;
  for (int64_t b = blockIdx.y; b < p.B; b += gridDim.y) {
    const int64_t slot = p.slots ? p.slots[b] : b;
    float2 h = make_float2(0.f, 0.f);
    if (slot >= 0 && slot < p.n_slots) {
      const float2 lam = load_f32(p.decay + d, n);
      const float2 xv = load2<E, VEC>(static_cast<const E*>(p.x) + b * p.x_stride + d, n);
      const float2 rv = load2<E, VEC>(static_cast<const E*>(p.r) + b * p.r_stride + d, n);
      const float2 iv = load2<E, VEC>(static_cast<const E*>(p.i) + b * p.i_stride + d, n);
      float* state = p.state + slot * p.state_stride + d;
      h = load_f32(state, n);
      const Gate g0 = gate(rv.x, iv.x, p.c * softplus(lam.x));
      const Gate g1 = gate(rv.y, iv.y, p.c * softplus(lam.y));
      h.x = fmaf(g0.a, h.x, g0.gain * g0.si * xv.x);
      h.y = fmaf(g1.a, h.y, g1.gain * g1.si * xv.y);
      store_f32(state, n, h);
    }
    store2<E, VEC>(static_cast<E*>(p.y) + b * p.y_stride + d, n, h);
  }
}

unsigned grid_of(RecurrenceParams& p, int cluster) {
  p.groups = (int32_t)((p.D + kChannels - 1) / kChannels);
  return (unsigned)(p.B * p.groups * cluster);
}

}  // namespace

int64_t recurrence_chunks(int64_t T) { return (T + kChunk - 1) / kChunk; }

// CTAs that share a row's time: doubled while the device (152 SMs, two CTAs each) has room and
// there are chunks to deal.
int recurrence_cluster(int64_t B, int64_t T, int64_t D) {
  const int64_t columns = B * ((D + kChannels - 1) / kChannels);
  int c = 1;
  while (c < kMaxCluster && columns * c < 2 * 152 && 2 * c <= recurrence_chunks(T)) c *= 2;
  return c;
}

cudaError_t launch_recurrence_forward(RecurrenceParams p, int dtype, bool vec, cudaStream_t s) {
  const int cluster = recurrence_cluster(p.B, p.T, p.D);
  const unsigned grid = grid_of(p, cluster);
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return vec ? launch_cluster(k_recurrence_forward<E, true>, dim3(grid), dim3(kThreads), 0, cluster, s, p)
               : launch_cluster(k_recurrence_forward<E, false>, dim3(grid), dim3(kThreads), 0, cluster, s, p);
  });
}

cudaError_t launch_recurrence_backward(RecurrenceParams p, float* ddecay, int dtype, bool vec, cudaStream_t s) {
  const int cluster = recurrence_cluster(p.B, p.T, p.D);
  const unsigned grid = grid_of(p, cluster);
  cudaError_t err = grid == 0 ? cudaSuccess : with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return vec ? launch_cluster(k_recurrence_backward<E, true>, dim3(grid), dim3(kThreads), 0, cluster, s, p)
               : launch_cluster(k_recurrence_backward<E, false>, dim3(grid), dim3(kThreads), 0, cluster, s, p);
  });
  if (err != cudaSuccess) return err;
  return launch(k_recurrence_decay, dim3((unsigned)((p.D + 31) / 32)), dim3(256), s, (const float*)p.partial,
                p.B * cluster, p.D, p.decay, p.c, ddecay);
}

cudaError_t launch_recurrence_step(const RecurrenceStepParams& p, int dtype, bool vec, cudaStream_t s) {
  const dim3 grid((unsigned)((p.D + 255) / 256), (unsigned)(p.B < 65535 ? p.B : 65535));
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return vec ? launch(k_recurrence_step<E, true>, grid, dim3(128), s, p)
               : launch(k_recurrence_step<E, false>, grid, dim3(128), s, p);
  });
}

}  // namespace gs
