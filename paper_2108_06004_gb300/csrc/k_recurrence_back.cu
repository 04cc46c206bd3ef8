// Backward pass of the gated linear recurrence.
//
// With the flow F_t = a_{t+1} g_{t+1} into token t from behind (dh_last past the end) and
// g_t = dy_t + F_t, F is the same kind of recurrence as h, walked from the end: F_{t-1} = a_t (F_t + dy_t).
// Per token, with K = sqrt(1 - a^2) sigmoid(i), b = K x and 1 - a^2 = sigmoid(r) X:
//   dx = g K,  di = g b (1 - sigmoid(i)),
//   m = a g (h_{t-1} sigmoid(r) - b a / X),   dr = -rate (1 - sigmoid(r)) m,   ddecay = -c sigmoid(lambda) sum m.
// h_{t-1} is recomputed in fp32 from the state at the start of the chunk, which the forward pass
// kept (4 bytes for kStateEvery tokens and channel), not read back from the rounded y.
//
// The cut of time over threads, warps and cluster CTAs is that of the forward pass, with runs of 8
// tokens: a token's five factors (a, sigmoid(r), K, b (1 - sigmoid(i)), b a / X) stay in registers from the
// first walk, which needs all transcendental functions, to the last, which writes.
#include "recurrence.cuh"

namespace gs {
namespace {

using namespace rec;

constexpr int kLen = 8;                  // tokens of a run
constexpr int kChunk = kSlots * kLen;    // tokens of a CTA's step
static_assert(kChunk == kStateEvery, "a step starts at a kept state");

template <typename E>
struct BackwardShared {
  E tile[2][4][kChunk][kChannels];       // x, r, i, dy; the next step's are under way
  float4 run[kSlots][kPairs];            // the map of h over each warp's run
  float2 back[kSlots][kPairs];           // the offset of the flow's map (its factor is the same)
  uint32_t cut[kSlots];
  Totals totals;
};

template <typename E, int UNIT, bool PAIR, bool RESET>
__global__ void __launch_bounds__(kThreads, sizeof(E) == 2 ? 2 : 1)
k_recurrence_backward(const __grid_constant__ RecurrenceParams p) {
  extern __shared__ __align__(128) unsigned char raw[];
  BackwardShared<E>& sh = *reinterpret_cast<BackwardShared<E>*>(raw);
  using Raw = typename Pack2<E>::type;
  grid_begin();
  const Place w = place(p);
  if (w.cluster > 1) cg::this_cluster().sync();  // every CTA of the cluster runs before its memory is written
  const int64_t steps = ((w.len + kChunk - 1) / kChunk + w.cluster - 1) / w.cluster;
  const int64_t kept = (p.T + kStateEvery - 1) / kStateEvery;
  const int channels = clamp_int(p.D - w.d0, kChannels);
  const E* x = static_cast<const E*>(p.x.data) + w.b * p.x.batch + w.d0;
  const E* r = static_cast<const E*>(p.r.data) + w.b * p.r.batch + w.d0;
  const E* i = static_cast<const E*>(p.i.data) + w.b * p.i.batch + w.d0;
  const E* dy = static_cast<const E*>(p.dy.data) + w.b * p.dy.batch + w.d0;
  E* dx = static_cast<E*>(p.dx.data) + w.b * p.dx.batch + w.d;
  E* dr = static_cast<E*>(p.dr.data) + w.b * p.dr.batch + w.d;
  E* di = static_cast<E*>(p.di.data) + w.b * p.di.batch + w.d;
  auto load = [&](int64_t s) {
    const int64_t t0 = (s * w.cluster + w.rank) * kChunk;
    const int live = clamp_int(w.len - t0, kChunk);
    load_tile<E, UNIT, kChunk>(&sh.tile[s & 1][0][0][0], x, p.x.token, t0, live, channels);
    load_tile<E, UNIT, kChunk>(&sh.tile[s & 1][1][0][0], r, p.r.token, t0, live, channels);
    load_tile<E, UNIT, kChunk>(&sh.tile[s & 1][2][0][0], i, p.i.token, t0, live, channels);
    load_tile<E, UNIT, kChunk>(&sh.tile[s & 1][3][0][0], dy, p.dy.token, t0, live, channels);
  };
  auto first_token = [&](int64_t s) { return (s * w.cluster + w.rank) * kChunk + w.slot * kLen; };
  if (steps > 0) load(steps - 1);
  copy_commit();
  const float2 rate = decay_rate(load_f32(p.decay + w.d, w.n), p.c);
  const bool series = __all_sync(0xFFFFFFFFu, rate.x <= kSeries && rate.y <= kSeries);
  float2 flow = load_f32(p.dh_last ? p.dh_last + w.b * p.D + w.d : nullptr, w.n);
  float2 sum = two(0.f);
  uint8_t flag = 0;
  if (RESET && steps > 0)
    flag = reset_flag(p, w, first_token(steps - 1), clamp_int(w.len - first_token(steps - 1), kLen));
  for (int64_t s = steps - 1; s >= 0; --s) {
    const int64_t t0 = first_token(s);
    const int live = clamp_int(w.len - t0, kLen);
    const uint32_t resets = RESET ? __ballot_sync(0xFFFFFFFFu, flag != 0) : 0;
    if (RESET && s > 0) flag = reset_flag(p, w, first_token(s - 1), clamp_int(w.len - first_token(s - 1), kLen));
    const int64_t chunk = s * w.cluster + w.rank;
    float2 h = chunk < kept ? load_f32(p.states + (w.b * kept + chunk) * p.D + w.d, w.n) : two(0.f);
    copy_wait<0>();
    __syncthreads();  // the tile is here, and the one before has been read
    if (s > 0) load(s - 1);
    copy_commit();
    auto value = [&](int which, int k) {
      return Pack2<E>::up(reinterpret_cast<const Raw*>(sh.tile[s & 1][which][w.slot * kLen + k])[w.pair]);
    };
    float2 a[kLen], sr[kLen], K[kLen], U[kLen], Q[kLen];
    Run run = identity();
    auto gates = [&](auto some, auto in_series) {
      constexpr bool SOME = decltype(some)::value;
#pragma unroll
      for (int k = 0; k < kLen; ++k) {
        const float2 xv = value(0, k);
        const Gate g = gate<decltype(in_series)::value>(value(1, k), value(2, k), rate);
        const bool cut = RESET && (resets >> k & 1u);
        a[k] = choose(cut, two(0.f), g.a);
        sr[k] = g.sr;
        K[k] = mul(choose(cut, two(1.f), g.gain), g.si);
        float2 b = mul(K[k], xv);
        U[k] = mul(b, fma(g.si, two(-1.f), two(1.f)));
        Q[k] = mul(mul(b, g.a), mul(g.rx, g.rx));
        if (SOME && k >= live) {  // past the end of the row: the state and the flow stay
          a[k] = two(1.f);
          K[k] = b = two(0.f);
        }
        run.a = mul(run.a, a[k]);
        run.b = RESET ? apply(Run{a[k], b}, cut, run.b) : fma(a[k], run.b, b);
      }
    };
    if (live == kLen) {
      if (series)
        gates(std::false_type(), std::true_type());
      else
        gates(std::false_type(), std::false_type());
    } else {
      gates(std::true_type(), std::false_type());
    }
    float2 back = two(0.f);
#pragma unroll
    for (int k = kLen - 1; k >= 0; --k) {
      const float2 f = mul(a[k], add(back, value(3, k)));  // past the end dy is zero in the tile
      back = RESET ? choose(resets >> k & 1u, two(0.f), f) : f;
    }
    sh.run[w.slot][w.pair] = as_float4(run);
    sh.back[w.slot][w.pair] = back;
    if (RESET && w.pair == 0) sh.cut[w.slot] = resets;
    __syncthreads();
    // the maps of the flow over the warps after this one, and over the whole chunk; the state
    // before this warp's run
    Run after, total = identity();
    bool after_cut, cut = false;
#pragma unroll
    for (int k = kSlots - 1; k >= 0; --k) {
      if (k == w.slot) {
        after = total;
        after_cut = cut;
      }
      Run m = as_run(sh.run[k][w.pair]);
      m.b = sh.back[k][w.pair];
      extend(total, cut, m, RESET && sh.cut[k] != 0);
    }
#pragma unroll
    for (int k = 0; k < kSlots - 1; ++k)
      if (k < w.slot) h = apply(as_run(sh.run[k][w.pair]), RESET && sh.cut[k] != 0, h);
    float2 f = flow;
    if (w.cluster > 1) {
      exchange(sh.totals, (int)(s & 1), w, total, cut);
      for (int k = w.cluster - 1; k >= 0; --k) {
        if (k == w.rank) f = flow;
        flow = apply(as_run(sh.totals.run[s & 1][k][w.pair]), RESET && sh.totals.cut[s & 1][k] != 0, flow);
      }
    } else {
      flow = apply(total, cut, flow);
    }
    f = apply(after, after_cut, f);
#pragma unroll
    for (int k = 0; k < kLen; ++k) {
      Q[k] = fma(h, sr[k], make_float2(-Q[k].x, -Q[k].y));
      const float2 b = mul(K[k], value(0, k));
      h = RESET ? apply(Run{a[k], b}, resets >> k & 1u, h) : fma(a[k], h, b);
    }
    float2 part = two(0.f);
    E *out_x = dx + (t0 + kLen - 1) * p.dx.token, *out_r = dr + (t0 + kLen - 1) * p.dr.token,
      *out_i = di + (t0 + kLen - 1) * p.di.token;
#pragma unroll
    for (int k = kLen - 1; k >= 0; --k) {
      if (k < live) {
        const bool cut = RESET && (resets >> k & 1u);
        const float2 g = add(f, value(3, k));
        f = choose(cut, two(0.f), mul(a[k], g));
        const float2 m = choose(cut, two(0.f), mul(f, Q[k]));
        part = add(part, m);
        const float2 slope = mul(rate, fma(sr[k], two(1.f), two(-1.f)));
        store2<E, PAIR>(out_x, w.n, mul(g, K[k]));
        store2<E, PAIR>(out_i, w.n, mul(g, U[k]));
        store2<E, PAIR>(out_r, w.n, mul(slope, m));
      } else if (t0 + k < p.T) {
        store2<E, PAIR>(out_x, w.n, two(0.f));
        store2<E, PAIR>(out_i, w.n, two(0.f));
        store2<E, PAIR>(out_r, w.n, two(0.f));
      }
      out_x -= p.dx.token;
      out_r -= p.dr.token;
      out_i -= p.di.token;
    }
    sum = add(sum, part);
  }
  // past the last step every token is masked
  for (int64_t chunk = steps * w.cluster + w.rank; chunk * kChunk < p.T; chunk += w.cluster)
    for (int k = 0; k < kLen; ++k) {
      const int64_t t = chunk * kChunk + w.slot * kLen + k;
      if (t < p.T) {
        store2<E, PAIR>(dx + t * p.dx.token, w.n, two(0.f));
        store2<E, PAIR>(dr + t * p.dr.token, w.n, two(0.f));
        store2<E, PAIR>(di + t * p.di.token, w.n, two(0.f));
      }
    }
  if (p.dh0 && w.rank == 0 && w.slot == 0) store_f32(p.dh0 + w.b * p.D + w.d, w.n, flow);
  // the CTA's share of the decay's gradient, its warps in order
  __syncthreads();
  sh.back[w.slot][w.pair] = sum;
  __syncthreads();
  if (w.slot == 0) {
#pragma unroll
    for (int k = 1; k < kSlots; ++k) sum = add(sum, sh.back[k][w.pair]);
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

template <typename E, int UNIT, bool PAIR, bool RESET>
cudaError_t run_backward(const RecurrenceParams& p, unsigned grid, int cluster, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kernel = k_recurrence_backward<E, UNIT, PAIR, RESET>;
  const cudaError_t e = prepare_kernel(kernel, sizeof(BackwardShared<E>), done);
  if (e != cudaSuccess) return e;
  return launch_cluster(kernel, dim3(grid), dim3(kThreads), sizeof(BackwardShared<E>), cluster, s, p);
}

template <typename E, int UNIT, bool PAIR>
cudaError_t run_backward(const RecurrenceParams& p, unsigned grid, int cluster, cudaStream_t s) {
  return p.reset ? run_backward<E, UNIT, PAIR, true>(p, grid, cluster, s)
                 : run_backward<E, UNIT, PAIR, false>(p, grid, cluster, s);
}

}  // namespace

cudaError_t launch_recurrence_backward(RecurrenceParams p, float* ddecay, int dtype, int unit, bool pair,
                                       cudaStream_t s) {
  const int cluster = recurrence_cluster(p.B, p.T, p.D);
  p.groups = (int32_t)((p.D + kChannels - 1) / kChannels);
  const unsigned grid = (unsigned)(p.B * p.groups * cluster);
  cudaError_t err = grid == 0 ? cudaSuccess : with_type(dtype, [&](auto e) {
    using E = decltype(e);
    if (unit == 16 && pair) return run_backward<E, 16, true>(p, grid, cluster, s);
    if constexpr (sizeof(E) == 2) {
      if (unit >= 4 && pair) return run_backward<E, 4, true>(p, grid, cluster, s);
      return run_backward<E, 2, false>(p, grid, cluster, s);
    } else {
      return run_backward<E, 4, false>(p, grid, cluster, s);
    }
  });
  if (err != cudaSuccess) return err;
  return launch(k_recurrence_decay, dim3((unsigned)((p.D + 31) / 32)), dim3(256), s, (const float*)p.partial,
                p.B * cluster, p.D, p.decay, p.c, ddecay);
}

}  // namespace gs
