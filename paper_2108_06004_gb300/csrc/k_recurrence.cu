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
#include "recurrence.cuh"

namespace gs {
namespace {

using namespace rec;

constexpr int kLen = 16;                 // tokens of a run

template <typename E, int CH>
struct ForwardShared {
  static constexpr int kRuns = Tile<E, CH, kLen>::kRuns;
  static constexpr int kStages = sizeof(E) == 2 ? 2 : 1;
  Tile<E, CH, kLen> tile[kStages][3];    // x, r, i; those of steps to come are under way
  float4 run[kRuns][CH / 2];             // the map of each run
  uint32_t cut[kRuns];
};

template <typename E, int CH, int UNIT, bool PAIR, bool RESET>
__global__ void __launch_bounds__(kThreads, 4)
k_recurrence_forward(const __grid_constant__ RecurrenceParams p) {
  using Shared = ForwardShared<E, CH>;
  constexpr int kRuns = Shared::kRuns, kStages = Shared::kStages, kChunk = kRuns * kLen;
  extern __shared__ __align__(128) unsigned char raw[];
  Shared& sh = *reinterpret_cast<Shared*>(raw);
  grid_begin();
  const Place w = place<CH>(p);
  Total<CH>* totals = reinterpret_cast<Total<CH>*>(raw + sizeof(Shared));  // [2][cluster], with a cluster
  if (w.cluster > 1) cg::this_cluster().sync();  // every CTA of the cluster runs before its memory is written
  const int64_t chunks = (w.len + kChunk - 1) / kChunk;
  const int steps = (int)((chunks + w.cluster - 1) / w.cluster);
  const int64_t kept = (p.T + kStateEvery - 1) / kStateEvery;
  const int channels = clamp_int(p.D - w.d0, CH);
  const E* x = static_cast<const E*>(p.x.data) + w.b * p.x.batch + w.d0;
  const E* r = static_cast<const E*>(p.r.data) + w.b * p.r.batch + w.d0;
  const E* i = static_cast<const E*>(p.i.data) + w.b * p.i.batch + w.d0;
  E* y = static_cast<E*>(p.y.data) + w.b * p.y.batch + w.d;
  auto chunk_token = [&](int s) { return ((int64_t)s * w.cluster + w.rank) * kChunk; };
  auto load = [&](int s) {
    const int64_t t0 = chunk_token(s);
    const int live = clamp_int(w.len - t0, kChunk);
    load_tile<UNIT>(sh.tile[s % kStages][0], x, p.x.token, t0, live, channels);
    load_tile<UNIT>(sh.tile[s % kStages][1], r, p.r.token, t0, live, channels);
    load_tile<UNIT>(sh.tile[s % kStages][2], i, p.i.token, t0, live, channels);
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) {
    if (s < steps) load(s);
    copy_commit();
  }
  const float2 rate = decay_rate(load_f32(p.decay + w.d, w.n), p.c);
  const bool series = __all_sync(0xFFFFFFFFu, rate.x <= kSeries && rate.y <= kSeries);
  float2 state = load_f32(p.h0 ? p.h0 + w.b * p.D + w.d : nullptr, w.n);
  uint8_t flag = RESET ? reset_flag<kLen>(p, w, chunk_token(0) + w.slot * kLen) : 0;
  for (int s = 0; s < steps; ++s) {
    const int64_t t0 = chunk_token(s) + w.slot * kLen;
    const bool full = chunk_token(s) + kChunk <= w.len;  // the chunk has no masked token
    const uint32_t resets = RESET ? reset_bits<CH, kLen>(flag) : 0;
    if (RESET) flag = reset_flag<kLen>(p, w, chunk_token(s + 1) + w.slot * kLen);
    copy_wait<kStages - 1>();
    __syncthreads();
    // the run's tokens as a_t and b_t, and their composition
    float2 a[kLen], b[kLen];
    Run run = identity();
    auto gates = [&](auto some, auto in_series) {
      const auto& tile = sh.tile[s % kStages];
#pragma unroll
      for (int k = 0; k < kLen; ++k) {
        const bool cut = RESET && (resets >> k & 1u);
        float2 K;
        gate_forward<decltype(in_series)::value>(capped(tile[1].at(w, k)), capped(tile[2].at(w, k)), rate, cut, a[k], K);
        b[k] = mul(K, widen(tile[0].at(w, k)));
        if (decltype(some)::value && t0 + k >= w.len) {  // past the end of the row: the state stays
          a[k] = two(1.f);
          b[k] = two(0.f);
        }
        run.a = mul(run.a, a[k]);
        run.b = RESET ? apply(Run{a[k], b[k]}, cut, run.b) : fma(a[k], run.b, b[k]);
      }
    };
    if (!full)
      gates(std::true_type(), std::false_type());
    else if (series)
      gates(std::false_type(), std::true_type());
    else
      gates(std::false_type(), std::false_type());
    sh.run[w.slot][w.pair] = as_float4(run);
    if (RESET && w.pair == 0) sh.cut[w.slot] = resets;
    __syncthreads();
    if (s + kStages < steps) load(s + kStages);  // this step's tile has been read
    copy_commit();
    // the maps of the runs before this one, and of the whole chunk
    Run before, total = identity();
    bool before_cut, cut = false;
#pragma unroll
    for (int k = 0; k < kRuns; ++k) {
      if (k == w.slot) {
        before = total;
        before_cut = cut;
      }
      extend(total, cut, as_run(sh.run[k][w.pair]), RESET && sh.cut[k] != 0);
    }
    float2 h = state;
    if (w.cluster > 1) {
      Total<CH>* table = totals + (s & 1) * w.cluster;
      exchange<CH, kRuns>(table, w, total, cut);
      for (int k = 0; k < w.cluster; ++k) {
        if (k == w.rank) h = state;
        state = apply(as_run(table[k].run[w.pair]), RESET && table[k].cut != 0, state);
      }
    } else {
      state = apply(total, cut, state);
    }
    h = apply(before, before_cut, h);
    if (p.states && t0 % kStateEvery == 0 && t0 / kStateEvery < kept)
      store_f32(p.states + (w.b * kept + t0 / kStateEvery) * p.D + w.d, w.n, h);
    E* out = y + t0 * p.y.token;
    if (full && PAIR && w.n == 2) {
#pragma unroll
      for (int k = 0; k < kLen; ++k) {
        h = RESET ? apply(Run{a[k], b[k]}, resets >> k & 1u, h) : fma(a[k], h, b[k]);
        *reinterpret_cast<typename Pack2<E>::type*>(out) = Pack2<E>::down(h);
        out += p.y.token;
      }
    } else {
#pragma unroll
      for (int k = 0; k < kLen; ++k) {
        h = RESET ? apply(Run{a[k], b[k]}, resets >> k & 1u, h) : fma(a[k], h, b[k]);
        if (t0 + k < p.T) store2<E, PAIR>(out, w.n, t0 + k < w.len ? h : two(0.f));
        out += p.y.token;
      }
    }
  }
  // past the last step every token is masked
  for (int64_t t0 = chunk_token(steps); t0 < p.T; t0 += (int64_t)w.cluster * kChunk)
    for (int k = 0; k < kLen; ++k) {
      const int64_t t = t0 + w.slot * kLen + k;
      if (t < p.T) store2<E, PAIR>(y + t * p.y.token, w.n, two(0.f));
    }
  if (p.h_last && w.rank == 0 && w.slot == 0) store_f32(p.h_last + w.b * p.D + w.d, w.n, state);
}

template <typename E, int CH, int UNIT, bool PAIR, bool RESET>
cudaError_t run_forward(RecurrenceParams p, const RecurrenceShape& shape, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kernel = k_recurrence_forward<E, CH, UNIT, PAIR, RESET>;
  constexpr size_t kBase = sizeof(ForwardShared<E, CH>), kTotal = 2 * sizeof(Total<CH>);
  const cudaError_t e = prepare_kernel(kernel, kBase + kMaxCluster * kTotal, done);
  if (e != cudaSuccess) return e;
  p.groups = shape.groups;
  const size_t smem = kBase + (shape.cluster > 1 ? shape.cluster * kTotal : 0);
  return launch_cluster(kernel, dim3(shape.grid), dim3(kThreads), smem, shape.cluster, s, p);
}

template <typename E, int CH, int UNIT, bool PAIR>
cudaError_t run_forward(const RecurrenceParams& p, const RecurrenceShape& shape, cudaStream_t s) {
  return p.reset ? run_forward<E, CH, UNIT, PAIR, true>(p, shape, s) : run_forward<E, CH, UNIT, PAIR, false>(p, shape, s);
}

// Two adjacent channels of one token, zero where they do not exist.
template <typename E, bool PAIR>
__device__ __forceinline__ float2 load2(const E* p, int n) {
  if (PAIR && n == 2) return widen(*reinterpret_cast<const typename Pack2<E>::type*>(p));
  return make_float2(n > 0 ? to_f32(p[0]) : 0.f, n > 1 ? to_f32(p[1]) : 0.f);
}

template <typename E, bool PAIR>
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
      const float2 xv = load2<E, PAIR>(static_cast<const E*>(p.x) + b * p.x_stride + d, n);
      const float2 rv = load2<E, PAIR>(static_cast<const E*>(p.r) + b * p.r_stride + d, n);
      const float2 iv = load2<E, PAIR>(static_cast<const E*>(p.i) + b * p.i_stride + d, n);
      float* state = p.state + slot * p.state_stride + d;
      h = load_f32(state, n);
      float2 a, K;
      gate_forward<false>(capped(rv), capped(iv), decay_rate(lam, p.c), false, a, K);
      h = fma(a, h, mul(K, xv));
      store_f32(state, n, h);
    }
    store2<E, PAIR>(static_cast<E*>(p.y) + b * p.y_stride + d, n, h);
  }
}

}  // namespace

int64_t recurrence_states(int64_t T) { return (T + kStateEvery - 1) / kStateEvery; }

// How a pass of `run` tokens a thread is cut: the channels of a CTA, and the CTAs of a cluster that
// share a row's time.  SMs hold about four CTAs; the cluster is doubled until there are three for
// each SM or no chunks left to deal.  Where 64 channels a CTA do not get there, 32 do better: twice
// the CTAs, with twice the tokens each.
RecurrenceShape recurrence_shape(int64_t B, int64_t T, int64_t D, int run, bool narrow) {
  RecurrenceShape best = {};
  for (int channels : {64, 32}) {
    RecurrenceShape c;
    c.channels = channels;
    c.groups = (int32_t)((D + channels - 1) / channels);
    const int64_t columns = B * c.groups, chunk = kThreads / (channels / 2) * run;
    c.cluster = 1;
    while (c.cluster < kMaxCluster && columns * c.cluster < 3 * kSMs && 2 * c.cluster * chunk <= T) c.cluster *= 2;
    c.grid = (unsigned)(columns * c.cluster);
    if (channels == 64) best = c;
    else if (narrow && best.grid < 2 * kSMs && c.grid > best.grid) best = c;
  }
  return best;
}

cudaError_t launch_recurrence_forward(const RecurrenceParams& p, int dtype, int unit, bool pair, cudaStream_t s) {
  const RecurrenceShape shape = recurrence_shape(p.B, p.T, p.D, kLen, unit == 16 && pair);
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    if (unit == 16 && pair)
      return shape.channels == 64 ? run_forward<E, 64, 16, true>(p, shape, s) : run_forward<E, 32, 16, true>(p, shape, s);
    if constexpr (sizeof(E) == 2) {
      if (unit >= 4 && pair) return run_forward<E, 64, 4, true>(p, shape, s);
      return run_forward<E, 64, 2, false>(p, shape, s);
    } else {
      return run_forward<E, 64, 4, false>(p, shape, s);
    }
  });
}

cudaError_t launch_recurrence_step(const RecurrenceStepParams& p, int dtype, bool pair, cudaStream_t s) {
  const dim3 grid((unsigned)((p.D + 255) / 256), (unsigned)(p.B < 65535 ? p.B : 65535));
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return pair ? launch(k_recurrence_step<E, true>, grid, dim3(128), s, p)
                : launch(k_recurrence_step<E, false>, grid, dim3(128), s, p);
  });
}

}  // namespace gs
