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
constexpr int kChunk = kSlots * kLen;    // tokens of a CTA's step

template <typename E>
struct ForwardShared {
  E tile[2][3][kChunk][kChannels];       // x, r, i; the next step's are under way
  float4 run[kSlots][kPairs];            // the map of each warp's run
  uint32_t cut[kSlots];
  Totals totals;
};

template <typename E, int UNIT, bool PAIR, bool RESET>
__global__ void __launch_bounds__(kThreads, sizeof(E) == 2 ? 2 : 1)
k_recurrence_forward(const __grid_constant__ RecurrenceParams p) {
  extern __shared__ __align__(128) unsigned char raw[];
  ForwardShared<E>& sh = *reinterpret_cast<ForwardShared<E>*>(raw);
  grid_begin();
  const Place w = place(p);
  if (w.cluster > 1) cg::this_cluster().sync();  // every CTA of the cluster runs before its memory is written
  const int64_t chunks = (w.len + kChunk - 1) / kChunk;
  const int64_t steps = (chunks + w.cluster - 1) / w.cluster;
  const int64_t kept = (p.T + kStateEvery - 1) / kStateEvery;
  const int channels = clamp_int(p.D - w.d0, kChannels);
  const E* x = static_cast<const E*>(p.x.data) + w.b * p.x.batch + w.d0;
  const E* r = static_cast<const E*>(p.r.data) + w.b * p.r.batch + w.d0;
  const E* i = static_cast<const E*>(p.i.data) + w.b * p.i.batch + w.d0;
  E* y = static_cast<E*>(p.y.data) + w.b * p.y.batch + w.d;
  auto load = [&](int64_t s) {
    const int64_t t0 = (s * w.cluster + w.rank) * kChunk;
    const int live = clamp_int(w.len - t0, kChunk);
    load_tile<E, UNIT, kChunk>(&sh.tile[s & 1][0][0][0], x, p.x.token, t0, live, channels);
    load_tile<E, UNIT, kChunk>(&sh.tile[s & 1][1][0][0], r, p.r.token, t0, live, channels);
    load_tile<E, UNIT, kChunk>(&sh.tile[s & 1][2][0][0], i, p.i.token, t0, live, channels);
  };
  auto first_token = [&](int64_t s) { return (s * w.cluster + w.rank) * kChunk + w.slot * kLen; };
  if (steps > 0) load(0);
  copy_commit();
  if (steps > 1) load(1);
  copy_commit();
  const float2 rate = decay_rate(load_f32(p.decay + w.d, w.n), p.c);
  const bool series = __all_sync(0xFFFFFFFFu, rate.x <= kSeries && rate.y <= kSeries);
  float2 state = load_f32(p.h0 ? p.h0 + w.b * p.D + w.d : nullptr, w.n);
  uint8_t flag = 0;
  if (RESET && steps > 0) flag = reset_flag(p, w, first_token(0), clamp_int(w.len - first_token(0), kLen));
  for (int64_t s = 0; s < steps; ++s) {
    const int64_t t0 = first_token(s);
    const int live = clamp_int(w.len - t0, kLen);
    const uint32_t resets = RESET ? __ballot_sync(0xFFFFFFFFu, flag != 0) : 0;
    if (RESET && s + 1 < steps)
      flag = reset_flag(p, w, first_token(s + 1), clamp_int(w.len - first_token(s + 1), kLen));
    copy_wait<1>();
    __syncthreads();
    // the run's tokens as a_t and b_t, and their composition
    float2 a[kLen], b[kLen];
    Run run = identity();
    auto gates = [&](auto some, auto in_series) {
      constexpr bool SOME = decltype(some)::value;
#pragma unroll
      for (int k = 0; k < kLen; ++k) {
        using Raw = typename Pack2<E>::type;
        const int row = w.slot * kLen + k;
        const float2 xv = Pack2<E>::up(reinterpret_cast<const Raw*>(sh.tile[s & 1][0][row])[w.pair]);
        const float2 rv = Pack2<E>::up(reinterpret_cast<const Raw*>(sh.tile[s & 1][1][row])[w.pair]);
        const float2 iv = Pack2<E>::up(reinterpret_cast<const Raw*>(sh.tile[s & 1][2][row])[w.pair]);
        const Gate g = gate<decltype(in_series)::value>(rv, iv, rate);
        const bool cut = RESET && (resets >> k & 1u);
        a[k] = choose(cut, two(0.f), g.a);
        b[k] = mul(mul(choose(cut, two(1.f), g.gain), g.si), xv);
        if (SOME && k >= live) {  // past the end of the row: the state stays
          a[k] = two(1.f);
          b[k] = two(0.f);
        }
        run.a = mul(run.a, a[k]);
        run.b = RESET ? apply(Run{a[k], b[k]}, cut, run.b) : fma(a[k], run.b, b[k]);
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
    sh.run[w.slot][w.pair] = as_float4(run);
    if (RESET && w.pair == 0) sh.cut[w.slot] = resets;
    __syncthreads();
    if (s + 2 < steps) load(s + 2);  // this step's tile has been read
    copy_commit();
    // the maps of the warps before this one, and of the whole chunk
    Run before, total = identity();
    bool before_cut, cut = false;
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      if (k == w.slot) {
        before = total;
        before_cut = cut;
      }
      extend(total, cut, as_run(sh.run[k][w.pair]), RESET && sh.cut[k] != 0);
    }
    float2 h = state;
    if (w.cluster > 1) {
      exchange(sh.totals, (int)(s & 1), w, total, cut);
      for (int k = 0; k < w.cluster; ++k) {
        if (k == w.rank) h = state;
        state = apply(as_run(sh.totals.run[s & 1][k][w.pair]), RESET && sh.totals.cut[s & 1][k] != 0, state);
      }
    } else {
      state = apply(total, cut, state);
    }
    h = apply(before, before_cut, h);
    if (p.states && w.slot % (kStateEvery / kLen) == 0 && t0 / kStateEvery < kept)
      store_f32(p.states + (w.b * kept + t0 / kStateEvery) * p.D + w.d, w.n, h);
    E* out = y + t0 * p.y.token;
#pragma unroll
    for (int k = 0; k < kLen; ++k) {
      if (k < live) {
        h = RESET ? apply(Run{a[k], b[k]}, resets >> k & 1u, h) : fma(a[k], h, b[k]);
        store2<E, PAIR>(out, w.n, h);
      } else if (t0 + k < p.T) {
        store2<E, PAIR>(out, w.n, two(0.f));
      }
      out += p.y.token;
    }
  }
  // past the last step every token is masked
  for (int64_t chunk = steps * w.cluster + w.rank; chunk * kChunk < p.T; chunk += w.cluster)
    for (int k = 0; k < kLen; ++k) {
      const int64_t t = chunk * kChunk + w.slot * kLen + k;
      if (t < p.T) store2<E, PAIR>(y + t * p.y.token, w.n, two(0.f));
    }
  if (p.h_last && w.rank == 0 && w.slot == 0) store_f32(p.h_last + w.b * p.D + w.d, w.n, state);
}

template <typename E, int UNIT, bool PAIR, bool RESET>
cudaError_t run_forward(const RecurrenceParams& p, unsigned grid, int cluster, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kernel = k_recurrence_forward<E, UNIT, PAIR, RESET>;
  const cudaError_t e = prepare_kernel(kernel, sizeof(ForwardShared<E>), done);
  if (e != cudaSuccess) return e;
  return launch_cluster(kernel, dim3(grid), dim3(kThreads), sizeof(ForwardShared<E>), cluster, s, p);
}

template <typename E, int UNIT, bool PAIR>
cudaError_t run_forward(const RecurrenceParams& p, unsigned grid, int cluster, cudaStream_t s) {
  return p.reset ? run_forward<E, UNIT, PAIR, true>(p, grid, cluster, s)
                 : run_forward<E, UNIT, PAIR, false>(p, grid, cluster, s);
}

// Two adjacent channels of one token, zero where they do not exist.
template <typename E, bool PAIR>
__device__ __forceinline__ float2 load2(const E* p, int n) {
  if (PAIR && n == 2) return Pack2<E>::up(*reinterpret_cast<const typename Pack2<E>::type*>(p));
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
      const Gate g = gate<false>(rv, iv, decay_rate(lam, p.c));
      h = fma(g.a, h, mul(mul(g.gain, g.si), xv));
      store_f32(state, n, h);
    }
    store2<E, PAIR>(static_cast<E*>(p.y) + b * p.y_stride + d, n, h);
  }
}

}  // namespace

int64_t recurrence_states(int64_t T) { return (T + kStateEvery - 1) / kStateEvery; }

// CTAs that share a row's time: doubled while the device (152 SMs, two CTAs each) has room and
// there are chunks to deal.
int recurrence_cluster(int64_t B, int64_t T, int64_t D) {
  const int64_t columns = B * ((D + kChannels - 1) / kChannels), chunks = (T + kChunk - 1) / kChunk;
  int c = 1;
  while (c < kMaxCluster && columns * c < 2 * 152 && 2 * c <= chunks) c *= 2;
  return c;
}

cudaError_t launch_recurrence_forward(RecurrenceParams p, int dtype, int unit, bool pair, cudaStream_t s) {
  const int cluster = recurrence_cluster(p.B, p.T, p.D);
  p.groups = (int32_t)((p.D + kChannels - 1) / kChannels);
  const unsigned grid = (unsigned)(p.B * p.groups * cluster);
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    if (unit == 16 && pair) return run_forward<E, 16, true>(p, grid, cluster, s);
    if constexpr (sizeof(E) == 2) {
      if (unit >= 4 && pair) return run_forward<E, 4, true>(p, grid, cluster, s);
      return run_forward<E, 2, false>(p, grid, cluster, s);
    } else {
      return run_forward<E, 4, false>(p, grid, cluster, s);
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
