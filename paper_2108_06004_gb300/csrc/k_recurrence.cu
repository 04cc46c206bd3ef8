// Forward pass of the gated linear recurrence over time, and its single-token step.
//
//   log a_t = -c softplus(lambda) sigmoid(r_t),   v_t = 1 - a_t^2,
//   h_t = a_t h_{t-1} + sqrt(v_t) sigmoid(i_t) x_t,   y_t = h_t      (at a reset a_t = 0)
//
// A run of tokens acts on the state as h -> A h + B with A the product of its a_t, and such maps
// compose, so time is cut three times: a thread owns kLen tokens of two channels, a CTA owns adjacent
// runs (a chunk), and where the rows and channels alone do not fill the device a cluster of CTAs
// owns adjacent chunks.  Each thread works out (A, B) of its run; the runs' maps are exchanged in
// shared memory and the chunks' in distributed shared memory; then the run is walked again from
// its true starting state.  Every tensor is read from and written to memory once, nothing waits for
// another cluster, and the order of all operations is fixed by the sizes.  For the backward pass the
// state is kept in fp32 every kStateEvery tokens.
//
// It has to move 4 elements a token and channel.  bf16 64x512x1024 takes 48 us (83 % of the copy rate),
// 16x2048x2048 100 us (79 %), 8x2048x2048 56 us (71 %: 512 CTAs, four on some SMs and three on others),
// 1x65536x1024 135 us (59 %: the same, and a meeting of 16 CTAs at every step); fp32 32x1024x1024
// 85 us (93 %).  What bounds it in bf16 is latency: 11 to 14 warps of an SM are active on average, and they
// issue 2.0 to 2.2 instructions a cycle of the 4 that it could, about 61 a token and pair of channels and 74
// in clusters; the busiest pipe is at 32 %.  With 32 channels a CTA a warp holds two runs whose rows lie in the same 16
// banks, so every tile access takes two turns (shared memory 34 % busy, 16 % with 64 channels).  Runs of 16
// tokens and 128 registers do better than runs of 8 and 24 warps (1x65536x1024: 226 us), which meet twice as
// often.  Decay rates above 1/2 leave the polynomial: 16x2048x2048 with rates of 0.2 to 6 takes 116 us.
#include "recurrence.cuh"

namespace gs {
namespace {

using namespace rec;

constexpr int kLen = 16;                 // tokens of a run

template <typename E, int CH, int STAGES>
struct ForwardShared {
  static constexpr int kRuns = Tile<E, CH, kLen>::kRuns;
  Tile<E, CH, kLen> in[STAGES][3];       // x, r, i
  float4 run[kRuns][CH / 2];             // the map of each run
  uint32_t cut[kRuns];
  uint64_t full[STAGES];                 // a stage's tiles have come
};

// UNIT: how the inputs are moved (16: tiles; 4; 2).  STAGES: steps whose inputs fit in shared memory.
template <typename E, int CH, int UNIT, int STAGES, bool RESET>
__global__ void __launch_bounds__(kThreads, 4)
k_recurrence_forward(const __grid_constant__ RecurrenceParams p) {
  constexpr bool TILES = UNIT == 16, PAIR = UNIT > (int)sizeof(E);  // results as pairs
  using Shared = ForwardShared<E, CH, STAGES>;
  using Raw = typename Pack2<E>::type;
  constexpr int kRuns = Shared::kRuns, kChunk = kRuns * kLen;
  extern __shared__ __align__(128) unsigned char raw[];
  Shared& sh = *reinterpret_cast<Shared*>(raw);
  begin_cluster((int)cg::this_cluster().num_blocks());
  const Place w = place<CH>(p);
  Table<CH>& table = *reinterpret_cast<Table<CH>*>(raw + sizeof(Shared));  // there with a cluster only
  const int64_t chunks = (w.len + kChunk - 1) / kChunk;
  const int steps = (int)((chunks + w.cluster - 1) / w.cluster);
  const int64_t kept = (p.T + kStateEvery - 1) / kStateEvery;
  const int channels = clamp_int(p.D - w.d0, CH);
  const E* x = static_cast<const E*>(p.x.data) + w.b * p.x.batch + w.d0;
  const E* r = static_cast<const E*>(p.r.data) + w.b * p.r.batch + w.d0;
  const E* i = static_cast<const E*>(p.i.data) + w.b * p.i.batch + w.d0;
  E* y = static_cast<E*>(p.y.data) + w.b * p.y.batch + w.d;
  auto chunk_token = [&](int s) { return ((int64_t)s * w.cluster + w.rank) * kChunk; };
  bool here = true, linked = true;  // no wait for tiles, for messages, has run out
  auto load = [&](int s) {
    if (s >= steps) return;
    const int64_t t0 = chunk_token(s);
    auto& in = sh.in[s % STAGES];
    if constexpr (TILES) {
      if (threadIdx.x == 0 && here) {
        uint64_t* bar = &sh.full[s % STAGES];
        barrier_expect(bar, 3 * sizeof(in[0]));
        for (int k = 0; k < 3; ++k) tile_load(&in[k], &p.maps[kMapX + k], (int)w.d0, (int)t0, (int)w.b, bar);
      }
    } else {
      const int live = clamp_int(w.len - t0, kChunk);
      copy_tile<UNIT>(in[0], x, p.x.token, t0, live, channels);
      copy_tile<UNIT>(in[1], r, p.r.token, t0, live, channels);
      copy_tile<UNIT>(in[2], i, p.i.token, t0, live, channels);
    }
    copy_commit();
  };
  if (TILES && threadIdx.x == 0) {
    for (int k = 0; k < STAGES; ++k) barrier_init(&sh.full[k]);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tile_fence();
  }
  for (int s = 0; s < STAGES; ++s) load(s);
  if (w.cluster > 1)
    open_table(table);
  else
    __syncthreads();
  const float2 rate = decay_rate(load_f32(p.decay + w.d, w.n), p.c);
  const bool slow = rates_within(w, rate, kSeries), medium = rates_within(w, rate, kModerate);
  float2 state = load_f32(p.h0 ? p.h0 + w.b * p.D + w.d : nullptr, w.n);
  uint8_t flag = RESET ? reset_flag<kLen>(p, w, chunk_token(0) + w.slot * kLen) : 0;
  for (int s = 0; s < steps; ++s) {
    const int64_t t0 = chunk_token(s) + w.slot * kLen;
    const bool full = chunk_token(s) + kChunk <= w.len;  // the chunk has no masked token
    uint32_t resets = RESET ? reset_bits<CH, kLen>(flag) : 0;
    if (RESET) flag = reset_flag<kLen>(p, w, chunk_token(s + 1) + w.slot * kLen);
    if constexpr (TILES) {
      here = here && barrier_wait<false>(&sh.full[s % STAGES], s / STAGES, p.tile_tries);
    } else {
      if (s + 1 < steps)
        copy_wait<STAGES - 1>();
      else
        copy_wait<0>();
    }
    // the tiles are here; the tables of the step before have been read
    __syncthreads();
    auto& tile = sh.in[s % STAGES];
    // the run's tokens as a_t and b_t, and their composition
    float2 a[kLen], b[kLen];
    Run run = identity();
    // SOME: there may be masked tokens and resets.  Runs of whole chunks without a reset, nearly all
    // of them, do without the selections.
    auto gates = [&](auto some, auto rates) {
      constexpr bool SOME = decltype(some)::value;
#pragma unroll
      for (int k = 0; k < kLen; ++k) {
        const bool cut = RESET && SOME && (resets >> k & 1u);
        float2 K;
        gate_forward<decltype(rates)::value>(capped<kMostForward>(tile[1].at(w, k)), capped<kMostForward>(tile[2].at(w, k)), rate, cut, a[k], K);
        b[k] = mul(K, widen(tile[0].at(w, k)));
        if (SOME && t0 + k >= w.len) {  // past the end of the row: the state stays
          a[k] = two(1.f);
          b[k] = two(0.f);
        }
        run.a = mul(run.a, a[k]);
        run.b = RESET && SOME ? apply(Run{a[k], b[k]}, cut, run.b) : fma(a[k], run.b, b[k]);
      }
    };
    const bool plain = full && !(RESET && __any_sync(0xFFFFFFFFu, resets != 0));
    if (!plain || !medium)
      gates(std::true_type(), std::integral_constant<int, kAny>());
    else if (slow)
      gates(std::false_type(), std::integral_constant<int, kSlow>());
    else
      gates(std::false_type(), std::integral_constant<int, kMedium>());
    if (TILES && !here) {  // the run turns whatever state into NaN
      run = Run{two(nanf("")), two(nanf(""))};
      resets = 0;
    }
    sh.run[w.slot][w.pair] = as_float4(run);
    if (RESET && w.pair == 0) sh.cut[w.slot] = resets;
    __syncthreads();
    load(s + STAGES);  // this step's tiles have been read
    // the state at the start of the run, and at the end of the step
    float2 h = state;
    if (w.cluster > 1) {
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
      if (linked) {
        send<CH, kRuns>(table, s & 1, w, total, RESET && cut);
        linked = barrier_wait<true>(&table.arrived[s & 1], s >> 1, p.message_tries);
      }
#pragma unroll 4
      for (int k = 0; k < w.rank; ++k) state = apply_total<RESET>(table, s & 1, k, w, state);
      h = apply(before, RESET && before_cut, state);
#pragma unroll 4
      for (int k = w.rank; k < w.cluster; ++k) state = apply_total<RESET>(table, s & 1, k, w, state);
      if (!linked) {
        state = two(nanf(""));
        h = apply(before, RESET && before_cut, state);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kRuns; ++k) {
        if (k == w.slot) h = state;
        state = apply(as_run(sh.run[k][w.pair]), RESET && sh.cut[k] != 0, state);
      }
    }
    if (TILES && !here) h = two(nanf(""));
    if (p.states && t0 % kStateEvery == 0 && t0 / kStateEvery < kept)
      store_f32(p.states + (w.b * kept + t0 / kStateEvery) * p.D + w.d, w.n, h);
    E* out = y + t0 * p.y.token;
    if (plain && PAIR && w.n == 2) {
#pragma unroll
      for (int k = 0; k < kLen; ++k) {
        h = fma(a[k], h, b[k]);
        *reinterpret_cast<Raw*>(out) = Pack2<E>::down(h);
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
  // no CTA leaves while another may still write to it, and all have read h0, which h_last may be
  if (w.cluster > 1) cg::this_cluster().sync();
  if (!here || !linked) pause();
  if (p.h_last && w.rank == 0 && w.slot == 0) store_f32(p.h_last + w.b * p.D + w.d, w.n, state);
}

template <typename E, int CH, int UNIT, int STAGES, bool RESET>
cudaError_t run_forward(RecurrenceParams& p, const RecurrenceShape& shape, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kernel = k_recurrence_forward<E, CH, UNIT, STAGES, RESET>;
  constexpr size_t kBase = sizeof(ForwardShared<E, CH, STAGES>), kTable = sizeof(Table<CH>);
  const cudaError_t e = prepare_kernel(kernel, kBase + kTable, done);
  if (e != cudaSuccess) return e;
  p.groups = shape.groups;
  const size_t smem = kBase + (shape.cluster > 1 ? kTable : 0);
  return launch_cluster(kernel, dim3(shape.grid), dim3(kThreads), smem, shape.cluster, s, p);
}

// Two stages where four CTAs an SM still have room for them: a 2-byte type, and no table of the
// cluster's maps.
template <typename E, int CH, int UNIT>
cudaError_t run_forward(RecurrenceParams& p, const RecurrenceShape& shape, cudaStream_t s) {
  if constexpr (sizeof(E) == 2 && UNIT == 16)
    if (shape.cluster == 1)
      return p.reset ? run_forward<E, CH, UNIT, 2, true>(p, shape, s) : run_forward<E, CH, UNIT, 2, false>(p, shape, s);
  return p.reset ? run_forward<E, CH, UNIT, 1, true>(p, shape, s) : run_forward<E, CH, UNIT, 1, false>(p, shape, s);
}

// Two adjacent channels of one token, zero where they do not exist.  PAIR: both exist or neither.
template <typename E, bool PAIR>
__device__ __forceinline__ float2 load2(const E* p, int n) {
  if (PAIR) return n > 0 ? widen(*reinterpret_cast<const typename Pack2<E>::type*>(p)) : two(0.f);
  return make_float2(n > 0 ? to_f32(p[0]) : 0.f, n > 1 ? to_f32(p[1]) : 0.f);
}

// One token of each of p.B rows.  A thread owns two channels of `rows` rows, so that a channel's rate is
// worked out once for them, and loads kAhead rows at a time.  In a graph 1x1024 bf16 takes 1.8 us, all of
// it latency, and 256x4096 6.3 us (9.5 us with one row a thread; 6.8 with four at a time, 7.3 with one and
// 4864 CTAs; 2.3 us at the copy rate: ramp and latency).
constexpr int kStepThreads = 128, kAhead = 2;

template <typename E, bool PAIR>
__global__ void __launch_bounds__(kStepThreads)
k_recurrence_step(const __grid_constant__ RecurrenceStepParams p, int64_t rows) {
  grid_begin();
  const int64_t d = 2 * ((int64_t)blockIdx.x * kStepThreads + threadIdx.x);
  const int n = (int)(p.D - d < 0 ? 0 : p.D - d < 2 ? p.D - d : 2);
  if (n == 0) return;
  const float2 lam = load_f32(p.decay + d, n);
  const int64_t b0 = (int64_t)blockIdx.y * rows, b1 = b0 + rows < p.B ? b0 + rows : p.B;
  float2 rate = two(0.f);
  for (int64_t b = b0; b < b1; b += kAhead) {
    // loads without a branch in between: a row past the end reads the last one, an idle one its own
    int64_t slot[kAhead];
    float2 x[kAhead], r[kAhead], i[kAhead], h[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t row = b + k < b1 ? b + k : b1 - 1;
      slot[k] = p.slots ? p.slots[row] : row;
      x[k] = load2<E, PAIR>(static_cast<const E*>(p.x) + row * p.x_stride + d, n);
      r[k] = load2<E, PAIR>(static_cast<const E*>(p.r) + row * p.r_stride + d, n);
      i[k] = load2<E, PAIR>(static_cast<const E*>(p.i) + row * p.i_stride + d, n);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const bool live = slot[k] >= 0 && slot[k] < p.n_slots;
      h[k] = load2<float, PAIR>(p.state + slot[k] * p.state_stride + d, live ? n : 0);
    }
    if (b == b0) rate = decay_rate(lam, p.c);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (b + k >= b1) break;
      if (slot[k] >= 0 && slot[k] < p.n_slots) {
        float2 a, K;
        gate_forward<kAny>(capped<kMostForward>(r[k]), capped<kMostForward>(i[k]), rate, false, a, K);
        h[k] = fma(a, h[k], mul(K, x[k]));
        store2<float, PAIR>(p.state + slot[k] * p.state_stride + d, n, h[k]);
      }
      store2<E, PAIR>(static_cast<E*>(p.y) + (b + k) * p.y_stride + d, n, h[k]);
    }
  }
}

}  // namespace

int64_t recurrence_states(int64_t T) { return (T + kStateEvery - 1) / kStateEvery; }

// How a pass of `run` tokens a thread is cut: the channels of a CTA, and the CTAs of a cluster that
// share a row's time.  An SM holds four CTAs, three with fp32.  64 channels a CTA where that makes three for each
// SM; fewer columns are cut to 32 channels (twice the CTAs, with twice the tokens each: forward and
// backward of 8x2048x2048 bf16 took 56 and 96 us against 56 and 109 us with 64, but 64x512x1024,
// which has enough columns, 56 and 104 against 53 and 91 us, all when the cut was chosen), and then share time in clusters until
// there are three CTAs for each SM or no chunks left to deal.  A cluster meets at every step, so it comes last:
// 8x2048x2048 with 64 channels and clusters of two takes 58 and 134 us.  More CTAs than stay
// resident are no use (fp32 4x2048x2048: 256 CTAs 48 and 86 us, 512 in clusters of two 57 and
// 103 us).  The cut goes by sizes and type alone, so that results do not depend on alignment.
RecurrenceShape recurrence_shape(int64_t B, int64_t T, int64_t D, int run, bool fp32) {
  constexpr int64_t kEnough = 3 * kSMs;
  const int64_t resident = (fp32 ? 3 : 4) * kSMs;
  RecurrenceShape c = {};
  c.channels = B * ((D + 63) / 64) < kEnough ? 32 : 64;
  c.groups = (int32_t)((D + c.channels - 1) / c.channels);
  const int64_t columns = B * c.groups, chunk = kThreads / (c.channels / 2) * run;
  c.cluster = 1;
  while (c.cluster < kMaxCluster && columns * c.cluster < kEnough && columns * c.cluster * 2 <= resident &&
         2 * c.cluster * chunk <= T)
    c.cluster *= 2;
  c.grid = (unsigned)(columns * c.cluster);
  return c;
}

cudaError_t launch_recurrence_forward(RecurrenceParams& p, int dtype, int unit, cudaStream_t s) {
  const RecurrenceShape shape = recurrence_shape(p.B, p.T, p.D, kLen, dtype == GS_F32);
  if (unit == 16) {
    const int tokens = kThreads / (shape.channels / 2) * kLen;
    if (!describe(p.maps[kMapX], p.x, p, dtype, shape.channels, tokens) ||
        !describe(p.maps[kMapR], p.r, p, dtype, shape.channels, tokens) ||
        !describe(p.maps[kMapI], p.i, p, dtype, shape.channels, tokens))
      unit = 4;
  }
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return with_cut(shape, unit, [&](auto channels, auto copies) {
      constexpr int CH = decltype(channels)::value, UNIT = decltype(copies)::value;
      if constexpr (UNIT == 2 && sizeof(E) == 4)
        return cudaErrorInvalidValue;
      else
        return run_forward<E, CH, UNIT>(p, shape, s);
    });
  });
}

cudaError_t launch_recurrence_step(const RecurrenceStepParams& p, int dtype, bool pair, cudaStream_t s) {
  const int64_t columns = (p.D + 2 * kStepThreads - 1) / (2 * kStepThreads);
  // about as many CTAs as stay resident, and no more than a grid has rows
  int64_t rows = (p.B * columns + 24 * kSMs - 1) / (24 * kSMs);
  if (rows < (p.B + 65534) / 65535) rows = (p.B + 65534) / 65535;
  const dim3 grid((unsigned)columns, (unsigned)((p.B + rows - 1) / rows));
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return pair ? launch(k_recurrence_step<E, true>, grid, dim3(kStepThreads), s, p, rows)
                : launch(k_recurrence_step<E, false>, grid, dim3(kStepThreads), s, p, rows);
  });
}

}  // namespace gs
