// Backward pass of the gated linear recurrence.
//
// With the flow F_t = a_{t+1} g_{t+1} into token t from behind (dh_last past the end) and
// g_t = dy_t + F_t, F is the same kind of recurrence as h, walked from the end: F_{t-1} = a_t (F_t + dy_t).
// Per token, with K = sqrt(1 - a^2) sigmoid(i), b = K x and 1 - a^2 = sigmoid(r) X:
//   dx = g K,  di = g b (1 - sigmoid(i)),
//   m = a g (h_{t-1} rate sigmoid(r) - b a rate / X),   dr = -(1 - sigmoid(r)) m,
//   ddecay = -c sigmoid(lambda) / rate sum m.
// The rate stands inside m, where it meets the small sigmoid of a gate that keeps a fast decay's state
// alive; outside, m would be as small as that sigmoid and lose bits below the smallest numbers.
// h_{t-1} is recomputed in fp32 from the state at the start of the chunk, which the forward pass
// kept (4 bytes for kStateEvery tokens and channel), not read back from the rounded y.
//
// The cut of time over threads, warps and cluster CTAs is that of the forward pass, with runs of 8
// tokens: a token's five factors (a, sigmoid(r), K, b (1 - sigmoid(i)), b a rate / X) stay in registers from the
// first walk, which needs all transcendental functions, to the last, which writes.
//
// It has to move 7 elements a token and channel (and 4 bytes of state for 32 tokens); bf16 64x512x1024
// takes 85 us, 81 % of the copy rate, 16x2048x2048 176 us (79 %), 8x2048x2048 102 us (68 %), 1x65536x1024 251 us
// (55 %); fp32 8x2048x1024 80 us (87 %), 32x1024x1024 175 us (79 %).  What bounds it is latency: 12 to 14
// active warps of an SM issue 2.1 to 2.4 instructions a cycle, about 111 a token and pair of channels, 144 in
// clusters.  With 32 channels a CTA two runs of a warp share 16 banks (see the forward pass): shared memory is
// 55 % busy, 38 % with 64 channels.  Rates of 0.2 to 6: 16x2048x2048 191 us.
#include "recurrence.cuh"

namespace gs {
namespace {

using namespace rec;

constexpr int kLen = 8;                  // tokens of a run

template <typename E, int CH, bool OUT>
struct BackwardShared {
  static constexpr int kRuns = Tile<E, CH, kLen>::kRuns;
  Tile<E, CH, kLen> in[2][4];            // x, r, i, dy; the next step's are under way
  Tile<E, CH, OUT ? kLen : 0> out[3];    // dx, dr, di
  float4 run[kRuns][CH / 2];             // the map of h over each run
  float2 back[kRuns][CH / 2];            // the offset of the flow's map (its factor is the same)
  uint32_t cut[kRuns];
  uint64_t full[2];                      // a stage's tiles have come
};

// UNIT: how the inputs are moved (16: tiles; 4; 2).  OUT: results leave as tiles too.
template <typename E, int CH, int UNIT, bool OUT, bool RESET>
__global__ void __launch_bounds__(kThreads, 4)
k_recurrence_backward(const __grid_constant__ RecurrenceParams p) {
  constexpr bool TILES = UNIT == 16, PAIR = UNIT > (int)sizeof(E);  // results as pairs
  using Shared = BackwardShared<E, CH, OUT>;
  using Raw = typename Pack2<E>::type;
  constexpr int kRuns = Shared::kRuns, kChunk = kRuns * kLen;
  static_assert(kChunk % kStateEvery == 0, "a step starts at a kept state");
  extern __shared__ __align__(128) unsigned char raw[];
  Shared& sh = *reinterpret_cast<Shared*>(raw);
  begin_cluster((int)cg::this_cluster().num_blocks());
  const Place w = place<CH>(p);
  Table<CH>& table = *reinterpret_cast<Table<CH>*>(raw + sizeof(Shared));  // there with a cluster only
  const int steps = (int)(((w.len + kChunk - 1) / kChunk + w.cluster - 1) / w.cluster);
  const int64_t kept = (p.T + kStateEvery - 1) / kStateEvery;
  const int channels = clamp_int(p.D - w.d0, CH);
  const E* x = static_cast<const E*>(p.x.data) + w.b * p.x.batch + w.d0;
  const E* r = static_cast<const E*>(p.r.data) + w.b * p.r.batch + w.d0;
  const E* i = static_cast<const E*>(p.i.data) + w.b * p.i.batch + w.d0;
  const E* dy = static_cast<const E*>(p.dy.data) + w.b * p.dy.batch + w.d0;
  E* dx = static_cast<E*>(p.dx.data) + w.b * p.dx.batch + w.d;
  E* dr = static_cast<E*>(p.dr.data) + w.b * p.dr.batch + w.d;
  E* di = static_cast<E*>(p.di.data) + w.b * p.di.batch + w.d;
  auto chunk_token = [&](int s) { return ((int64_t)s * w.cluster + w.rank) * kChunk; };
  bool here = true, linked = true;  // no wait for tiles, for messages, has run out
  // step s is the turn-th from the end
  auto load = [&](int turn) {
    const int64_t t0 = chunk_token(steps - 1 - turn);
    auto& in = sh.in[turn & 1];
    if constexpr (TILES) {
      if (threadIdx.x == 0 && here) {
        uint64_t* bar = &sh.full[turn & 1];
        barrier_expect(bar, 4 * sizeof(in[0]));
        for (int k = 0; k < 4; ++k) tile_load(&in[k], &p.maps[kMapX + k], (int)w.d0, (int)t0, (int)w.b, bar);
      }
    } else {
      const int live = clamp_int(w.len - t0, kChunk);
      copy_tile<UNIT>(in[0], x, p.x.token, t0, live, channels);
      copy_tile<UNIT>(in[1], r, p.r.token, t0, live, channels);
      copy_tile<UNIT>(in[2], i, p.i.token, t0, live, channels);
      copy_tile<UNIT>(in[3], dy, p.dy.token, t0, live, channels);
      copy_commit();
    }
  };
  if (TILES && threadIdx.x == 0) {
    for (int k = 0; k < 2; ++k) barrier_init(&sh.full[k]);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tile_fence();
  }
  if (steps > 0) load(0);
  if (w.cluster > 1)
    open_table(table);
  else
    __syncthreads();
  const float2 rate = decay_rate(load_f32(p.decay + w.d, w.n), p.c);
  const bool series = rates_within(w, rate, kSeries);
  float2 flow = load_f32(p.dh_last ? p.dh_last + w.b * p.D + w.d : nullptr, w.n);
  float2 sum = two(0.f);
  uint8_t flag = RESET && steps > 0 ? reset_flag<kLen>(p, w, chunk_token(steps - 1) + w.slot * kLen) : 0;
  for (int s = steps - 1; s >= 0; --s) {
    const int64_t t0 = chunk_token(s) + w.slot * kLen;
    const bool full = chunk_token(s) + kChunk <= w.len;  // the chunk has no masked token
    uint32_t resets = RESET ? reset_bits<CH, kLen>(flag) : 0;
    if (RESET && s > 0) flag = reset_flag<kLen>(p, w, chunk_token(s - 1) + w.slot * kLen);
    const int64_t kept_at = chunk_token(s) / kStateEvery;
    float2 h = kept_at < kept ? load_f32(p.states + (w.b * kept + kept_at) * p.D + w.d, w.n) : two(0.f);
    const int turn = steps - 1 - s;
    if constexpr (TILES) {
      here = here && barrier_wait<false>(&sh.full[turn & 1], turn >> 1, p.tile_tries);
    } else {
      copy_wait<0>();
    }
    __syncthreads();  // the tiles are here, and those of the step before have been read
    if (s > 0) load(turn + 1);
    auto& tile = sh.in[turn & 1];
    float2 a[kLen], sr[kLen], K[kLen], U[kLen], Q[kLen];
    // 1 - sigmoid(r), for which no registers are left, stays where the thread has read its gates, in one
    // word of each tile with a 2-byte type.  kTurned: two runs of a warp, whose rows lie in the same banks,
    // do so in every other row the other way round (backward of 1x65536x1024 bf16 251 us, 259 without).
    constexpr bool kTurned = sizeof(E) == 2 && CH < 64;
    const int turned = kTurned ? w.slot % 2 * (CH / 2) : 0;
    auto word = [&](int which, int k) -> Raw& { return *(&tile[which].at(w, k) + (k % 2 == 0 ? turned : -turned)); };
    auto keep = [&](int k, float2 v) {
      if constexpr (sizeof(E) == 4) {
        tile[1].at(w, k) = v;
      } else {
        memcpy(&word(1, k), &v.x, sizeof(Raw));
        memcpy(&word(2, k), &v.y, sizeof(Raw));
      }
    };
    auto kept_value = [&](int k) {
      float2 v;
      if constexpr (sizeof(E) == 4) {
        v = tile[1].at(w, k);
      } else {
        memcpy(&v.x, &word(1, k), sizeof(Raw));
        memcpy(&v.y, &word(2, k), sizeof(Raw));
      }
      return v;
    };
    float2 last_shut = two(0.f);
    Run run = identity();
    // SOME: there may be masked tokens and resets.  Runs of whole chunks without a reset, nearly all
    // of them, do without the selections.
    auto gates = [&](auto some, auto in_series) {
      constexpr bool SOME = decltype(some)::value;
#pragma unroll
      for (int k = 0; k < kLen; ++k) {
        const bool cut = RESET && SOME && (resets >> k & 1u);
        const Gate g = gate_backward<decltype(in_series)::value>(capped<kMostBackward>(tile[1].at(w, k)),
                                                                    capped<kMostBackward>(tile[2].at(w, k)), rate, cut);
        a[k] = g.a;
        sr[k] = g.sr;
        if (!kTurned) keep(k, g.shut);
        if (kTurned && k % 2 == 1) {
          keep(k - 1, last_shut);
          keep(k, g.shut);
        }
        last_shut = g.shut;
        K[k] = g.K;
        float2 b = mul(g.K, widen(tile[0].at(w, k)));
        U[k] = mul(b, g.off);
        Q[k] = mul(b, mul(g.a, g.rate_X));
        if (SOME && t0 + k >= w.len) {  // past the end of the row: the state and the flow stay
          a[k] = two(1.f);
          K[k] = b = two(0.f);
        }
        run.a = mul(run.a, a[k]);
        run.b = RESET && SOME ? apply(Run{a[k], b}, cut, run.b) : fma(a[k], run.b, b);
      }
    };
    const bool plain = full && !(RESET && __any_sync(0xFFFFFFFFu, resets != 0));
    if (!plain)
      gates(std::true_type(), std::false_type());
    else if (series)
      gates(std::false_type(), std::true_type());
    else
      gates(std::false_type(), std::false_type());
    float2 back = two(0.f);
    auto flows = [&](auto some) {
#pragma unroll
      for (int k = kLen - 1; k >= 0; --k) {
        float2 d = widen(tile[3].at(w, k));
        if (decltype(some)::value && t0 + k >= w.len) d = two(0.f);
        const float2 f = mul(a[k], add(back, d));
        back = RESET && decltype(some)::value ? choose(resets >> k & 1u, two(0.f), f) : f;
      }
    };
    if (plain)
      flows(std::false_type());
    else
      flows(std::true_type());
    if (TILES && !here) {  // the run turns whatever state and flow into NaN
      run = Run{two(nanf("")), two(nanf(""))};
      back = two(nanf(""));
      resets = 0;
    }
    sh.run[w.slot][w.pair] = as_float4(run);
    sh.back[w.slot][w.pair] = back;
    if (RESET && w.pair == 0) sh.cut[w.slot] = resets;
    if (OUT && threadIdx.x == 0) store_wait();  // the step before's results have left
    __syncthreads();
    // the maps of the flow over the runs after this one, and over the whole chunk; the state
    // before this run
#pragma unroll
    for (int k = 0; k < kRuns - 1; ++k)
      if (k < w.slot) h = apply(as_run(sh.run[k][w.pair]), RESET && sh.cut[k] != 0, h);
    float2 f = flow;
    auto back_run = [&](int k) {
      Run m = as_run(sh.run[k][w.pair]);
      m.b = sh.back[k][w.pair];
      return m;
    };
    if (w.cluster > 1) {
      Run after, total = identity();
      bool after_cut, cut = false;
#pragma unroll
      for (int k = kRuns - 1; k >= 0; --k) {
        if (k == w.slot) {
          after = total;
          after_cut = cut;
        }
        extend(total, cut, back_run(k), RESET && sh.cut[k] != 0);
      }
      if (linked) {
        send<CH, kRuns>(table, turn & 1, w, total, RESET && cut);
        linked = barrier_wait<true>(&table.arrived[turn & 1], turn >> 1, p.message_tries);
      }
#pragma unroll 4
      for (int k = w.cluster - 1; k > w.rank; --k) flow = apply_total<RESET>(table, turn & 1, k, w, flow);
      f = apply(after, RESET && after_cut, flow);
#pragma unroll 4
      for (int k = w.rank; k >= 0; --k) flow = apply_total<RESET>(table, turn & 1, k, w, flow);
      if (!linked) {
        flow = two(nanf(""));
        f = apply(after, RESET && after_cut, flow);
      }
    } else {
#pragma unroll
      for (int k = kRuns - 1; k >= 0; --k) {
        if (k == w.slot) f = flow;
        flow = apply(back_run(k), RESET && sh.cut[k] != 0, flow);
      }
    }
    if (TILES && !here) f = two(nanf(""));
    auto states = [&](auto some) {
#pragma unroll
      for (int k = 0; k < kLen; ++k) {
        Q[k] = fma(h, mul(rate, sr[k]), make_float2(-Q[k].x, -Q[k].y));
        const float2 b = mul(K[k], widen(tile[0].at(w, k)));
        h = RESET && decltype(some)::value ? apply(Run{a[k], b}, resets >> k & 1u, h) : fma(a[k], h, b);
      }
    };
    if (plain)
      states(std::false_type());
    else
      states(std::true_type());
    float2 part = two(0.f);
    auto token = [&](bool some, int k, float2& ox, float2& orr, float2& oi) {
      const bool cut = RESET && some && (resets >> k & 1u);
      const float2 g = add(f, widen(tile[3].at(w, k)));
      f = choose(cut, two(0.f), mul(a[k], g));
      const float2 m = choose(cut, two(0.f), mul(f, Q[k]));
      part = add(part, m);
      ox = mul(g, K[k]);
      oi = mul(g, U[k]);
      orr = choose(cut, two(0.f), mul(kept_value(k), make_float2(-m.x, -m.y)));
    };
    if constexpr (OUT) {
      auto results = [&](auto some) {
#pragma unroll
        for (int k = kLen - 1; k >= 0; --k) {
          float2 ox = two(0.f), orr = two(0.f), oi = two(0.f);
          if (!decltype(some)::value || t0 + k < w.len) token(decltype(some)::value, k, ox, orr, oi);
          sh.out[0].at(w, k) = Pack2<E>::down(ox);
          sh.out[1].at(w, k) = Pack2<E>::down(orr);
          sh.out[2].at(w, k) = Pack2<E>::down(oi);
        }
      };
      if (plain)
        results(std::false_type());
      else
        results(std::true_type());
      tile_fence();
      __syncthreads();
      if (threadIdx.x == 0 && chunk_token(s) < p.T) {
        for (int k = 0; k < 3; ++k) tile_store(&sh.out[k], &p.maps[kMapDx + k], (int)w.d0, (int)chunk_token(s), (int)w.b);
        store_commit();
      }
    } else {
      E *out_x = dx + (t0 + kLen - 1) * p.dx.token, *out_r = dr + (t0 + kLen - 1) * p.dr.token,
        *out_i = di + (t0 + kLen - 1) * p.di.token;
      auto results = [&](auto some) {
#pragma unroll
        for (int k = kLen - 1; k >= 0; --k) {
          float2 ox = two(0.f), orr = two(0.f), oi = two(0.f);
          if (!decltype(some)::value || t0 + k < w.len) token(decltype(some)::value, k, ox, orr, oi);
          if (!decltype(some)::value || t0 + k < p.T) {
            store2<E, PAIR>(out_x, w.n, ox);
            store2<E, PAIR>(out_r, w.n, orr);
            store2<E, PAIR>(out_i, w.n, oi);
          }
          out_x -= p.dx.token;
          out_r -= p.dr.token;
          out_i -= p.di.token;
        }
      };
      if (plain)
        results(std::false_type());
      else
        results(std::true_type());
      if (TILES) tile_fence();  // the tiles, which the threads have written to, are loaded again
    }
    sum = add(sum, part);
  }
  // past the last step every token is masked
  for (int64_t t0 = chunk_token(steps); t0 < p.T; t0 += (int64_t)w.cluster * kChunk)
    for (int k = 0; k < kLen; ++k) {
      const int64_t t = t0 + w.slot * kLen + k;
      if (t < p.T) {
        store2<E, PAIR>(dx + t * p.dx.token, w.n, two(0.f));
        store2<E, PAIR>(dr + t * p.dr.token, w.n, two(0.f));
        store2<E, PAIR>(di + t * p.di.token, w.n, two(0.f));
      }
    }
  // no CTA leaves while another may still write to it, and all have read dh_last, which dh0 may be
  if (w.cluster > 1) cg::this_cluster().sync();
  if (!here || !linked) pause();
  if (p.dh0 && w.rank == 0 && w.slot == 0) store_f32(p.dh0 + w.b * p.D + w.d, w.n, flow);
  if (OUT && threadIdx.x == 0) store_wait();     // nor while its tiles are being read
  // the CTA's share of the decay's gradient, its runs in order
  __syncthreads();
  sh.back[w.slot][w.pair] = sum;
  __syncthreads();
  if (w.slot == 0) {
#pragma unroll
    for (int k = 1; k < kRuns; ++k) sum = add(sum, sh.back[k][w.pair]);
    store_f32(p.partial + (w.b * w.cluster + w.rank) * p.D + w.d, w.n, make_float2(sum.x / rate.x, sum.y / rate.y));
  }
}

template <typename E, int CH, int UNIT, bool OUT, bool RESET>
cudaError_t run_backward(RecurrenceParams& p, const RecurrenceShape& shape, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kernel = k_recurrence_backward<E, CH, UNIT, OUT, RESET>;
  constexpr size_t kBase = sizeof(BackwardShared<E, CH, OUT>), kTable = sizeof(Table<CH>);
  const cudaError_t e = prepare_kernel(kernel, kBase + kTable, done);
  if (e != cudaSuccess) return e;
  p.groups = shape.groups;
  const size_t smem = kBase + (shape.cluster > 1 ? kTable : 0);
  return launch_cluster(kernel, dim3(shape.grid), dim3(kThreads), smem, shape.cluster, s, p);
}

// Results leave as tiles where shared memory has room for them beside two stages of inputs at four
// CTAs an SM: with a 2-byte type.
template <typename E, int CH, int UNIT>
cudaError_t run_backward(RecurrenceParams& p, const RecurrenceShape& shape, cudaStream_t s) {
  constexpr bool OUT = UNIT == 16 && sizeof(E) == 2;
  return p.reset ? run_backward<E, CH, UNIT, OUT, true>(p, shape, s) : run_backward<E, CH, UNIT, OUT, false>(p, shape, s);
}

}  // namespace

// Rows of the workspace: one for each row of the batch and CTA of a cluster.
int64_t recurrence_partials(int64_t B, int64_t T, int64_t D) {
  const int a = recurrence_shape(B, T, D, kLen, true).cluster, b = recurrence_shape(B, T, D, kLen, false).cluster;
  return B * (a > b ? a : b);
}

cudaError_t launch_recurrence_backward(RecurrenceParams& p, float* ddecay, int dtype, int unit, cudaStream_t s) {
  const RecurrenceShape shape = recurrence_shape(p.B, p.T, p.D, kLen, dtype == GS_F32);
  if (unit == 16 && shape.grid > 0) {
    const int tokens = kThreads / (shape.channels / 2) * kLen;
    const Seq<const void*>* in[4] = {&p.x, &p.r, &p.i, &p.dy};
    const Seq<void*>* out[3] = {&p.dx, &p.dr, &p.di};
    bool all = true;
    for (int k = 0; k < 4; ++k) all = all && describe(p.maps[kMapX + k], *in[k], p, dtype, shape.channels, tokens);
    if (dtype != GS_F32)  // whose results are stored from registers
      for (int k = 0; k < 3; ++k) all = all && describe(p.maps[kMapDx + k], *out[k], p, dtype, shape.channels, tokens);
    if (!all) unit = 4;
  }
  cudaError_t err = shape.grid == 0 ? cudaSuccess : with_type(dtype, [&](auto e) {
    using E = decltype(e);
    return with_cut(shape, unit, [&](auto channels, auto copies) {
      constexpr int CH = decltype(channels)::value, UNIT = decltype(copies)::value;
      if constexpr (UNIT == 2 && sizeof(E) == 4)
        return cudaErrorInvalidValue;
      else
        return run_backward<E, CH, UNIT>(p, shape, s);
    });
  });
  if (err != cudaSuccess) return err;
  return launch_column_sums(p.partial, p.B * shape.cluster, p.D, p.decay, p.c, ddecay, s);
}

}  // namespace gs
