// Shared pieces of the gated linear recurrence's kernels: the gates' arithmetic, the maps of runs
// of tokens, tile loads, and the exchange of maps over a cluster.
#pragma once

#include <cooperative_groups.h>

#include <cudaTypedefs.h>

#include <atomic>

#include "gs_layer.cuh"

namespace gs {
namespace rec {

namespace cg = cooperative_groups;

constexpr int kThreads = 128;
constexpr int kStateEvery = 32;          // tokens between the states kept for the backward pass
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

// Two adjacent elements in fp32.
__device__ __forceinline__ float2 widen(float2 v) { return v; }
__device__ __forceinline__ float2 widen(__half2 v) { return Pack2<__half>::up(v); }
__device__ __forceinline__ float2 widen(__nv_bfloat162 v) { return Pack2<__nv_bfloat16>::up(v); }

// A gate's value, capped where its sigmoid has long been 1 in fp32, so that no square of an exponential
// below overflows: 27 in the forward pass, 80 in the backward pass, which needs 1 - sigmoid too and has
// it right up to there.  The cap is exact in every type and taken before widening, two elements at once.
constexpr int kMostForward = 27, kMostBackward = 80;

template <int MOST>
__device__ __forceinline__ float2 capped(float2 v) {
  return make_float2(at_most(v.x, MOST), at_most(v.y, MOST));
}
template <int MOST>
__device__ __forceinline__ float2 capped(__half2 v) { return widen(__hmin2_nan(v, __float2half2_rn(MOST))); }
template <int MOST>
__device__ __forceinline__ float2 capped(__nv_bfloat162 v) { return widen(__hmin2_nan(v, __float2bfloat162_rn(MOST))); }

// Two channels at a time: one instruction for both.
__device__ __forceinline__ float2 two(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 add(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 fmac(float2 a, float2 b, float c) { return __ffma2_rn(a, b, two(c)); }
__device__ __forceinline__ float2 mulc(float2 a, float c) { return __fmul2_rn(a, two(c)); }
__device__ __forceinline__ float2 addc(float2 a, float c) { return __fadd2_rn(a, two(c)); }
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 choose(bool c, float2 a, float2 b) { return make_float2(c ? a.x : b.x, c ? a.y : b.y); }

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSeries = 0.5f;     // the series serves -q up to here
constexpr float kModerate = 0x1p40f;  // rates for which one root serves all of K

// What is known of a warp's rates.
enum Rates { kSlow, kMedium, kAny };  // at most kSeries, at most kModerate, at most 2^100

// softplus without overflow; for very negative arguments it is exp(x) and goes to zero.
__device__ __forceinline__ float softplus(float x) { return x > 20.f ? x : log1pf(expf(x)); }

// c softplus(lambda), kept from underflowing so that rsqrt(X) below stays finite, and below 2^100 so
// that X and its products do.
__device__ __forceinline__ float decay_rate(float lam, float c) {
  return fminf(fmaxf(c * softplus(lam), 1e-37f), 0x1p100f);
}
__device__ __forceinline__ float2 decay_rate(float2 lam, float c) {
  return make_float2(decay_rate(lam.x, c), decay_rate(lam.y, c));
}

// What a token's gates give, with rate = c softplus(lambda) and q = log a = -rate sigmoid(r):
//   sigmoid(r) = p^2 / (1 + p^2), p = e^(r/2), and i alike;  z = sqrt(sigmoid(r)) = p / sqrt(1 + p^2);
//   a = 1 + q s,  s = (e^q - 1) / q,  1 - a^2 = (1 - a)(1 + a) = sigmoid(r) X,  X = rate s (1 + a);
//   K = sqrt(1 - a^2) sigmoid(i).
// Halving the exponents keeps both gates, and the root of the first, exact to a few roundings down
// to the smallest numbers.  1 - a is never taken as a difference where it is small: for q >= -1/2
// s is the polynomial of degree 4 through its values at the five Chebyshev points (relative error
// below 9e-8), and a = 1 + q s is then off by half a rounding, where the exponential's own bias
// would add up over the thousands of tokens that a state lives.  X is about 2 rate even where the
// gate is shut, so nothing here is 0/0.

// SERIES: rate is at most kSeries in both channels, so q always is in the polynomial's range.  SMALL: a
// keeps its value below the smallest normal number too, as the square of half the exponent's power.
template <bool SERIES, bool SMALL>
__device__ __forceinline__ void decay_of(float2 sr, float2 rate, float2& a, float2& X) {
  const float2 q = mul(make_float2(-rate.x, -rate.y), sr);
  float2 s = addc(mulc(q, 0.006782862555491099f), 0.041013210491015605f);
  s = fmac(q, s, 0.16655192765429086f);
  s = fmac(q, s, 0.4999928833780279f);
  s = fmac(q, s, 0.999999928937559f);
  a = fmac(q, s, 1.f);
  if (!SERIES) {
    const auto power = [](float q) {
      if (!SMALL) return ex2(kLog2e * q);
      const float root = ex2(0.5f * kLog2e * q);
      return root * root;
    };
    if (q.x < -kSeries) {
      a.x = power(q.x);
      s.x = (1.f - a.x) * rcp(-q.x);
    }
    if (q.y < -kSeries) {
      a.y = power(q.y);
      s.y = (1.f - a.y) * rcp(-q.y);
    }
  }
  X = mul(mul(rate, s), addc(a, 1.f));
}

__device__ __forceinline__ float2 half_exp(float2 v) {
  const float2 h = mulc(v, 0.5f * kLog2e);
  return make_float2(ex2(h.x), ex2(h.y));
}
__device__ __forceinline__ float2 rcp(float2 v) { return make_float2(rcp(v.x), rcp(v.y)); }
__device__ __forceinline__ float2 rsq(float2 v) { return make_float2(rsq(v.x), rsq(v.y)); }

// a and K, from capped gate values.  The three roots and quotients of K are one reciprocal root.  X is at
// most twice the rate, and large only where sigmoid(r) is small and 1 + p^2 then about 1, so that with the
// cap the root's argument stays below 2^120 for rates up to kModerate.  For larger ones X with 1 + p^2 has
// a root of its own (16x2048x2048 bf16 with rates of 0.2 to 6 takes 128 us that way, 116 the other).
// `cut`: a reset, a = 0 and K = sigmoid(i).
template <int RATES>
__device__ __forceinline__ void gate_forward(float2 r, float2 i, float2 rate, bool cut, float2& a, float2& K) {
  const float2 pr = half_exp(r), pi = half_exp(i);
  const float2 sqr = mul(pr, pr), sqi = mul(pi, pi);
  const float2 ur = addc(sqr, 1.f), ui = addc(sqi, 1.f);
  float2 X;
  decay_of<RATES == kSlow, false>(mul(sqr, rcp(ur)), rate, a, X);
  if (RATES != kAny) {
    K = mul(mul(mul(pr, sqi), X), rsq(mul(mul(ur, ui), mul(ui, X))));
    if (cut) K = mul(sqi, rcp(ui));
  } else {
    const float2 si = mul(sqi, rcp(ui));
    K = choose(cut, si, mul(mul(pr, mul(X, rsq(mul(ur, X)))), si));
  }
  if (cut) a = two(0.f);
}

// What the backward pass needs.  The differences from 1 are not taken as such, which would leave them no
// digits from gate values of 17 on.
struct Gate {
  float2 sr, shut;  // sigmoid(r), 1 - sigmoid(r)
  float2 a, K;
  float2 off;       // 1 - sigmoid(i)
  float2 rate_X;    // rate / X
};
template <bool SERIES>
__device__ __forceinline__ Gate gate_backward(float2 r, float2 i, float2 rate, bool cut) {
  Gate g;
  const float2 one = two(1.f);
  const float2 pr = half_exp(r), pi = half_exp(i);
  const float2 w = rsq(fma(pr, pr, one)), z = mul(pr, w), sr = mul(z, z), sqi = mul(pi, pi);
  g.off = rcp(add(sqi, one));
  g.sr = sr;
  g.shut = mul(w, w);
  float2 X;
  decay_of<SERIES, true>(sr, rate, g.a, X);
  const float2 si = mul(sqi, g.off), rx = rsq(X);
  g.rate_X = mul(mul(rx, rx), rate);
  g.K = mul(mul(mul(z, X), rx), si);
  if (cut) {
    g.a = two(0.f);
    g.K = si;
  }
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
// The CTA owns CH channels and kThreads / (CH / 2) runs of tokens.
struct Place {
  int64_t b, d0, d;      // row, first channel of the CTA, first channel of the thread
  int n;                 // the thread's channels that exist, 0 ... 2
  int pair, slot;
  int rank, cluster;
  int64_t len;           // tokens of the row
};

template <int CH>
__device__ __forceinline__ Place place(const RecurrenceParams& p) {
  Place w;
  w.cluster = (int)cg::this_cluster().num_blocks();
  w.rank = (int)cg::this_cluster().block_rank();
  const unsigned column = blockIdx.x / (unsigned)w.cluster;
  w.b = column / (unsigned)p.groups;
  w.pair = threadIdx.x % (CH / 2);
  w.slot = threadIdx.x / (CH / 2);
  w.d0 = (int64_t)(column - (unsigned)w.b * (unsigned)p.groups) * CH;
  w.d = w.d0 + 2 * w.pair;
  w.n = (int)(p.D - w.d < 0 ? 0 : p.D - w.d < 2 ? p.D - w.d : 2);
  w.len = p.T;
  if (p.lengths) {
    const int64_t l = p.lengths[w.b];
    w.len = l < 0 ? 0 : l < p.T ? l : p.T;
  }
  return w;
}

// Whether the rates of all channels of the warp are at most `most`.
__device__ __forceinline__ bool rates_within(const Place& w, float2 rate, float most) {
  return __all_sync(0xFFFFFFFFu, (w.n < 1 || rate.x <= most) && (w.n < 2 || rate.y <= most));
}

__device__ __forceinline__ int clamp_int(int64_t v, int most) { return v < 0 ? 0 : v < most ? (int)v : most; }

// Resets among the LEN tokens of a run from t0 on, one bit each.  The first LEN lanes that work on
// the run read one flag each, ahead of time; the warp collects them.
template <int LEN>
__device__ __forceinline__ uint8_t reset_flag(const RecurrenceParams& p, const Place& w, int64_t t0) {
  return w.pair < LEN && t0 + w.pair < w.len ? p.reset[w.b * p.T + t0 + w.pair] : 0;
}
template <int CH, int LEN>
__device__ __forceinline__ uint32_t reset_bits(uint8_t flag) {
  const uint32_t all = __ballot_sync(0xFFFFFFFFu, flag != 0);
  constexpr int kLanes = CH / 2 < 32 ? CH / 2 : 32;
  return (all >> (threadIdx.x & 31) / kLanes * kLanes) & ((1u << LEN) - 1);
}

// ---- tile loads -----------------------------------------------------------------------------
// A tile holds CH channels of kThreads / (CH / 2) runs of LEN tokens in shared memory.  The tiles of
// tensors whose rows start at multiples of 16 bytes (UNIT 16) are moved by the tensor memory
// accelerator, one instruction a tile and no address arithmetic in the threads (with 16-byte copies
// by each thread instead, the forward pass issues an eighth more instructions, and it is bound by
// those); tokens and channels past a tensor's end read as zero and are not written.  Others are
// copied 4 bytes at a time asynchronously, or by single 2-byte elements through registers where
// rows of a 2-byte type start at odd elements, and their results stored from registers.
template <typename E, int CH, int LEN>
struct Tile {
  static constexpr int kRuns = kThreads / (CH / 2);
  static constexpr int kTokens = kRuns * LEN;
  using Raw = typename Pack2<E>::type;
  E v[LEN ? kTokens * CH : 8];
  __device__ __forceinline__ Raw& at(const Place& w, int k) {
    return reinterpret_cast<Raw*>(v + (w.slot * LEN + k) * CH)[w.pair];
  }
};

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint64_t* bar) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(bar)) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_address(bar)), "r"(bytes) : "memory");
}
// Whether the barrier's `phase`-th phase has come to its end.  Every wait is bounded: a try is suspended
// for a microsecond at most, so kMostTries take about a second.  A wait that runs out, which nothing
// that these kernels do can cause, is the thread's last of its kind.  Without its tiles a thread
// publishes and stores NaN, and thread 0 loads no more of them.  Without its messages its state is
// NaN, and it sends no more, so that no half of a table is written before it has been read.  Either
// way nothing that has not come gets into a result.  CLUSTER: other CTAs of the cluster write what the phase stands for, so
// the wait has to acquire at their scope; for the CTA's own tiles its own is enough.
template <bool CLUSTER>
__device__ __forceinline__ bool barrier_wait(uint64_t* bar, int phase, int tries) {
  for (; tries > 0; --tries) {
    uint32_t done;
    if (CLUSTER)
      asm volatile(
          "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, 1000;\n selp.u32 %0, 1, 0, p;\n}"
          : "=r"(done)
          : "r"(shared_address(bar)), "r"(phase & 1)
          : "memory");
    else
      asm volatile(
          "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2, 1000;\n selp.u32 %0, 1, 0, p;\n}"
          : "=r"(done)
          : "r"(shared_address(bar)), "r"(phase & 1)
          : "memory");
    if (done) return true;
  }
  return false;
}

__device__ __forceinline__ void tile_load(void* to, const CUtensorMap* map, int d, int t, int b, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          shared_address(to)),
      "l"(map), "r"(d), "r"(t), "r"(b), "r"(shared_address(bar))
      : "memory");
}
__device__ __forceinline__ void tile_store(const void* from, const CUtensorMap* map, int d, int t, int b) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(d), "r"(t),
               "r"(b), "r"(shared_address(from))
               : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// All stores of this thread have read their tiles.
__device__ __forceinline__ void store_wait() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
// What this thread has written to shared memory is seen by tile stores that are issued after.
__device__ __forceinline__ void tile_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void copy_async(void* to, const void* from, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(shared_address(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// Tokens t0 ... t0 + live - 1 of the CTA's channels, of which `channels` exist; zeros for the rest.
template <int UNIT, typename E, int CH, int LEN>
__device__ __forceinline__ void copy_tile(Tile<E, CH, LEN>& tile, const E* from, int64_t token_stride, int64_t t0,
                                          int live, int channels) {
  using Shape = Tile<E, CH, LEN>;
  constexpr int PER = UNIT / (int)sizeof(E);      // elements of a copy
  constexpr int U = CH / PER;                     // copies of a token
  constexpr int R = kThreads / U;                 // tokens at a time
  constexpr int N = Shape::kTokens / R;
  const int u = threadIdx.x % U, row = threadIdx.x / U;
  const E* src = from + (t0 + row) * token_stride + u * PER;
  const int have = clamp_int(channels - u * PER, PER);
  auto to = [&](int j) { return tile.v + (row + j * R) * CH + u * PER; };
  if constexpr (UNIT == 2) {
    constexpr int BATCH = N < 16 ? N : 16;  // forward 32x512x1023 bf16: 8 118 us, 16 82, 32 84
#pragma unroll
    for (int j0 = 0; j0 < N; j0 += BATCH) {
      E v[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
        v[j] = have > 0 && row + (j0 + j) * R < live ? src[(int64_t)(j0 + j) * R * token_stride] : from_f32<E>(0.f);
#pragma unroll
      for (int j = 0; j < BATCH; ++j) *to(j0 + j) = v[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const bool some = have > 0 && row + j * R < live;
      copy_async(to(j), some ? src : from, some ? have * (int)sizeof(E) : 0);
      src += R * token_stride;
    }
  }
}

// ---- exchange over the cluster ----------------------------------------------------------------
// The chunks' maps.  Each CTA sends its own into every CTA's table, at its rank; the threads of run
// k send to the CTAs k, k + RUNS, ...  A message is an asynchronous store that reports its bytes to
// the receiver's mbarrier, so neither side has to wait for the stores of results that are still
// under way, as the release of a cluster barrier does (64x512x1024, which needs no exchange,
// against 1x65536x1024, bf16 forward, per element: 1.5 and 2.0 ps, with the cluster barrier 3.3).  The table and its
// mbarrier alternate between two halves: a CTA sends step s + 2 only when it has all of step s + 1,
// which every CTA sends only after it has read step s.  A map that holds a reset is sent with the
// factor -1, which no product of decays is.
template <int CH>
struct Table {
  float4 run[2][kMaxCluster][CH / 2];
  uint64_t arrived[2];
};

// What a thread that has given up does last: copies and messages still under way to its CTA land before
// the shared memory is given back.
__device__ __forceinline__ void pause() {
  for (int k = 0; k < 1000; ++k) __nanosleep(1000);
}

__device__ __forceinline__ uint32_t in_cta(uint32_t address, int rank) {
  uint32_t there;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(address), "r"(rank));
  return there;
}

// Called by all threads of the cluster before anything else touches the table.
template <int CH>
__device__ __forceinline__ void open_table(Table<CH>& t) {
  if (threadIdx.x == 0) {
    barrier_init(&t.arrived[0]);
    barrier_init(&t.arrived[1]);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  cg::this_cluster().sync();
}

template <int CH, int RUNS>
__device__ __forceinline__ void send(Table<CH>& t, int half, const Place& w, Run mine, bool cut) {
  if (threadIdx.x == 0) barrier_expect(&t.arrived[half], (uint32_t)w.cluster * sizeof(t.run[0][0]));
  if (cut) mine.a = two(-1.f);
  const uint32_t slot = shared_address(&t.run[half][w.rank][w.pair]), bar = shared_address(&t.arrived[half]);
  for (int k = w.slot; k < w.cluster; k += RUNS)
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(in_cta(slot, k)),
                 "f"(mine.a.x), "f"(mine.a.y), "f"(mine.b.x), "f"(mine.b.y), "r"(in_cta(bar, k))
                 : "memory");
}

// The table's map of the chunk of CTA k, applied to h.
template <bool RESET, int CH>
__device__ __forceinline__ float2 apply_total(const Table<CH>& t, int half, int k, const Place& w, float2 h) {
  const Run m = as_run(t.run[half][k][w.pair]);
  return apply(m, RESET && m.a.x < 0.f, h);
}

// ---- host side --------------------------------------------------------------------------------
// The encoder of tile descriptors is a function of the driver.
inline PFN_cuTensorMapEncodeTiled_v12000 tile_encoder() {
  static const PFN_cuTensorMapEncodeTiled_v12000 found = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult how;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &how) != cudaSuccess ||
        how != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  }();
  return found;
}

// Describes a tensor as tiles of `channels` x `tokens`; false where that is not possible.
template <typename P>
inline bool describe(CUtensorMap& map, const Seq<P>& t, const RecurrenceParams& p, int dtype, int channels, int tokens) {
  const uint64_t item = dtype == GS_F32 ? 4 : 2;
  const cuuint64_t row = (cuuint64_t)((p.D * item + 15) / 16 * 16);
  const cuuint64_t size[3] = {(cuuint64_t)p.D, (cuuint64_t)p.T, (cuuint64_t)p.B};
  // a dimension of one entry may come with any stride
  const cuuint64_t stride[2] = {p.T > 1 ? t.token * item : row, p.B > 1 ? t.batch * item : row};
  const cuuint32_t box[3] = {(cuuint32_t)channels, (cuuint32_t)tokens, 1}, step[3] = {1, 1, 1};
  const CUtensorMapDataType type = dtype == GS_F32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == GS_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                     : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const auto encode = tile_encoder();
  return encode && stride[0] && stride[1] &&
         encode(&map, type, 3, const_cast<void*>(static_cast<const void*>(t.data)), size, stride, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Calls f with the channels of a CTA and the size of a copy as constants.
template <typename F>
inline cudaError_t with_cut(const RecurrenceShape& shape, int unit, F&& f) {
  using std::integral_constant;
  auto with_unit = [&](auto channels) {
    return unit == 16  ? f(channels, integral_constant<int, 16>())
           : unit == 4 ? f(channels, integral_constant<int, 4>())
                       : f(channels, integral_constant<int, 2>());
  };
  return shape.channels == 64 ? with_unit(integral_constant<int, 64>()) : with_unit(integral_constant<int, 32>());
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
