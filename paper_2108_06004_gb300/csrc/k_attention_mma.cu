// A walk of linear attention (see attention.cuh) on the tensor cores, for 16-bit types.
//
// In blocks of 128 tokens, w_n = e^(g n), with i and j counted along the walk from the block's first token and S the state
// before it:
//   P = Q K' (scores),  A_ij = in w_{i-j} P_ij for j <= i, else 0,  U = (in w_{127-j} K_j)' V
//   O_i = out (w_{i+1} (Q S)_i + (A V)_i),   S <- w_128 S + U
// (backwards w_i for w_{i+1} and w_{128-j} for w_{127-j}).  S stays in fp32 in the threads' registers: a block's U is summed in
// tensor memory from zero, where what a product cuts off is small, and added to S with a rounding (with S itself as the
// sum in tensor memory, a last state was off by 3.5e-6 instead of 3e-7).  U does not need S and is made one block ahead.
// Where e^(-128 g) is at most e^8, w_{i+1} comes last, with w_{-j-1} in place of w_{i-j}: Q S and A V are one sum then.
//
// Operands are 16-bit.  Q, K and V are as they are in memory; A and S as factors are a sum of two parts of the type,
// which keeps 2^-17 or better of each, well below the rounding of a stored o: one in 300 to 500 is the neighbour of what fp32
// factors would give (a first part that is cut off keeps 2^-16, twice as many neighbours, and is 3 % faster for 16x4096x16x128;
// one part is a tenth faster and would make the error of o 1.4 times the one of its rounding); the weighted keys are three parts of bf16 (24 bits) where a state is
// given back in fp32 and otherwise two, and two of fp16 (22 bits).  fp16 has no room for scores and states of any size, so
// its parts are taken from values scaled by powers of two: block by block bounds of all of them follow from the
// largest |q|, |k| and |v|, which three warps that have nothing else to do find, and the scales from the bounds.
//
// Eight or sixteen warps do the arithmetic between the products; a thread of one more issues products and loads (three
// others are there because registers can be moved from four warps at once only).  In a block: parts of S | Q S runs: A |
// A V runs: S after the block, weighted keys of the next one | its U and scores run: o is stored.  A lane of tensor memory is a
// token for P, A and O and a row of the state for U and the weighted keys.
//
// Bound by the tensor cores and by the arithmetic between them in turn, which overlap in part: a product of 128 x 128 x 16
// takes 64 clocks at the nominal rate and about 80 at that of a large library product, of which a block of 128 x 128 heads needs 56 or
// 64.  16x4096x16x128 bf16 forward takes 225 us without a last state where all decays are slow, 231 where all are quick, 279 and
// 299 with one (70 and 57 % of the copy rate for the slow ones); 16x4096x32x64: 299, 316, 338 and 355; in fp16 287 to 360. Copies of
// the kernel when it took 276 took 222 without the arithmetic, 220 without the products and 261 out of L2. 256 heads are 1.7 waves of
// 152 CTAs.  What made it faster,
// from 671 us: descriptors by addition (spilled ones cost 180 clocks a product); o by way of shared memory and as tiles;
// sixteen warps in place of eight; U one block ahead; keys transposed by matrix loads; one arrival a warp.
#include <cudaTypedefs.h>

#include <atomic>

#include "attention.cuh"
#include "tensor_core.cuh"

namespace gs {
namespace {

using namespace tc;

constexpr int kBlockTokens = 128, kTableBytes = 3 << 10;

// One walk a launch: parameters at a place that a CTA has to work out cost a walk that fills the device 5 %.
struct AttentionMmaParams {
  CUtensorMap q, k, v, o;
  AttentionParams a;
};

// C rows of the state (64 or 128) and D columns of it a CTA.  The smallest one leaves room for two CTAs an SM.
template <int C, int D>
struct Plan {
  static constexpr bool kNarrow = C == 64 && D == 64;
  static constexpr int kCtas = kNarrow ? 2 : 1, kColumns = 512 / kCtas;
  // Worker warps in groups of four; a group takes 1 / kGroups of the columns.  All threads have the same number of
  // registers at first, and then the workers more and the others fewer, whose sum is at most as many.
  static constexpr int kGroups = D == 64 ? 2 : 4, kWorkers = 128 * kGroups, kThreads = kWorkers + 128;
  static constexpr int kAtFirst = kNarrow ? 80 : D == 64 ? 168 : 96, kWorker = kNarrow ? 96 : D == 64 ? 224 : 112,
                       kOther = kNarrow ? 48 : D == 64 ? 56 : 32;
  static_assert(kGroups * kWorker + kOther <= (kGroups + 1) * kAtFirst, "more registers than the CTA has");
  // columns: the block's own sum of keys and values, O, P (A takes its place), and the weighted keys: of either half of
  // the block, as many of 32 as they have parts.  Narrow, they take the place of O and P when o has been read; three
  // parts of the second half that of P.
  static constexpr int U = 0, O = kNarrow ? 64 : 128, P = kNarrow ? 128 : 256, W0 = kNarrow ? 64 : 384;
  static constexpr int kPanel = kBlockTokens * 128;  // bytes of 64 columns of a block
  static constexpr int kQ = C / 64 * kPanel, kV = D / 64 * kPanel, kPart = C * D * 2;
  static constexpr int oQ = 0, oK = kQ, oV = oK + 2 * kQ, oS = oV + 2 * kV, oTables = oS + 2 * kPart;
  static constexpr int kBytes = oTables + kTableBytes;
};
struct Tables {
  float weight[256];  // in w_d of a score at weight[128 + row - column], zero past the diagonal
  alignas(16) float rise[128];  // in / w of a score's column, where the row's factor comes last
  float power[129];   // w_n
  alignas(16) float key[128];  // of a row's weighted key, zero past the block's tokens
  uint64_t q_full, kv_full[2], scores, read, done, summed, state_ready, a_ready, w_ready[2];
  // fp16: the largest |q|, |k| and |v| of a block as three warps have found them, two blocks in turn, and |first state|
  uint64_t q_known, kv_known[2];
  float largest[2][3][3];
  int first;
  uint32_t tmem;
};
static_assert(sizeof(Tables) <= kTableBytes, "tables do not fit");
static_assert(Plan<128, 128>::kBytes <= 232448, "a CTA's shared memory");

template <int WORKERS>
__device__ __forceinline__ void sync_workers() {
  asm volatile("bar.sync 1, %0;" ::"n"(WORKERS) : "memory");
}

// Two values as a sum of parts of the type, each the nearest one to what the parts before leave.
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 mul(float2 a, float b) { return __fmul2_rn(a, make_float2(b, b)); }
__device__ __forceinline__ float2 less(float2 a, float2 b) { return __ffma2_rn(b, make_float2(-1.f, -1.f), a); }
template <typename E>
__device__ __forceinline__ uint32_t last_part(float2 v) {
  const typename Pack2<E>::type h = Pack2<E>::down(v);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename E>
__device__ __forceinline__ uint32_t part_of(float2& v) {
  const uint32_t h = last_part<E>(v);
  v = less(v, Pack2<E>::up(*reinterpret_cast<const typename Pack2<E>::type*>(&h)));
  return h;
}
__device__ __forceinline__ float2 pair_of(const uint32_t* x) { return make_float2(__uint_as_float(x[0]), __uint_as_float(x[1])); }

// 2^-n for the power of two that brings a bound to [2^13, 2^14); 1 for a bound of zero.
__device__ __forceinline__ int exponent_of(float bound) {
  return bound > 0.f ? min(max((int)(__float_as_uint(bound) >> 23) - 127 - 13, -100), 100) : 0;
}
__device__ __forceinline__ float power_of_two(int n) { return __uint_as_float((uint32_t)(min(max(n, -126), 126) + 127) << 23); }

// PARTS: of a weighted key.  SUMS: only the piece's own sum, from a state of zero, into carry.
template <typename E, typename R, int C, int D, int PARTS, bool SUMS>
__global__ void __launch_bounds__(Plan<C, D>::kThreads, Plan<C, D>::kCtas)
k_attention_mma(const __grid_constant__ AttentionMmaParams params) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  using L = Plan<C, D>;
  constexpr bool HALF = std::is_same<E, __half>::value;
  constexpr int kWorkers = L::kWorkers, COLS = D / L::kGroups;  // columns of a thread
  constexpr int W1 = L::kNarrow || PARTS == 2 ? L::W0 + 32 * PARTS : L::P;
  extern __shared__ __align__(1024) char base[];
  Tables& tab = *reinterpret_cast<Tables*>(base + L::oTables);
  const AttentionParams& p = params.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int slices = (p.D + D - 1) / D;
  const int slice = blockIdx.x % slices, head = blockIdx.x / slices % p.H, item = blockIdx.x / slices / p.H;
  Piece w;
  if (!find_piece(p, item, w)) return;
  if (SUMS && (w.ends || w.t0 >= w.length)) return;  // nothing comes after it
  const int blocks = w.t1 > w.t0 ? (w.t1 - w.t0 + kBlockTokens - 1) / kBlockTokens : 0, c0 = slice * D;
  const float g = log_decay_of(p, head);
  // tokens of block n, and the first of them; row r of its tiles is the token r after that
  const auto tokens = [&](int n) { return min(kBlockTokens, w.t1 - w.t0 - n * kBlockTokens); };
  const auto first_token = [&](int n) {
    const int at = w.t0 + n * kBlockTokens;
    return w.start + (p.back ? w.length - at - tokens(n) : at);
  };

  if (threadIdx.x == kWorkers) {
    barrier_init(&tab.q_full, 1);
    barrier_init(&tab.kv_full[0], 1);
    barrier_init(&tab.kv_full[1], 1);
    for (uint64_t* b : {&tab.scores, &tab.read, &tab.done, &tab.summed}) barrier_init(b, 1);
    for (uint64_t* b : {&tab.state_ready, &tab.a_ready, &tab.w_ready[0], &tab.w_ready[1]}) barrier_init(b, kWorkers / 32);
    for (uint64_t* b : {&tab.q_known, &tab.kv_known[0], &tab.kv_known[1]}) barrier_init(b, 3);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kWorkers / 32) tmem_alloc<L::kColumns>(&tab.tmem);
  if (threadIdx.x == 9) tab.first = 0;
  if (threadIdx.x < 129) tab.power[threadIdx.x] = expf(g * (float)threadIdx.x);
  if (threadIdx.x < 256) {
    const int d = p.back ? 128 - (int)threadIdx.x : (int)threadIdx.x - 128;  // tokens from a key to a query
    tab.weight[threadIdx.x] = d >= 0 ? expf(g * (float)d) * p.in_scale : 0.f;
  }
  before_sync();
  __syncthreads();
  after_sync();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tmem = tab.tmem;
  // Waits end after a second or so (which nothing that this kernel does can cause). A thread whose wait has run out announces nothing
  // more, so that the waits of all that have to do with it run out too; a worker then stores NaN.
  bool lost = false;

  if (threadIdx.x >= kWorkers) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::kOther));
    if (HALF && warp > kWorkers / 32) {
      // the three other warps: the largest values of a tile's first m rows, before anyone needs them
      const int mine = warp - kWorkers / 32 - 1;
      const auto largest = [&](const char* tile, int panels, int m) {
        __half2 most = __float2half2_rn(0.f);
        for (int panel = 0; panel < panels; ++panel)
#pragma unroll 4
          for (int at = mine * 32 + lane; at < m * 8; at += 96) {
            const uint4 x = *reinterpret_cast<const uint4*>(tile + panel * L::kPanel + at * 16);
            const __half2* h = reinterpret_cast<const __half2*>(&x);
#pragma unroll
            for (int j = 0; j < 4; ++j) most = __hmax2(most, __habs2(h[j]));
          }
        float f = fmaxf(__low2float(most), __high2float(most));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) f = fmaxf(f, __shfl_xor_sync(0xFFFFFFFFu, f, o));
        return f;
      };
      // A block's places are free: what was in them was read before the block before last was done, and its tiles
      // come after that.
      for (int n = 0; n < blocks; ++n) {
        float* const to = tab.largest[n & 1][mine];
        if (lost = !barrier_wait(&tab.kv_full[n & 1], n >> 1, p.find_tries); __any_sync(0xFFFFFFFFu, lost)) break;
        const float k = largest(base + L::oK + (n & 1) * L::kQ, C / 64, tokens(n)), v = largest(base + L::oV + (n & 1) * L::kV, D / 64, tokens(n));
        if (lane == 0) {
          to[1] = k;
          to[2] = v;
          barrier_arrive(&tab.kv_known[n & 1]);
        }
        if (SUMS) continue;
        if (lost = !barrier_wait(&tab.q_full, n, p.find_tries); __any_sync(0xFFFFFFFFu, lost)) break;
        const float q = largest(base + L::oQ, C / 64, tokens(n));
        if (lane == 0) {
          to[0] = q;
          barrier_arrive(&tab.q_known);
        }
      }
    }
    if (threadIdx.x == kWorkers && blocks > 0) {
      const auto load_kv = [&](int n) {
        const int s = n & 1, t = (int)first_token(n);
        barrier_expect(&tab.kv_full[s], L::kQ + L::kV);
        for (int j = 0; j < C / 64; ++j)
          tile_load(base + L::oK + s * L::kQ + j * L::kPanel, &params.k, j * 64, head / p.k.share, t, w.batch, &tab.kv_full[s]);
        for (int j = 0; j < D / 64; ++j)
          tile_load(base + L::oV + s * L::kV + j * L::kPanel, &params.v, c0 + j * 64, head / p.v.share, t, w.batch, &tab.kv_full[s]);
      };
      const auto load_q = [&](int n) {
        barrier_expect(&tab.q_full, L::kQ);
        for (int j = 0; j < C / 64; ++j)
          tile_load(base + L::oQ + j * L::kPanel, &params.q, j * 64, head / p.q.share, (int)first_token(n), w.batch, &tab.q_full);
      };
      const uint32_t q = matrix(shared_address(base + L::oQ), 0), parts = matrix(shared_address(base + L::oS), C * 128);
      const auto values = [&](int n) { return matrix(shared_address(base + L::oV + (n & 1) * L::kV), L::kPanel); };
      const auto wait = [&](uint64_t* bar, int phase) { return barrier_wait(bar, phase, p.issue_tries); };
      // U = K' V of block n
      const auto sum = [&](int n) {
        const uint32_t v = values(n);
        if (!wait(&tab.kv_full[n & 1], n >> 1)) return false;
        const auto half = [&](auto which) {
          constexpr int h = decltype(which)::value;
          if (!wait(&tab.w_ready[h], n)) return false;
          after_sync();
          each<4 * PARTS>([&](auto step) {  // the smallest parts first, while the sum is small
            constexpr int part = PARTS - 1 - decltype(step)::value / 4, j = decltype(step)::value % 4;
            multiply_t<(h ? W1 : L::W0) + part * 32 + j * 8, (h * 4 + j) * 2048>(tmem + L::U, tmem, v, product<E>(D, true),
                                                                                            h > 0 || decltype(step)::value > 0);
          });
          return true;
        };
        if (!half(std::integral_constant<int, 0>()) || !half(std::integral_constant<int, 1>())) return false;
        commit(&tab.summed);
        return true;
      };
      // P = Q K' of block n.  Its place is free when the products that read it are done: only products with the same
      // sum are ordered among themselves.  Keys and queries arrive apart, so both are waited for.
      const auto score = [&](int n) {
        const uint32_t k = matrix(shared_address(base + L::oK + (n & 1) * L::kQ), 0);
        if (!wait(&tab.kv_full[n & 1], n >> 1) || !wait(&tab.q_full, n)) return false;
        each<C / 16>([&](auto step) {
          constexpr int j = decltype(step)::value, at = j / 4 * L::kPanel + j % 4 * 32;
          multiply<at, at>(tmem + L::P, q, k, product<E>(128, false), j > 0);
        });
        commit(&tab.scores);
        return true;
      };
      constexpr bool APART = !L::kNarrow && PARTS == 2;  // the weighted keys are not in P's place
      // False where a wait has run out.
      const auto issue = [&] {
        load_kv(0);
        if (!SUMS) load_q(0);
        if (blocks > 1) load_kv(1);
        if (!sum(0)) return false;
        if constexpr (SUMS) {
          for (int n = 1; n < blocks; ++n) {
            if (!wait(&tab.summed, n - 1)) return false;
            if (n + 1 < blocks) load_kv(n + 1);
            if (!sum(n)) return false;
          }
        } else {
          if (!APART && !wait(&tab.summed, 0)) return false;
          if (!score(0)) return false;
          for (int n = 0; n < blocks; ++n) {
            if (!wait(&tab.state_ready, n)) return false;
            after_sync();
            each<C / 8>([&](auto step) {
              constexpr int part = decltype(step)::value / (C / 16), j = decltype(step)::value % (C / 16);
              multiply<j / 4 * L::kPanel + j % 4 * 32, part * L::kPart + j * 2048>(tmem + L::O, q, parts, product<E>(D, true), part + j > 0);
            });
            commit(&tab.read);
            if (n + 1 < blocks) {
              if (!wait(&tab.read, n)) return false;
              load_q(n + 1);
            }
            if (!wait(&tab.a_ready, n)) return false;
            after_sync();
            const uint32_t v = values(n);
            each<16>([&](auto step) {
              constexpr int part = decltype(step)::value / 8, j = decltype(step)::value % 8;
              multiply_t<j * 16 + part * 8, j * 2048>(tmem + L::O, tmem + L::P, v, product<E>(D, true), true);
            });
            commit(&tab.done);
            if (n + 1 >= blocks) break;
            if (!wait(&tab.done, n)) return false;
            if (APART) {
              if (n + 2 < blocks) load_kv(n + 2);  // in the place of block n's, whose last product is done
              // Rows of K that are not the block's tokens are zeroed by the workers, which say so with the weighted keys: a
              // block that is cut short has its scores after its sum.
              const bool cut = tokens(n + 1) < kBlockTokens;
              if (!cut && !score(n + 1)) return false;
              if (!sum(n + 1)) return false;
              if (cut && !score(n + 1)) return false;
            } else {
              if (!sum(n + 1) || !wait(&tab.summed, n + 1)) return false;
              if (n + 2 < blocks) load_kv(n + 2);
              if (!score(n + 1)) return false;
            }
          }
        }
        return true;
      };
      lost = !issue();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::kWorker));
    const auto wait = [&](uint64_t* bar, int phase) {
      lost = !barrier_wait(bar, phase, lost ? 1 : p.work_tries) || lost;
      lost = __any_sync(0xFFFFFFFFu, lost);
    };
    // What this warp has written is there for the thread that issues products.
    const auto arrive = [&](uint64_t* bar) {
      before_sync();
      __syncwarp();
      if (lane == 0 && !lost) barrier_arrive(bar);
    };
    // Whether the queries' decay w_{i+1} comes last, after both products, and A_ij has w_{-j-1} in place of w_{i-j}: only where
    // that makes them no more than e^8 times as large. (With e^32 for bf16, train 16x4096x16x128 took 1111 us, 1119 with e^8, and
    // inputs of 1e9 left fp32's range half way to outputs that are well inside.)
    const bool rises = -g * kBlockTokens <= 8.f;
    const int quad = warp & 3, group = warp >> 2, row = quad * 32 + lane, col0 = group * COLS;
    const uint32_t mine = tmem + ((uint32_t)(quad * 32) << 16);
    // Rows of the state: 64 are in the lanes of the warps that have less of A to work out, which is triangular.
    const int above = C == 64 && p.back ? 2 : 0, state_quad = quad - above, state_row = state_quad * 32 + lane;
    const bool holds = state_quad >= 0 && state_quad * 32 < C;
    const int64_t state = ((int64_t)w.sequence * p.H + head) * p.C * p.D;
    float* carry = p.carry + ((int64_t)item * p.H + head) * p.C * p.D;
    const float nan = __uint_as_float(0x7FC00000u);
    if (!SUMS && !p.offsets) {  // tokens past the row's length
      const int64_t until = min((int64_t)w.t0 + p.segment, p.T);
      for (int64_t t = max(w.t0, w.length) + warp; t < until; t += kWorkers / 32)
        for (int d = lane; d < D && c0 + d < p.D; d += 32)
          static_cast<R*>(p.o.data)[w.batch * p.o.batch + t * p.o.token + head * p.o.head + c0 + d] = from_f32<R>(0.f);
    }
    // the state: this thread's row, the group's columns
    float S[COLS];
    float bound = 0.f;
    if (holds) {
      const bool given = (w.opens && w.ends) || p.chained, mine_too = !SUMS && state_row < p.C;
#pragma unroll
      for (int j = 0; j < COLS; ++j) {
        const int col = c0 + col0 + j;
        S[j] = 0.f;
        if (mine_too && given && p.first && col < p.D) S[j] = p.first[state + state_row * p.state_row + col * p.state_col];
      }
      if (mine_too && w.t0 < w.length) {
        const Decay d = decay_of(g * (float)p.segment);
        // the state before the piece, or the sums of the pieces before it
        for (int n = p.chained ? w.t0 / p.segment : given ? -1 : 0; n >= (p.chained ? 1 : 0); --n) {
          const float* u = carry + ((int64_t)state_row - (int64_t)n * p.H * p.C) * p.D + c0 + col0;
#pragma unroll
          for (int j = 0; j < COLS; j += 4) {
            if (c0 + col0 + j >= p.D) continue;
            const float4 x = *reinterpret_cast<const float4*>(u + j);
            S[j] = decayed(S[j], d, x.x);
            S[j + 1] = decayed(S[j + 1], d, x.y);
            S[j + 2] = decayed(S[j + 2], d, x.z);
            S[j + 3] = decayed(S[j + 3], d, x.w);
          }
        }
      }
      if (HALF && !SUMS) {
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < COLS; ++j) most = fmaxf(most, fabsf(S[j]));
        atomicMax(&tab.first, __float_as_int(most));
      }
    }
    const auto known = [&](int n, int what) {
      const auto& l = tab.largest[n & 1];
      return fmaxf(l[0][what], fmaxf(l[1][what], l[2][what]));
    };
    if (HALF && blocks > 0) {
      sync_workers<kWorkers>();
      bound = __int_as_float(tab.first);
    }
    int made = -1;  // tokens that the keys' weights are made for
    // What is known of a block before its keys are weighted, and of the one whose o is being worked out.
    struct Block {
      int m, scale;
      float k, v;
      Decay decay;
    } next, now;
    next.m = 0;
    const auto open = [&](int n) {
      const int m = tokens(n);
      if (m != next.m) next.decay = decay_of(g * (float)m);
      next.m = m;
      char* k = base + L::oK + (n & 1) * L::kQ;
      char* v = base + L::oV + (n & 1) * L::kV;
      wait(&tab.kv_full[n & 1], n >> 1);
      if (made != next.m) {
        if (made >= 0) sync_workers<kWorkers>();  // the tables before have been used
        if (threadIdx.x < 128) {
          const int r = threadIdx.x;
          tab.key[r] = r < next.m ? tab.power[p.back ? r + 1 : next.m - 1 - r] * p.in_scale : 0.f;
          tab.rise[r] = expf(-g * (float)(p.back ? next.m - 1 - r : r + 1)) * p.in_scale;
        }
        if (next.m < kBlockTokens) {
          // rows that are not the block's tokens: zeros, whatever they were
          const auto trim = [&](char* tile, int panels) {
            const int rows = kBlockTokens - next.m;
            for (int at = threadIdx.x; at < panels * rows * 8; at += kWorkers)
              *reinterpret_cast<uint4*>(tile + at / 8 / rows * L::kPanel + (next.m + at / 8 % rows) * 128 + at % 8 * 16) = make_uint4(0, 0, 0, 0);
          };
          trim(k, C / 64);
          trim(v, D / 64);
          shared_fence();
        }
        sync_workers<kWorkers>();
      }
      next.scale = 0;
      if constexpr (HALF) {
        wait(&tab.kv_known[n & 1], n >> 1);
        next.k = known(n, 1);
        next.v = known(n, 2);
        next.scale = exponent_of(next.k * fabsf(p.in_scale));
      }
      made = next.m;
    };
    // The group's weighted keys of either half of block n, transposed to rows of the state: 32 rows, in two halves, of
    // 16 tokens, or twice 16.
    constexpr int PAIRS = 32 / L::kGroups;
    uint32_t part[PARTS][2][PAIRS / 2];
    const auto weigh = [&](int n, int h) {
      if (!holds) return;
      const uint32_t from = shared_address(base + L::oK + (n & 1) * L::kQ + state_quad / 2 * L::kPanel);
      const float shrink = HALF ? power_of_two(-next.scale) : 1.f;
#pragma unroll
      for (int j = 0; j < PAIRS / 8; ++j) {
        const int t = h * 64 + group * 2 * PAIRS + j * 16;
        const float2 weight[2] = {*reinterpret_cast<const float2*>(&tab.key[t + lane % 4 * 2]),
                                  *reinterpret_cast<const float2*>(&tab.key[t + 8 + lane % 4 * 2])};
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int word = (state_quad % 2) * 4 + r * 2 + (lane >> 3 & 1);
          uint32_t x[4];
          load_across(x, from + (t + (lane >> 4) * 8 + lane % 8) * 128 + (word ^ (lane % 8)) * 16);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float2 f = Pack2<E>::up(*reinterpret_cast<const typename Pack2<E>::type*>(&x[i]));
            f = mul(f, weight[i / 2]);
            if (HALF) f = mul(f, shrink);
#pragma unroll
            for (int q = 0; q + 1 < PARTS; ++q) part[q][r][j * 4 + i] = part_of<E>(f);
            part[PARTS - 1][r][j * 4 + i] = last_part<E>(f);
          }
        }
      }
    };
    const auto put = [&](int h) {
      if (holds) {
#pragma unroll
        for (int i = 0; i < PARTS; ++i)
#pragma unroll
          for (int r = 0; r < 2; ++r)
            tmem_store_matrices(part[i][r], mine + ((uint32_t)(r * 16) << 16) + (h ? W1 : L::W0) + i * 32 + group * PAIRS,
                                std::integral_constant<int, PAIRS / 2>());
        wait_store();
      }
      arrive(&tab.w_ready[h]);
    };
    // the state after block n
    const auto advance = [&](int n) {
      wait(&tab.summed, n);
      after_sync();
      if (!holds) return;
      uint32_t x[32];
      tmem_load(x, mine + L::U + col0);
      const float grow = HALF ? power_of_two(now.scale) : 1.f;
#pragma unroll
      for (int j = 0; j < COLS; j += 2) {
        float2 u = pair_of(x + j);
        if (HALF) u = mul(u, grow);
        float2 v = make_float2(S[j], S[j + 1]);
        v = __ffma2_rn(v, make_float2(now.decay.a, now.decay.a), __ffma2_rn(v, make_float2(now.decay.b, now.decay.b), u));
        S[j] = v.x;
        S[j + 1] = v.y;
      }
    };
    if (blocks > 0) {
      open(0);
      weigh(0, 0);
      put(0);
      weigh(0, 1);
      put(1);
      now = next;
    }
    for (int n = 0; n < blocks; ++n) {
      if constexpr (SUMS) {
        if (n + 1 < blocks) open(n + 1);
        advance(n);
        if (n + 1 < blocks) {
          weigh(n + 1, 0);
          put(0);
          weigh(n + 1, 1);
          put(1);
        }
        now = next;
        continue;
      }
      int a_scale = 0, s_scale = 0;
      bool last = rises;
      if (lane == 0) stores_read();
      sync_workers<kWorkers>();  // the last block's o has left the place of the parts
      if constexpr (HALF) {
        wait(&tab.q_known, n);
        s_scale = exponent_of(bound);
        const float score = known(n, 0) * now.k * (float)C * fabsf(p.in_scale);
        a_scale = exponent_of(score * expf(-g * kBlockTokens));
        last = rises && abs(a_scale - s_scale) <= 6;  // both products have one scale then
        if (last)
          a_scale = s_scale = max(s_scale, a_scale);
        else
          a_scale = exponent_of(score);
        bound = bound * (now.decay.a + now.decay.b) * 1.0001f + now.k * now.v * (float)now.m * fabsf(p.in_scale);
      }
      // the state as a factor
      if (holds) {
        const float shrink = HALF ? power_of_two(-s_scale) : 1.f;
#pragma unroll
        for (int j = 0; j < COLS / 8; ++j) {
          const int col = col0 + j * 8;
          char* to = base + L::oS + col / 64 * (C * 128) + state_row * 128 + (((col % 64) / 8) ^ (state_row & 7)) * 16;
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float2 f = make_float2(S[j * 8 + 2 * i], S[j * 8 + 2 * i + 1]);
            if (HALF) f = mul(f, shrink);
            hi[i] = part_of<E>(f);
            lo[i] = last_part<E>(f);
          }
          *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(to + L::kPart) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
      }
      shared_fence();
      arrive(&tab.state_ready);
      // scores to A, in their place
      wait(&tab.scores, n);
      after_sync();
      {
        const float shrink = HALF ? power_of_two(-a_scale) : 1.f;
        const float undo = last ? shrink / tab.power[p.back ? max(now.m - 1 - row, 0) : row + 1] : shrink;
#pragma unroll L::kNarrow ? 1 : 2
        for (int col = group * (128 / L::kGroups); col < (group + 1) * (128 / L::kGroups); col += 16) {
          uint32_t x[16], hi[8], lo[8];
          const int tile = col & ~31;
          if (p.back ? tile < quad * 32 : tile > quad * 32) {  // past the diagonal
#pragma unroll
            for (int j = 0; j < 8; ++j) hi[j] = lo[j] = 0;
          } else {
            tmem_load(x, mine + L::P + col);
            if (last && tile != quad * 32) {
#pragma unroll
              for (int j = 0; j < 8; j += 2) {
                const float4 rise = *reinterpret_cast<const float4*>(tab.rise + col + 2 * j);
                float2 f = mul(pair_of(x + 2 * j), make_float2(rise.x, rise.y)), e = mul(pair_of(x + 2 * j + 2), make_float2(rise.z, rise.w));
                if (HALF) f = mul(f, shrink), e = mul(e, shrink);
                hi[j] = part_of<E>(f);
                lo[j] = last_part<E>(f);
                hi[j + 1] = part_of<E>(e);
                lo[j + 1] = last_part<E>(e);
              }
            } else {
              const float* weight = tab.weight + 128 + row - col;
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                float2 f = mul(mul(pair_of(x + 2 * j), make_float2(weight[-2 * j], weight[-2 * j - 1])), undo);
                hi[j] = part_of<E>(f);
                lo[j] = last_part<E>(f);
              }
            }
          }
          tmem_store(hi, mine + L::P + col);
          tmem_store(lo, mine + L::P + col + 8);
        }
        wait_store();
      }
      // what has been read from the state, with the query's decay
      const int walked = p.back ? now.m - 1 - row : row + 1;
      float factor = row < now.m ? tab.power[walked] * (last ? p.out_scale : 1.f) : 0.f;
      if (HALF && last) factor *= power_of_two(a_scale);
      if (!last) {
        wait(&tab.read, n);
        after_sync();
        if (HALF) factor *= power_of_two(s_scale - a_scale);
        uint32_t x[32];
        tmem_load(x, mine + L::O + col0);
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
          const float2 f = mul(pair_of(x + j), factor);
          x[j] = __float_as_uint(f.x);
          x[j + 1] = __float_as_uint(f.y);
        }
        tmem_store(x, mine + L::O + col0);
        wait_store();
        factor = p.out_scale * (HALF ? power_of_two(a_scale) : 1.f);
      }
      arrive(&tab.a_ready);
      // the next block's weighted keys
      const bool more = n + 1 < blocks;
      if (more) open(n + 1);
      advance(n);
      if constexpr (!L::kNarrow) {
        if (more) {
          weigh(n + 1, 0);
          put(0);
          weigh(n + 1, 1);
          if (PARTS == 2) put(1);
        }
      }
      wait(&tab.done, n);
      after_sync();
      if constexpr (!L::kNarrow && PARTS == 3) {
        if (more) put(1);
      }
      {
        // By way of shared memory, where the parts of the state were: the warp's 32 tokens, 64 bytes of each at a time, as
        // a tile; in a block that is cut short, whose other rows may be another sequence's, row by row.
        constexpr int N = 64 / (int)sizeof(R), WORD = 16 / (int)sizeof(R);
        char* stage = base + L::oS + warp * 2048;
        const int64_t token = first_token(n) + quad * 32;
        uint32_t x[32];
        tmem_load(x, mine + L::O + col0);
        if (lost) {
#pragma unroll
          for (int j = 0; j < 32; ++j) x[j] = 0x7FC00000u;
        }
#pragma unroll
        for (int e = 0; e < 32 / N; ++e) {
          const int col = c0 + col0 + e * N;
          if (e > 0 && lane == 0) stores_read();
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint4 word;
            typename Pack2<R>::type* pair = reinterpret_cast<typename Pack2<R>::type*>(&word);
#pragma unroll
            for (int i = 0; i < WORD / 2; ++i) {
              pair[i] = Pack2<R>::down(mul(pair_of(x + e * N + j * WORD + 2 * i), factor));
            }
            *reinterpret_cast<uint4*>(stage + lane * 64 + ((j ^ (lane >> 1)) & 3) * 16) = word;
          }
          if (now.m == kBlockTokens) {
            shared_fence();
            __syncwarp();
            if (lane == 0 && col < p.D) tile_store(stage, &params.o, col, head, (int)token, w.batch);
          } else {
            __syncwarp();
            R* o = static_cast<R*>(p.o.data) + w.batch * p.o.batch + head * p.o.head;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int r = j * 8 + lane / 4, at = col + lane % 4 * WORD;
              const uint4 word = *reinterpret_cast<const uint4*>(stage + r * 64 + ((lane ^ (r >> 1)) & 3) * 16);
              if (quad * 32 + r < now.m && at < p.D) *reinterpret_cast<uint4*>(o + (token + r) * p.o.token + at) = word;
            }
          }
        }
      }
      if constexpr (L::kNarrow) {
        if (more) {
          sync_workers<kWorkers>();  // the keys go where O was read
          weigh(n + 1, 0);
          put(0);
          weigh(n + 1, 1);
          put(1);
        }
      }
      now = next;
    }
    if (!SUMS && lane == 0) stores_done();
    float* to = SUMS ? carry : w.ends ? p.last : nullptr;
    if (to && holds && state_row < p.C) {
      const int64_t down = SUMS ? p.D : p.state_row, along = SUMS ? 1 : p.state_col;
      to += (SUMS ? 0 : state) + state_row * down;
#pragma unroll
      for (int j = 0; j < COLS; ++j) {
        const int col = c0 + col0 + j;
        if (col < p.D) to[col * along] = lost ? nan : S[j];
      }
    }
    __syncwarp();
    before_sync();
  }
  const bool gone = __syncthreads_or(lost);
  after_sync();
  if (gone)  // copies and products still under way end before their memory is given back
    for (int k = 0; k < 1000; ++k) __nanosleep(1000);
  __syncwarp();
  if (warp == kWorkers / 32) tmem_free<L::kColumns>(tmem);
}

// The encoder of tile descriptors is a function of the driver.
PFN_cuTensorMapEncodeTiled_v12000 tile_encoder() {
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

// Describes a tensor of `heads` heads of `size` elements as tiles of 128 (or 64) bytes of a head x `tokens`; false where that
// is not possible.
bool describe(CUtensorMap& map, const HeadsIn& t, const AttentionParams& p, int size, int dtype, int bytes, int tokens) {
  const int64_t heads = p.H / t.share, rows = p.offsets ? 1 : p.B;
  const int64_t item = dtype == GS_F32 ? 4 : 2, any = 16;  // a dimension of one entry may come with any stride
  const cuuint64_t sizes[4] = {(cuuint64_t)size, (cuuint64_t)heads, (cuuint64_t)p.T, (cuuint64_t)rows};
  const int64_t step[3] = {heads > 1 ? t.head * item : any, p.T > 1 ? t.token * item : any, rows > 1 ? t.batch * item : any};
  if (reinterpret_cast<uintptr_t>(t.data) % 16 != 0) return false;
  for (const int64_t s : step)
    if (s <= 0 || s % 16 != 0 || s >= int64_t(1) << 40) return false;
  const cuuint64_t strides[3] = {(cuuint64_t)step[0], (cuuint64_t)step[1], (cuuint64_t)step[2]};
  const cuuint32_t box[4] = {(cuuint32_t)(bytes / item), 1, (cuuint32_t)tokens, 1}, unit[4] = {1, 1, 1, 1};
  const CUtensorMapDataType type = dtype == GS_F32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == GS_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                     : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const auto encode = tile_encoder();
  return encode && encode(&map, type, 4, const_cast<void*>(t.data), sizes, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename E, typename R, int C, int D, int PARTS, bool SUMS>
cudaError_t launch_mma(dim3 grid, cudaStream_t s, const AttentionMmaParams& p) {
  const auto kernel = k_attention_mma<E, R, C, D, PARTS, SUMS>;
  constexpr int smem = Plan<C, D>::kBytes;
  // shared memory beyond the default is asked for once per kernel and device
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(done.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    done.fetch_or(bit, std::memory_order_release);
  }
  return launch_cluster(kernel, grid, dim3(Plan<C, D>::kThreads), smem, 1, s, p);
}

template <typename E, typename R, int C, int D, int PARTS>
cudaError_t walk_parts(const AttentionMmaParams& q, cudaStream_t s) {
  const AttentionParams& p = q.a;
  const dim3 grid((unsigned)((int64_t)p.items * p.H * ((p.D + D - 1) / D)));
  if (p.segments > 1) {
    cudaError_t e = launch_mma<E, R, C, D, PARTS, true>(grid, s, q);
    if (e != cudaSuccess) return e;
    AttentionWalks one;
    one.of[0] = p;
    one.count = 1;
    if (!p.chained) e = launch_attention_carry(one, s);
    if (e != cudaSuccess) return e;
  }
  return launch_mma<E, R, C, D, PARTS, false>(grid, s, q);
}

// Keys of bf16 in three parts where a state is given back in fp32; two, which 16-bit outputs do not tell from more,
// where none is.
template <typename E, typename R, int C, int D>
cudaError_t walk(const AttentionMmaParams& q, cudaStream_t s) {
  if constexpr (std::is_same<E, __nv_bfloat16>::value)
    if (q.a.last) return walk_parts<E, R, C, D, 3>(q, s);
  return walk_parts<E, R, C, D, 2>(q, s);
}

}  // namespace

cudaError_t launch_attention_mma(const AttentionWalks& walks, int dtype, cudaStream_t s, bool& taken) {
  taken = false;
  const AttentionParams& p = walks.of[0];
  if (p.T == 0) return cudaSuccess;
  AttentionMmaParams q[3];
  for (int k = 0; k < walks.count; ++k) {
    const AttentionParams& a = q[k].a = walks.of[k];
    const HeadsIn o = {a.o.data, a.o.batch, a.o.token, a.o.head, 1};
    if (!describe(q[k].q, a.q, a, a.C, dtype, 128, kBlockTokens) || !describe(q[k].k, a.k, a, a.C, dtype, 128, kBlockTokens) ||
        !describe(q[k].v, a.v, a, a.D, dtype, 128, kBlockTokens) || !describe(q[k].o, o, a, a.D, a.wide ? GS_F32 : dtype, 64, 32))
      return cudaSuccess;
  }
  taken = true;
  const auto sizes = [&](auto e, auto r, const AttentionMmaParams& w) {
    using E = decltype(e);
    using R = decltype(r);
    if (p.C <= 64) return p.D <= 64 ? walk<E, R, 64, 64>(w, s) : walk<E, R, 64, 128>(w, s);
    return p.D <= 64 ? walk<E, R, 128, 64>(w, s) : walk<E, R, 128, 128>(w, s);
  };
  for (int k = 0; k < walks.count; ++k) {
    const cudaError_t e = dtype == GS_F16 ? (p.wide ? sizes(__half(), float(), q[k]) : sizes(__half(), __half(), q[k]))
                          : p.wide        ? sizes(__nv_bfloat16(), float(), q[k])
                                          : sizes(__nv_bfloat16(), __nv_bfloat16(), q[k]);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace gs
