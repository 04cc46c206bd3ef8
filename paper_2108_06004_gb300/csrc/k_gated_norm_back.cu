// Backward pass of the norms around a block:
//
//   m = y next_rstd,  u = dz w_next,  t = next_rstd (u - m mean(u m)) + dy,   dresidual = t
//   n = x rstd,  e = scale t,  dgate = e n w act'(gate),  p = e act(gate) w,
//   dx = rstd (p - n mean(p n)),  dw = sum over rows of e act(gate) n,  dw_next = sum over rows of dz m
//
// Every tensor is read and written once.  A CTA takes rows in turn; the weights' gradients are summed by
// each thread over its rows, whose columns and group are the same, then over the CTAs by a last kernel, in a fixed
// order.  Bound by memory, with the arithmetic close behind: 32768x4096 bf16 takes 422 us (75 % of the copy rate), 8192x16x128
// fp16 by heads 43 us (58 %).  Two reductions a row, one row ahead in registers: 661 us; one reduction: 532; what the results
// need of a row in registers, two rows ahead in shared memory: 502; rstd copied once a warp and not by every thread: 422.
#include <atomic>
#include <numeric>

#include "gated_norm.cuh"

namespace gs {
namespace {

using namespace norm;

// Rows that are whole 16-byte words are copied ahead into shared memory, each thread its own words, while the rows before are
// worked on.
template <typename E, int TPR, int V, int L>
constexpr bool kAhead = L == kEven && V == 1 && TPR <= 512;
template <typename E>
constexpr int kStages = sizeof(E) == 2 ? 3 : 2;  // rows in shared memory
// Threads of an SM: what registers leave room for.
constexpr int resident(int tpr) { return tpr <= 512 ? 512 : 1024; }
constexpr int kInputs = 5;
enum { kX, kGate, kDy, kDz, kY };

__device__ __forceinline__ void copy_word(uint4* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

__device__ __forceinline__ void copy_float(float* to, const float* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

// A row's two means come from three sums of one pass, and what the results need of it stays in registers: with
//   A = scale rstd act(gate),  G = scale rstd x w act'(gate),  t' = next_rstd u + dy,
// t is t' - y next_rstd^2 mean(u m), dgate = t G, dw += t A x, dx = t A w - x rstd^2 mean(p n), and
//   mean(p n) = mean(A w x t') - next_rstd^2 mean(u m) mean(A w x y).
template <typename E, int TPR, int V, int L>
__global__ void __launch_bounds__(kCtaThreads<TPR>, resident(TPR) / kCtaThreads<TPR>)
k_gated_norm_back(const __grid_constant__ GatedNormBackParams p, int outer) {
  grid_begin();
  __shared__ float scratch[2][3][32];
  constexpr int RPC = kRowsPerCta<TPR>;
  // [rows][inputs][words of a group][threads] and [rows][2][warps or, where they are more, rows] for rstd where rows are copied ahead; at the end, where RPC > 1 and a row is one
  // group, [RPC][width]
  extern __shared__ __align__(16) float fold[];
  constexpr bool AHEAD = kAhead<E, TPR, V, L>;
  constexpr int WORDS = sizeof(E) / 2, THREADS = kCtaThreads<TPR>, STAGES = kStages<E>;
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  // a thread's rows, `step` apart, have the same lead and the same group
  const int64_t step = (int64_t)gridDim.x * RPC, first = (int64_t)blockIdx.x * RPC;
  const int lead = lead_of<L>(first + sub, p.x_stride, p.lead);
  const Gate<E> gate(p.act);
  Eight dw[V], dnext[V], weight[V], follow[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) dw[v][j] = dnext[v][j] = weight[v][j] = follow[v][j] = two(0.f);
    const Span s = span<L>(v * TPR + lane, lead, p.width);
    if (!s.some()) continue;
    group_weight8<L>(p.weight, s, lead, p.width, p.groups, first + sub, reinterpret_cast<float(&)[8]>(weight[v]));
    if (p.dz) weight8<L>(p.next_weight, s, lead, p.width, reinterpret_cast<float(&)[8]>(follow[v]));
  }
  const void* const input[kInputs] = {p.x, p.gate, p.dy, p.dz, p.y};
  const int64_t stride[kInputs] = {p.x_stride, p.gate_stride, p.dy_stride, p.dz_stride, p.y_stride};
  uint4* const ahead = reinterpret_cast<uint4*>(fold) + threadIdx.x;
  constexpr int SHARERS = TPR < 32 ? TPR : 32, SLOTS = THREADS / SHARERS;  // threads that share a copy of a row's rstd
  float* const rstds = fold + STAGES * kInputs * WORDS * THREADS * 4 + threadIdx.x / SHARERS;
  const auto copy = [&](int64_t row, int stage) {
    if (row < p.rows) {
      const Span s = span<L>(lane, lead, p.width);
      if (s.some()) {
#pragma unroll
        for (int k = 0; k < kInputs; ++k) {
          if (!input[k]) continue;
          const E* from = static_cast<const E*>(input[k]) + group_start(row, outer, stride[k], p.width) + s.col;
#pragma unroll
          for (int q = 0; q < WORDS; ++q) copy_word(ahead + ((stage * kInputs + k) * WORDS + q) * THREADS, from + q * (16 / sizeof(E)));
        }
      }
      if (threadIdx.x % SHARERS == 0) {
        copy_float(rstds + stage * 2 * SLOTS, p.rstd + row);
        if (p.dz) copy_float(rstds + (stage * 2 + 1) * SLOTS, p.next_rstd + row);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if constexpr (AHEAD) {
#pragma unroll
    for (int k = 0; k + 1 < STAGES; ++k) copy(first + sub + k * step, k);
  }
  int turn = 0, stage = 0;
  for (int64_t row0 = first; row0 < p.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + sub;
    const bool live = row < p.rows, inner = p.spaced && row > 0 && row + 1 < p.rows;
    const auto put = [&](void* t, int64_t stride, const Span& s, const Eight& v) {
      store8<E, L>(static_cast<E*>(t) + group_start(row, outer, stride, p.width) + s.col, s, reinterpret_cast<const float(&)[8]>(v));
    };
    Raw8<E> raw[kInputs][V];
    float rstd = 0.f, next_rstd = 0.f;
    if constexpr (AHEAD) {
      copy(row + (STAGES - 1) * step, stage == 0 ? STAGES - 1 : stage - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
#pragma unroll
      for (int k = 0; k < kInputs; ++k)
        if (input[k]) {
#pragma unroll
          for (int q = 0; q < WORDS; ++q) raw[k][0].q[q] = ahead[((stage * kInputs + k) * WORDS + q) * THREADS];
        }
      __syncwarp();
      rstd = rstds[stage * 2 * SLOTS];
      next_rstd = p.dz ? rstds[(stage * 2 + 1) * SLOTS] : 0.f;
      stage = stage + 1 == STAGES ? 0 : stage + 1;
    } else if (live) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Span s = span<L>(v * TPR + lane, lead, p.width);
        if (!s.some()) continue;
#pragma unroll
        for (int k = 0; k < kInputs; ++k)
          if (input[k])
            raw[k][v] = fetch8<E, L>(static_cast<const E*>(input[k]) + group_start(row, outer, stride[k], p.width) + s.col, s, inner);
      }
      rstd = p.rstd[row];
      if (p.dz) next_rstd = p.next_rstd[row];
    }
    const float factor = p.scale * rstd;
    float2 sum[3] = {two(0.f), two(0.f), two(0.f)};
    Eight A[V], G[V], t[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Span s = span<L>(v * TPR + lane, lead, p.width);
      if (!live || !s.some()) continue;
      Eight x, q, a;
      unpack<E, L>(raw[kX][v], s, x);
      if (p.gate) {
        unpack<E, L>(raw[kGate][v], s, a);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float2 slope;
          A[v][j] = mul(gate.value(a[j], slope), factor);
          G[v][j] = mul(mul(slope, factor), mul(x[j], weight[v][j]));
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) A[v][j] = two(factor);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) q[j] = mul(mul(A[v][j], weight[v][j]), x[j]);
      if (p.dy) {
        unpack<E, L>(raw[kDy][v], s, t[v]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) t[v][j] = two(0.f);
      }
      if (p.dz) {
        Eight y;
        unpack<E, L>(raw[kDz][v], s, a);
        unpack<E, L>(raw[kY][v], s, y);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 r = mul(a[j], next_rstd), b = mul(y[j], r);  // zero where there is no element, as all sums are
          t[v][j] = fma(r, follow[v][j], t[v][j]);
          dnext[v][j] = add(dnext[v][j], b);
          sum[0] = fma(b, follow[v][j], sum[0]);
          sum[2] = fma(q[j], y[j], sum[2]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[1] = fma(q[j], t[v][j], sum[1]);
    }
    float sums[3] = {sum[0].x + sum[0].y, sum[1].x + sum[1].y, sum[2].x + sum[2].y};
    row_sums<TPR>(sums, scratch[turn]);
    // the same for every element: next_rstd^2 mean(u m) as a factor of y, and rstd mean(p n) as one of x
    const float part = 1.f / (float)p.width, from_y = sums[0] * part * next_rstd * next_rstd;
    const float from_x = (sums[1] - from_y * sums[2]) * part * rstd * -rstd;
    if (!live) continue;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Span s = span<L>(v * TPR + lane, lead, p.width);
      if (!s.some()) continue;
      Eight x;
      if (p.dz) {
        unpack<E, L>(raw[kY][v], s, x);
#pragma unroll
        for (int j = 0; j < 4; ++j) t[v][j] = fma(x[j], -from_y, t[v][j]);
      }
      if (p.dresidual) put(p.dresidual, p.dresidual_stride, s, t[v]);
      if (p.dgate) {
#pragma unroll
        for (int j = 0; j < 4; ++j) G[v][j] = mul(G[v][j], t[v][j]);
        put(p.dgate, p.dgate_stride, s, G[v]);
      }
      unpack<E, L>(raw[kX][v], s, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 e = mul(t[v][j], A[v][j]);
        dw[v][j] = fma(e, x[j], dw[v][j]);
        x[j] = fma(x[j], from_x, mul(e, weight[v][j]));
      }
      if (p.dx) put(p.dx, p.dx_stride, s, x);
    }
  }
  const int64_t n = (int64_t)gridDim.x * p.width;
  for (int which = 0; which < (p.next_weight ? 2 : 1); ++which) {
    // rows of sums: one of each CTA, or, where rows have several groups, of each of its rows
    const bool apart = p.groups > 1;
    float* part = p.partial + which * n + (int64_t)blockIdx.x * (apart ? RPC : 1) * p.width;
    float* to = RPC > 1 && !apart ? fold + sub * p.width : part + (apart ? sub * p.width : 0);
    if (RPC > 1 && !apart) __syncthreads();  // what was copied ahead has been used
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Span s = span<L>(v * TPR + lane, lead, p.width);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j >= s.lo && j < s.hi) to[s.col + j] = reinterpret_cast<const float(&)[8]>(which ? dnext[v] : dw[v])[j];
    }
    if (RPC > 1 && !apart) {
      __syncthreads();
      for (int col = threadIdx.x; col < p.width; col += blockDim.x) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < RPC; ++k) sum += fold[k * p.width + col];
        part[col] = sum;
      }
      __syncthreads();
    }
  }
}

// CTAs: as many as stay resident, the rows dealt round robin, so that a thread's rows share their group and (rows
// of a thread being a multiple of eight apart) their lead.
int64_t ctas_of(int64_t rows, int groups, const Shape& shape) {
  const int64_t need = (rows + shape.rows - 1) / shape.rows;
  const int64_t even = groups / std::gcd(groups, shape.rows);  // CTAs whose rows hold whole sets of groups
  int64_t most = (int64_t)kSMs * (resident(shape.tpr) / shape.threads);
  const int64_t unit = std::lcm(even, (int64_t)8);
  most = (most + unit - 1) / unit * unit;
  return need < most ? (need + even - 1) / even * even : most;
}

}  // namespace

// CTAs times the sums that each writes, for any alignment of the rows.
int64_t gated_norm_most_sums(int64_t rows, int groups, int wide_cols) {
  int64_t most = 0;
  for (int wide : {wide_cols, wide_cols + 7 <= kNormMaxCols ? wide_cols + 7 : wide_cols}) {
    const Shape shape = gated_shape(wide);
    const int64_t n = ctas_of(rows, groups, shape) * (groups > 1 ? shape.rows : 1);
    most = n > most ? n : most;
  }
  return most;
}

cudaError_t launch_gated_norm_backward(const GatedNormBackParams& p, int outer, float* dweight, float* dnext_weight,
                                       int dtype, Layout layout, cudaStream_t s) {
  if (width(p.width, layout) > kNormMaxCols) layout = kApart;
  const Shape shape = gated_shape(width(p.width, layout));
  const int64_t ctas = ctas_of(p.rows, p.groups, shape);
  if (ctas > 0) {
    const size_t fold = shape.rows > 1 && p.groups == 1 ? (size_t)shape.rows * p.width * sizeof(float) : 0;
    const cudaError_t err = with_type(dtype, [&](auto e) {
      using E = decltype(e);
      return with_gated_shape(shape, [&](auto tpr, auto v) {
        return with_layout(layout, [&](auto how) {
          constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value, L = decltype(how)::value;
          constexpr size_t copies = kAhead<E, TPR, V, L> ? (size_t)kStages<E> * kCtaThreads<TPR> * (kInputs * 8 * sizeof(E) + 2 * sizeof(float)) : 0;
          const auto kernel = k_gated_norm_back<E, TPR, V, L>;
          if constexpr (copies > 48 * 1024) {
            // shared memory beyond the default is asked for once per kernel and device
            static std::atomic<uint64_t> done{0};
            int dev = 0;
            cudaError_t e = cudaGetDevice(&dev);
            if (e != cudaSuccess) return e;
            const uint64_t bit = 1ull << (dev & 63);
            if (!(done.load(std::memory_order_acquire) & bit)) {
              e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)copies);
              if (e != cudaSuccess) return e;
              done.fetch_or(bit, std::memory_order_release);
            }
          }
          return launch_cluster(kernel, dim3((unsigned)ctas), dim3(shape.threads), copies > fold ? copies : fold, 1, s, p, outer);
        });
      });
    });
    if (err != cudaSuccess) return err;
  }
  const int64_t sums = p.groups > 1 ? ctas * shape.rows / p.groups : ctas;
  const cudaError_t err = launch_column_sums(p.partial, sums, (int64_t)p.groups * p.width, nullptr, 0.f, dweight, s);
  if (err != cudaSuccess || !p.next_weight) return err;
  return launch_column_sums(p.partial + ctas * p.width, ctas, p.width, nullptr, 0.f, dnext_weight, s);
}

}  // namespace gs
