// A walk of linear attention in fp32 arithmetic, for every type, head size, stride and alignment (see
// attention.cuh).
//
// In blocks of 16 tokens, with w_n = e^(g n), i and j counted from the block's first token and S the state before it:
//   o_i = out_scale (w_{i+1} S' q_i + sum over j <= i of w_{i-j} (q_i . k_j) v_j),
//   S  <- w_16 S + in_scale sum over j of w_{15-j} k_j v_j'.
// (Backwards a token's decay comes after it: w_i for w_{i+1}, and w_{16-j} for w_{15-j}.)
// A CTA holds 32 columns of one head's state in the registers of its eight warps (four for more than 128 rows), a share of
// the rows each; two multiply-adds a state element and token, two rows an instruction.  8x2048x8x128 fp32 takes 4.39 ms for
// forward and backward (5.17 with every token added to the state by itself, 5.49 with one row an instruction too), a tenth of the
// fp32 pipes' rate: with two CTAs an SM a scheduler issues in half of the clocks, while the pipe that reads shared
// memory is busy for 62 % of them and the multiply-adds' for 46 %; every 16 bytes of keys feed two instructions only.
//
// Long rows are cut into pieces: the pieces' own sums, the states before them, then all outputs.
//
// Small problems wait for memory and for one another: train 5x333x3x40/72 fp32 takes 129 us for forward and backward, in
// pieces of 64 tokens of four blocks each (599 us with four warps, loads one by one and pieces of 128); the loads of a
// block are under way while the one before is worked on.
#include "attention.cuh"

namespace gs {
namespace {

constexpr int kTok = 16, kCols = 32;

template <typename E>
__device__ __forceinline__ const E* row_of(const HeadsIn& t, int batch, int64_t token, int head) {
  return static_cast<const E*>(t.data) + batch * t.batch + token * t.token + head / t.share * t.head;
}

// SUMS: only the piece's own sum, from a state of zero, into carry.
template <typename E, typename O, int ROWS, int kWarps, bool SUMS>
__global__ void __launch_bounds__(kWarps * 32)
k_attention(const __grid_constant__ AttentionWalks walks) {
  grid_begin();
  const uint32_t each = gridDim.x / walks.count, block = blockIdx.x % each;
  const AttentionParams& p = walks.of[blockIdx.x / each];
  constexpr int C = kWarps * ROWS, kThreadsA = kWarps * 32;  // contracted rows, with those that do not exist
  // rows of four floats more: sixteen keys at once lie in different banks
  __shared__ __align__(16) float q[SUMS ? 1 : kTok][C + 4], k[kTok][C + 4];
  __shared__ float v[kTok][kCols], weighted[kTok][kCols], part[SUMS ? 1 : kWarps][kTok][kCols], score[kTok][kTok + 1], power[kTok + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slices = (p.D + kCols - 1) / kCols;
  const int slice = block % slices, head = block / slices % p.H, item = block / slices / p.H;
  Piece w;
  if (!find_piece(p, item, w)) return;
  const int c0 = slice * kCols, cols = min(p.D - c0, kCols), col = c0 + lane;
  const bool mine = lane < cols;
  const float g = log_decay_of(p, head);
  if (threadIdx.x <= kTok) power[threadIdx.x] = expf(g * (float)threadIdx.x);
  float S[ROWS];
  const int64_t state = ((int64_t)w.sequence * p.H + head) * p.C * p.D;
  float* carry = p.carry + ((int64_t)item * p.H + head) * p.C * p.D;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int c = warp * ROWS + r;
    S[r] = 0.f;
    if (SUMS || c >= p.C || !mine) continue;
    if ((w.opens && w.ends) || p.chained)
      S[r] = p.first ? p.first[state + c * p.state_row + col * p.state_col] : 0.f;
    else
      S[r] = carry[(int64_t)c * p.D + col];
  }
  if (SUMS && (w.ends || w.t0 >= w.length)) return;  // nothing comes after it
  if (!SUMS && p.chained && w.t0 < w.length) {
    const Decay d = decay_of(g * (float)p.segment);
    for (int n = w.t0 / p.segment; n > 0; --n) {
      const float* u = carry - (int64_t)n * p.H * p.C * p.D;
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const int c = warp * ROWS + r;
        if (c < p.C && mine) S[r] = decayed(S[r], d, u[(int64_t)c * p.D + col]);
      }
    }
  }
  if (!SUMS && !p.offsets) {                          // tokens past the row's length
    for (int t = max(w.t0, w.length) + warp; t < min((int64_t)w.t0 + p.segment, p.T); t += kWarps)
      if (mine)
        static_cast<O*>(p.o.data)[w.batch * p.o.batch + t * p.o.token + head * p.o.head + col] = from_f32<O>(0.f);
  }
  const int after = p.back ? 0 : 1;
  // The next block's rows are under way while a block is worked on.
  constexpr int PER = kTok * C / kThreadsA, VPER = kTok / kWarps;
  E next_q[SUMS ? 1 : PER], next_k[PER], next_v[VPER];
  const auto fetch = [&](int t0) {
    const int n = min(kTok, w.t1 - t0);
    const auto token = [&](int j) { return w.start + (p.back ? w.length - 1 - (t0 + j) : t0 + j); };
#pragma unroll
    for (int a = 0; a < PER; ++a) {
      const int j = (a * kThreadsA + (int)threadIdx.x) / C, c = (a * kThreadsA + (int)threadIdx.x) % C;
      const bool some = j < n && c < p.C;
      next_k[a] = some ? row_of<E>(p.k, w.batch, token(j), head)[c] : from_f32<E>(0.f);
      if constexpr (!SUMS) next_q[a] = some ? row_of<E>(p.q, w.batch, token(j), head)[c] : from_f32<E>(0.f);
    }
#pragma unroll
    for (int a = 0; a < VPER; ++a) {
      const int j = a * kWarps + warp;
      next_v[a] = j < n && mine ? row_of<E>(p.v, w.batch, token(j), head)[col] : from_f32<E>(0.f);
    }
  };
  if (w.t0 < w.t1) fetch(w.t0);
  for (int t0 = w.t0; t0 < w.t1; t0 += kTok) {
    const int n = min(kTok, w.t1 - t0);
    const auto token = [&](int j) { return w.start + (p.back ? w.length - 1 - (t0 + j) : t0 + j); };
    __syncthreads();
#pragma unroll
    for (int a = 0; a < PER; ++a) {
      const int j = (a * kThreadsA + (int)threadIdx.x) / C, c = (a * kThreadsA + (int)threadIdx.x) % C;
      k[j][c] = to_f32(next_k[a]);
      if constexpr (!SUMS) q[j][c] = to_f32(next_q[a]);
    }
#pragma unroll
    for (int a = 0; a < VPER; ++a) {
      const int j = a * kWarps + warp;
      v[j][lane] = to_f32(next_v[a]);
      weighted[j][lane] = j < n ? v[j][lane] * (p.in_scale * power[n - j - after]) : 0.f;
    }
    if (t0 + kTok < w.t1) fetch(t0 + kTok);
    __syncthreads();
    if constexpr (!SUMS) {
      // a score or two each thread, those above the diagonal zero
      for (int at = threadIdx.x; at < kTok * kTok; at += kThreadsA) {
        const int i = at / kTok, j = at % kTok;
        float sum = 0.f;
        if (j <= i) {
          float four[4] = {0.f, 0.f, 0.f, 0.f};  // sums that do not wait for one another
#pragma unroll 8
          for (int c = 0; c < C; c += 4) {
            const float4 a = *reinterpret_cast<const float4*>(&q[i][c]), b = *reinterpret_cast<const float4*>(&k[j][c]);
            four[0] = fmaf(a.x, b.x, four[0]);
            four[1] = fmaf(a.y, b.y, four[1]);
            four[2] = fmaf(a.z, b.z, four[2]);
            four[3] = fmaf(a.w, b.w, four[3]);
          }
          sum = ((four[0] + four[1]) + (four[2] + four[3])) * (power[i - j] * p.in_scale);
        }
        score[i][j] = sum;
      }
      // two rows an instruction, and eight tokens at a time, whose sums fit the registers
#pragma unroll
      for (int i0 = 0; i0 < kTok; i0 += 8) {
        float2 o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = make_float2(0.f, 0.f);
#pragma unroll
        for (int r = 0; r < ROWS; r += 4)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 a = *reinterpret_cast<const float4*>(&q[i0 + i][warp * ROWS + r]);
            o[i] = __ffma2_rn(make_float2(a.x, a.y), make_float2(S[r], S[r + 1]), o[i]);
            o[i] = __ffma2_rn(make_float2(a.z, a.w), make_float2(S[r + 2], S[r + 3]), o[i]);
          }
#pragma unroll
        for (int i = 0; i < 8; ++i) part[warp][i0 + i][lane] = o[i].x + o[i].y;
      }
    }
    // The block's own sum is made from zero and added to the state once: added token by token, a state that decays slowly is
    // rounded at its own size sixteen times as often. A few rows at a time, whose sums do not wait for one another; where a
    // thread has 64 of them, its registers are enough for sixteen and the keys of four tokens.
    const Decay d = decay_of(g * (float)n);
    constexpr int AT_ONCE = ROWS < 8 ? ROWS : ROWS < 64 ? 8 : 16, AHEAD = ROWS < 64 ? kTok : 4;
#pragma unroll
    for (int r0 = 0; r0 < ROWS; r0 += AT_ONCE) {
      float2 u[AT_ONCE / 2];
#pragma unroll
      for (int r = 0; r < AT_ONCE / 2; ++r) u[r] = make_float2(0.f, 0.f);
#pragma unroll AHEAD
      for (int j = 0; j < kTok; ++j) {
        const float x = weighted[j][lane];
#pragma unroll
        for (int r = 0; r < AT_ONCE; r += 4) {
          const float4 a = *reinterpret_cast<const float4*>(&k[j][warp * ROWS + r0 + r]);
          u[r / 2] = __ffma2_rn(make_float2(a.x, a.y), make_float2(x, x), u[r / 2]);
          u[r / 2 + 1] = __ffma2_rn(make_float2(a.z, a.w), make_float2(x, x), u[r / 2 + 1]);
        }
      }
#pragma unroll
      for (int r = 0; r < AT_ONCE; ++r) S[r0 + r] = decayed(S[r0 + r], d, r % 2 ? u[r / 2].y : u[r / 2].x);
    }
    if constexpr (!SUMS) {
      __syncthreads();
      for (int i = warp; i < n; i += kWarps) {
        float sum = 0.f, near = 0.f;
#pragma unroll
        for (int q = 0; q < kWarps; ++q) sum += part[q][i][lane];
#pragma unroll
        for (int j = 0; j < kTok; ++j) near = fmaf(score[i][j], v[j][lane], near);
        sum = fmaf(sum, power[i + after], near) * p.out_scale;
        if (mine)
          static_cast<O*>(p.o.data)[w.batch * p.o.batch + token(i) * p.o.token + head * p.o.head + col] = from_f32<O>(sum);
      }
    }
  }
  if (!SUMS && (!w.ends || !p.last)) return;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int c = warp * ROWS + r;
    if (c >= p.C || !mine) continue;
    if (SUMS)
      carry[(int64_t)c * p.D + col] = S[r];
    else
      p.last[state + c * p.state_row + col * p.state_col] = S[r];
  }
}

// The states before a sequence's pieces from the pieces' own sums, in their place.
__global__ void __launch_bounds__(256)
k_attention_carry(const __grid_constant__ AttentionWalks walks) {
  grid_begin();
  const uint32_t each = gridDim.x / walks.count;
  const AttentionParams& p = walks.of[blockIdx.x / each];
  const int64_t size = (int64_t)p.C * p.D;
  const int blocks = (int)((size + 255) / 256), row = blockIdx.x % each / blocks;
  const int sequence = row / p.H, head = row % p.H;
  const int n = pieces_of(length_of(p, sequence), p.segment);
  if (n == 1) return;  // nothing is read from its place
  const int64_t item0 = p.offsets ? pieces_before(p, sequence) : (int64_t)sequence * p.segments;
  const Decay d = decay_of(log_decay_of(p, head) * (float)p.segment);
  const int64_t at = (int64_t)(blockIdx.x % each % blocks) * 256 + threadIdx.x;
  if (at >= size) return;
  const int64_t c = at / p.D, e = at % p.D;
  float S = p.first ? p.first[((int64_t)sequence * p.H + head) * size + c * p.state_row + e * p.state_col] : 0.f;
  const int last = (int)min((int64_t)n, p.items - item0) - 1;  // the last piece's own sum is not known, nor needed
  const int64_t step = p.H * size;
  float* x = p.carry + (item0 * p.H + head) * size + at;
  constexpr int AHEAD = 16;
  for (int k0 = 0; k0 <= last; k0 += AHEAD) {
    float u[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) u[k] = k0 + k < last ? x[(k0 + k) * step] : 0.f;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (k0 + k > last) break;
      x[(k0 + k) * step] = S;
      S = decayed(S, d, u[k]);
    }
  }
}

template <typename E>
__global__ void __launch_bounds__(256)
k_head_sums(const __grid_constant__ HeadSumParams p) {
  grid_begin();
  const int64_t n = p.B * p.T * p.K * p.D;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < n; at += (int64_t)gridDim.x * 256) {
    const int64_t row = at / p.D, d = at % p.D, token = row / p.K, t = token % p.T, b = token / p.T;
    if (p.offsets && (t < p.offsets[0] || t >= p.offsets[p.sequences])) continue;
    const float* x = p.part + row * p.share * p.D + d;
    float sum = 0.f;
    for (int k = 0; k < p.share; ++k) sum += x[(int64_t)k * p.D];
    static_cast<E*>(p.out.data)[b * p.out.batch + t * p.out.token + row % p.K * p.out.head + d] = from_f32<E>(sum);
  }
}

template <typename E, typename O, int ROWS, int WARPS>
cudaError_t walk(const AttentionWalks& walks, cudaStream_t s) {
  const AttentionParams& p = walks.of[0];
  const dim3 grid((unsigned)((int64_t)walks.count * p.items * p.H * ((p.D + kCols - 1) / kCols)));
  if (p.segments > 1) {
    cudaError_t e = launch(k_attention<E, O, ROWS, WARPS, true>, grid, dim3(WARPS * 32), s, walks);
    if (e != cudaSuccess) return e;
    if (!p.chained) e = launch_attention_carry(walks, s);
    if (e != cudaSuccess) return e;
  }
  return launch(k_attention<E, O, ROWS, WARPS, false>, grid, dim3(WARPS * 32), s, walks);
}

}  // namespace

cudaError_t launch_attention_carry(const AttentionWalks& walks, cudaStream_t s) {
  const AttentionParams& p = walks.of[0];
  return launch(k_attention_carry, dim3((unsigned)(walks.count * (((int64_t)p.C * p.D + 255) / 256 * p.B * p.H))), dim3(256), s, walks);
}

AttentionShape attention_shape(int64_t B, int64_t T, int64_t H, int C, int D, int dtype, bool packed) {
  AttentionShape shape;
  const bool mma = for_tensor_cores(C, D, dtype);
  const int columns = mma ? (D <= 64 ? 64 : 128) : kCols;
  const int64_t heads = H * ((D + columns - 1) / columns), ctas = (packed ? 1 : B) * heads;
  // CTAs of a walk that share the device: for the fp32 one as many as registers leave room for, and two waves of those of more
  // than 128 rows (train 2x2048x8x32 fp32 154 us, 193 with three an SM; 4x1000x16x64 721, 817 with three and 850 with two;
  // 1x4096x8x128 1195, 1319 with three and 1287 with four; 1x4096x8x256 bf16 forward 1392, 1535 with three and 1559 with two)
  const int64_t slots = (int64_t)kSMs * (mma ? (C <= 64 && D <= 64 ? 2 : 1) : C > 64 && C <= 128 ? 2 : 4);
  // Rows are cut where there are too few of them: keys and values are then read twice, which costs about six tenths of a walk.
  // That is worth it up to three eighths of what the device holds: B x 2048 x 16 x 128 bf16 forward takes 94 us cut and 100
  // whole with 48 heads in all on 152 SMs, 137 and 100 with 64; heads of 64, 70 and 76 with 96 heads in 304 places, 98 and 78 with 128.
  // Packed sequences are of any length: where there are enough of them, only those are cut that are longer than three CTAs' fair
  // shares (train 24 in 32768x16x64 bf16 550 us, 611 with two shares, 668 with one, 547 with five; 200 in as many tokens 1021,
  // 1352, 1363 and 1012).
  const bool enough = (packed ? B : 1) * ctas * 16 >= slots * 6;
  int64_t segment = T;
  if (packed || !enough) segment = (T * ctas + slots - 1) / slots * (enough ? 3 : 1);
  const int64_t unit = mma ? 128 : 64;
  segment = segment < unit ? unit : (segment + unit - 1) / unit * unit;
  if (segment >= T) segment = T > 0 ? T : 1;
  shape.segment = (int32_t)segment;
  shape.segments = (int32_t)(T > 0 ? (T + segment - 1) / segment : 1);
  shape.items = packed ? B + T / segment : B * shape.segments;
  return shape;
}

cudaError_t launch_attention(const AttentionWalks& walks, int dtype, cudaStream_t s) {
  const AttentionParams& p = walks.of[0];
  if (for_tensor_cores(p.C, p.D, dtype)) {
    bool taken;
    const cudaError_t e = launch_attention_mma(walks, dtype, s, taken);
    if (taken || e != cudaSuccess) return e;
  }
  const auto rows = [&](auto e, auto o) {
    using E = decltype(e);
    using O = decltype(o);
    return p.C <= 32    ? walk<E, O, 4, 8>(walks, s)
           : p.C <= 64  ? walk<E, O, 8, 8>(walks, s)
           : p.C <= 128 ? walk<E, O, 16, 8>(walks, s)
                        : walk<E, O, 64, 4>(walks, s);
  };
  return with_type(dtype, [&](auto e) { return p.wide ? rows(e, float()) : rows(e, e); });
}

cudaError_t launch_head_sums(const HeadSumParams& p, int dtype, cudaStream_t s) {
  const int64_t n = (p.B * p.T * p.K * p.D + 255) / 256;
  return with_type(dtype, [&](auto e) {
    return launch(k_head_sums<decltype(e)>, dim3((unsigned)(n < kSMs * 8 ? n : kSMs * 8)), dim3(256), s, p);
  });
}

}  // namespace gs
