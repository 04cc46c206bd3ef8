// Linear attention with a decay for each head: declarations shared by its kernels.
//
// The three gradients are linear attentions too.  With S_t = e^g S_{t-1} + k_t v_t' and its gradient
// R_t = e^g R_{t+1} + scale q_t do_t' (at the last token, that of the last state + scale q_t do_t'),
//   o_t = scale S_t' q_t,  dq_t = scale S_t do_t,  dv_t = R_t' k_t,  dk_t = R_t v_t,
// so each is a walk over the tokens, forwards or backwards, in which "queries" read a state that
// "keys" and "values" add to: (q, k, v) for o, (do, v, k) with S' for dq, (k, q, do) for dv and
// (v, do, q) with R' for dk.  A walk's state has `C` rows, which its queries contract, and `D` columns.
#pragma once

#include "gs_layer.cuh"

namespace gs {

// One [B][T][heads][D] tensor as a walk sees it: `share` heads of the walk in turn use one of it.
struct HeadsIn {
  const void* data;
  int64_t batch, token, head;
  int32_t share;
};
struct HeadsOut {
  void* data;
  int64_t batch, token, head;
};

struct AttentionParams {
  HeadsIn q, k, v;
  HeadsOut o;
  const float* log_decay;
  const float* first;   // nullable, [B][H][..]: element (c, d) of a state at c * state_row + d * state_col
  float* last;          // nullable, likewise
  float* carry;         // [items][H][C][D]: each piece's sum; then, where not `chained`, the state before it
  int64_t state_row, state_col;
  const int32_t* lengths;  // nullable, [B]
  const int32_t* offsets;  // nullable, [B + 1]
  int64_t B, T;
  int32_t H, C, D;
  int32_t segment;      // tokens of a piece
  int32_t segments;     // pieces of a row, where sequences are rows
  int32_t items;        // pieces of all sequences, at most
  float in_scale, out_scale;  // of what is added to the state, and of what is read from it
  int32_t back;         // walks from each sequence's end, and takes a token's decay after it
  int32_t wide;         // o is fp32, for heads that are summed after
  int32_t chained;      // each piece adds up the sums of those before it itself
  int32_t issue_tries, find_tries, work_tries;  // of the tensor core walk's waits, before they give up
};
// Walks that run at once: of the same C, D, wide and, where one of them gives its last state, all do.
struct AttentionWalks {
  AttentionParams of[3];
  int32_t count;
};

constexpr int kAttentionMaxHead = 256;
constexpr float kLeastLogDecay = -8192.f;

// A piece: walk positions [t0, t1) of a sequence of `length` tokens, whose token 0 is at `start`.
struct Piece {
  int64_t start;
  int32_t batch, sequence, length, t0, t1;
  bool opens, ends;   // the sequence's first piece, its last one
};

// (length + segment may be past 32 bits)
__device__ __forceinline__ int pieces_of(int length, int segment) { return length > 0 ? (length - 1) / segment + 1 : 1; }
__device__ __forceinline__ int length_of(const AttentionParams& p, int sequence) {
  if (p.offsets) {
    const int a = min(max(p.offsets[sequence], 0), (int)p.T), e = min(max(p.offsets[sequence + 1], 0), (int)p.T);
    return max(e - a, 0);
  }
  return p.lengths ? min(max(p.lengths[sequence], 0), (int)p.T) : (int)p.T;
}

// The first piece of a packed sequence, counted over all of them; called by whole warps.
__device__ __forceinline__ int64_t pieces_before(const AttentionParams& p, int sequence) {
  const int lane = threadIdx.x & 31;
  int64_t n = 0;
  for (int s = lane; s < sequence; s += 32) n += pieces_of(length_of(p, s), p.segment);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xFFFFFFFFu, n, o);
  return n;
}

// Piece `item`, for whole warps; false where there are not as many.
__device__ __forceinline__ bool find_piece(const AttentionParams& p, int item, Piece& w) {
  int segment;
  if (!p.offsets) {
    w.sequence = item / p.segments;
    segment = item % p.segments;
    w.batch = w.sequence;
    w.start = 0;
  } else {
    const int lane = threadIdx.x & 31;
    int64_t before = 0;
    int found = -1;
    segment = 0;
    for (int s0 = 0; s0 < p.B && found < 0; s0 += 32) {
      const int s = s0 + lane;
      int sum = s < p.B ? pieces_of(length_of(p, s), p.segment) : 0;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const int other = __shfl_up_sync(0xFFFFFFFFu, sum, o);
        if (lane >= o) sum += other;
      }
      const uint32_t past = __ballot_sync(0xFFFFFFFFu, before + sum > item);
      if (past) {
        const int at = __ffs(past) - 1;
        const int until = __shfl_sync(0xFFFFFFFFu, sum, at > 0 ? at - 1 : 0);
        found = s0 + at;
        segment = (int)(item - before - (at > 0 ? until : 0));
      }
      before += __shfl_sync(0xFFFFFFFFu, sum, 31);
    }
    if (found < 0) return false;
    w.sequence = found;
    w.batch = 0;
    w.start = min(max(p.offsets[found], 0), (int)p.T);
  }
  w.length = length_of(p, w.sequence);
  w.t0 = segment * p.segment;
  w.t1 = (int)min((int64_t)w.length, (int64_t)w.t0 + p.segment);
  w.opens = segment == 0;
  w.ends = segment == pieces_of(w.length, p.segment) - 1;
  return true;
}

// In [kLeastLogDecay, 0]; NaN stays what it is.
__device__ __forceinline__ float taken(float log_decay) {
  return isnan(log_decay) ? log_decay : fminf(fmaxf(log_decay, kLeastLogDecay), 0.f);
}
__device__ __forceinline__ float log_decay_of(const AttentionParams& p, int head) { return taken(p.log_decay[head]); }

// e^x for x <= 0 as a sum of a factor and a small rest, so that S e^x = fma(S, a, fma(S, b, ...)) is right to
// a rounding of S however often it is applied: a rounded e^x close to one would bias a state
// that many such steps make up.
struct Decay {
  float a, b;
};
__device__ __forceinline__ Decay decay_of(float x) { return x > -0.5f ? Decay{1.f, expm1f(x)} : Decay{expf(x), 0.f}; }
__device__ __forceinline__ float decayed(float s, const Decay& d, float add) { return fmaf(s, d.a, fmaf(s, d.b, add)); }

// Where rows have few pieces, each one adds up those before it itself, which saves a launch and grows with the square of
// their number. From cold: train 24 in 32768x16x64 bf16 packed, which seldom have more than one piece and never more than 7, 551 us,
// 611 with the launch; 3x2048x16x128 in 3 pieces 310 and 363; 4x1000x8x64 in 8 pieces 135 and 127; forward 1x8192x24x128 in 6
// pieces 141 and 124; 1x4096x16x64 in 16 pieces 53 and 46. The first state must stay as it is meanwhile.
constexpr int kChainedPieces = 8;

struct AttentionStepParams {
  HeadsIn q, k, v;
  HeadsOut o;
  const float* log_decay;
  float* state;
  int64_t state_stride, n_slots;
  const int32_t* slots;  // nullable
  int64_t B;
  int32_t H, Dk, Dv;
  float scale;
};

// out[row][d] = sum over `share` adjacent heads of part[row][share][d], rows of all tokens and heads.
struct HeadSumParams {
  const float* part;    // [B][T][K][share][D]
  HeadsOut out;
  const int32_t* offsets;
  int64_t B, T;
  int32_t sequences, K, share, D;
};

// ---- launchers ------------------------------------------------------------------------------
struct AttentionShape {
  int32_t segment, segments;
  int64_t items;
};
// The pieces of a walk.  Walks for the tensor cores have blocks of 128 tokens.
inline bool for_tensor_cores(int C, int D, int dtype) { return dtype != GS_F32 && C <= 128 && C % 8 == 0 && D % 8 == 0; }
AttentionShape attention_shape(int64_t B, int64_t T, int64_t H, int C, int D, int dtype, bool packed);
cudaError_t launch_attention_carry(const AttentionWalks& walks, cudaStream_t s);
// The walks on the tensor cores, where for_tensor_cores; not taken where a tensor's strides do not allow it.
cudaError_t launch_attention_mma(const AttentionWalks& walks, int dtype, cudaStream_t s, bool& taken);
cudaError_t launch_attention(const AttentionWalks& walks, int dtype, cudaStream_t s);
cudaError_t launch_head_sums(const HeadSumParams& p, int dtype, cudaStream_t s);
cudaError_t launch_attention_step(const AttentionStepParams& p, int dtype, bool vec, cudaStream_t s);

struct RotaryParams {
  HeadsIn x;
  HeadsOut out;
  const double* frequencies;
  const int32_t* positions;  // nullable, [B][T]
  int64_t first, B, T;
  int32_t H, D, R;
  float magnitude, sign;
  bool copy;                 // elements from R on
};
cudaError_t launch_rotary(const RotaryParams& p, int dtype, bool interleaved, bool vec, cudaStream_t s);

struct GatedNormParams {
  const void* x;
  const void* gate;      // nullable
  const void* residual;  // nullable
  const float* weight;
  const float* next_weight;  // nullable
  void* y;
  void* z;
  float* rstd;
  float* next_rstd;
  int64_t x_stride, gate_stride, residual_stride, y_stride, z_stride;
  int64_t rows;          // of groups: row r is group r % groups of row r / groups
  int32_t groups, width; // columns of a group
  int lead;
  bool spaced;
  int act;
  float scale, eps;
};
struct GatedNormBackParams {
  const void* dy;        // nullable
  const void* dz;        // nullable
  const void* x;
  const void* gate;
  const void* y;
  const float* weight;
  const float* next_weight;
  const float* rstd;
  const float* next_rstd;
  void* dx;
  void* dgate;
  void* dresidual;
  float* partial;        // [CTAs][width], twice with a next norm; [CTAs * rows of one][width] with several groups
  int64_t dy_stride, dz_stride, x_stride, gate_stride, y_stride, dx_stride, dgate_stride, dresidual_stride;
  int64_t rows;
  int32_t groups, width;
  int lead;
  bool spaced;
  int act;
  float scale;
};
// outer: 1 where the groups of all rows are evenly apart (a stride is then from group to group), else `groups`.
cudaError_t launch_gated_norm(const GatedNormParams& p, int outer, int dtype, Layout layout, cudaStream_t s);
int64_t gated_norm_most_sums(int64_t rows, int groups, int width);
cudaError_t launch_gated_norm_backward(const GatedNormBackParams& p, int outer, float* dweight, float* dnext_weight,
                                       int dtype, Layout layout, cudaStream_t s);

}  // namespace gs
