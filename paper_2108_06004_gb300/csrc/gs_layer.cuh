// Shared declarations of the recurrent layer's operators: element types, the counter-based
// generator, parameter blocks and launchers called by the C ABI in gs_layer.cu.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gs_common.cuh"

namespace gs {

// Status and thread-local message of a failing call (defined beside gs_last_error).
gs_status record_failure(gs_status st, const char* msg) noexcept;
gs_status record_cuda_failure(cudaError_t e, const char* what) noexcept;

// ---- element types ------------------------------------------------------------------------
// Two adjacent elements as one load or store, computed on in fp32.  The only rounding to fewer
// bits is that of a stored result to the tensors' own type.
template <typename E> struct Pack2;
template <> struct Pack2<float> {
  using type = float2;
  static __device__ __forceinline__ float2 up(float2 v) { return v; }
  static __device__ __forceinline__ float2 down(float2 v) { return v; }
};
template <> struct Pack2<__half> {
  using type = __half2;
  static __device__ __forceinline__ float2 up(__half2 v) { return __half22float2(v); }
  static __device__ __forceinline__ __half2 down(float2 v) { return __floats2half2_rn(v.x, v.y); }
};
template <> struct Pack2<__nv_bfloat16> {
  using type = __nv_bfloat162;
  // bf16 is the upper half of an fp32 value
  static __device__ __forceinline__ float2 up(__nv_bfloat162 v) {
    const uint32_t u = *reinterpret_cast<const uint32_t*>(&v);
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
  }
  static __device__ __forceinline__ __nv_bfloat162 down(float2 v) { return __floats2bfloat162_rn(v.x, v.y); }
};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename E> __device__ __forceinline__ E from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Rows are worked on in groups of eight adjacent elements, in one of three ways.
//   kEven: every row starts at a 16-byte boundary (by the element's size: at eight elements) and
//     has whole groups only.
//   kTogether: all tensors of a call have their rows at the same distance, `lead` elements, past
//     a boundary.  The groups start at the boundaries: group k of a row holds columns 8k - lead ...
//     8k - lead + 7, so that all groups but a row's first and last move as 16-byte words whatever
//     the width and the alignment are.  Contiguous tensors of an odd width are of this kind.
//     The first and last groups are read as whole words too (`inner`) where the rows before and
//     after, or the space between rows, are what lies beside them.
//   kApart: anything else; elements move one by one.
enum Layout { kApart, kEven, kTogether };

struct Span {
  int col;     // of the group's first element; negative where the row starts inside the group
  int lo, hi;  // the elements of the group that exist
  __device__ __forceinline__ bool some() const { return hi > lo; }
  __device__ __forceinline__ bool whole() const { return hi - lo == 8; }
};
template <int L>
__device__ __forceinline__ Span span(int64_t group, int lead, int64_t cols) {
  const int64_t col = group * 8 - (L == kTogether ? lead : 0);
  if (L == kEven) return Span{(int)col, 0, col < cols ? 8 : 0};
  return Span{(int)col, col < 0 ? (int)-col : 0, cols - col < 8 ? (int)(cols - col) : 8};
}
// lead of a row of `stride` elements from the row before, where row 0 has `first`.
template <int L>
__device__ __forceinline__ int lead_of(int64_t row, int64_t stride, int first) {
  return L == kTogether ? (int)(((uint32_t)row * (uint32_t)stride + (uint32_t)first) & 7u) : 0;
}

// A group as it is in memory, so that loads can be issued well before their values are needed.
template <typename E>
struct Raw8 {
  uint4 q[sizeof(E) / 2];
};

template <typename E, int L>
__device__ __forceinline__ Raw8<E> fetch8(const E* p, const Span& g, bool inner = false) {
  Raw8<E> r;
  if (L == kEven || (L == kTogether && (g.whole() || inner))) {
#pragma unroll
    for (int k = 0; k < (int)(sizeof(E) / 2); ++k) r.q[k] = reinterpret_cast<const uint4*>(p)[k];
  } else {
    E* e = reinterpret_cast<E*>(&r);
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = j >= g.lo && j < g.hi ? p[j] : from_f32<E>(0.f);
  }
  return r;
}

// Its values, zero where there is no element.
template <typename E, int L>
__device__ __forceinline__ void unpack8(const Raw8<E>& r, const Span& g, float (&v)[8]) {
  const typename Pack2<E>::type* h = reinterpret_cast<const typename Pack2<E>::type*>(&r);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = Pack2<E>::up(h[j]);
    v[2 * j] = f.x;
    v[2 * j + 1] = f.y;
  }
  if (L == kTogether && !g.whole()) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j >= g.lo && j < g.hi ? v[j] : 0.f;
  }
}

template <typename E, int L>
__device__ __forceinline__ void store8(E* p, const Span& g, const float (&v)[8]) {
  if (L == kEven || (L == kTogether && g.whole())) {
    constexpr int Q = sizeof(E) / 2;
    uint4 raw[Q];
    typename Pack2<E>::type* h = reinterpret_cast<typename Pack2<E>::type*>(raw);
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = Pack2<E>::down(make_float2(v[2 * j], v[2 * j + 1]));
#pragma unroll
    for (int q = 0; q < Q; ++q) reinterpret_cast<uint4*>(p)[q] = raw[q];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= g.lo && j < g.hi) p[j] = from_f32<E>(v[j]);
  }
}

// ---- counter-based generator ----------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC 2011): ten rounds of two 32 x 32 -> 64 bit
// products over a 128-bit counter.  The key depends on the seed alone, so its ten pairs are
// worked out on the host and read as kernel constants.
struct DropParams {
  uint32_t key[20];
  uint64_t offset;     // upper half of the counter
  uint32_t threshold;  // dropped when the element's 16 bits are below it; 0 ... 65536
  float scale;         // 65536 / (65536 - threshold), 0 when everything is dropped
};

__device__ __forceinline__ uint4 philox(uint64_t block, const DropParams& d) {
  uint32_t x0 = (uint32_t)block, x1 = (uint32_t)(block >> 32);
  uint32_t x2 = (uint32_t)d.offset, x3 = (uint32_t)(d.offset >> 32);
#pragma unroll
  for (int k = 0; k < 10; ++k) {
    const uint64_t m0 = (uint64_t)x0 * 0xD2511F53u, m1 = (uint64_t)x2 * 0xCD9E8D57u;
    x0 = (uint32_t)(m1 >> 32) ^ x1 ^ d.key[2 * k];
    x1 = (uint32_t)m1;
    x2 = (uint32_t)(m0 >> 32) ^ x3 ^ d.key[2 * k + 1];
    x3 = (uint32_t)m0;
  }
  return make_uint4(x0, x1, x2, x3);
}

// Dropout of the eight elements of a block.  Element 2w + h takes half h of word w.  A half is
// compared in the upper 16 bits of a word, where what lies below it does not matter.  A dropped
// element is zero whatever its value was (infinities and NaN included).
__device__ __forceinline__ void drop_block(float (&v)[8], uint64_t block, const DropParams& d) {
  const uint4 w = philox(block, d);
  const uint32_t word[4] = {w.x, w.y, w.z, w.w}, least = d.threshold << 16;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float2 s = __fmul2_rn(make_float2(v[2 * q], v[2 * q + 1]), make_float2(d.scale, d.scale));
    v[2 * q] = word[q] << 16 >= least ? s.x : 0.f;
    v[2 * q + 1] = word[q] >= least ? s.y : 0.f;
  }
}

// Bit j set: element 8 * block + j is kept.
__device__ __forceinline__ uint32_t keep_block(uint64_t block, const DropParams& d) {
  const uint4 w = philox(block, d);
  const uint32_t word[4] = {w.x, w.y, w.z, w.w}, least = d.threshold << 16;
  uint32_t bits = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    bits |= (word[q] << 16 >= least ? 1u : 0u) << (2 * q);
    bits |= (word[q] >= least ? 1u : 0u) << (2 * q + 1);
  }
  return bits;
}

// Dropout of the eight elements from `first` on, which lie in one block or in two.  `first` is
// negative where a row's first group starts before the first element of all; what does not exist
// may get any mask.
template <bool ALIGNED>
__device__ __forceinline__ void drop8(float (&v)[8], int64_t first, const DropParams& d) {
  if (d.threshold == 0) return;
  if (d.threshold > 0xFFFF) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    return;
  }
  const int64_t block = first >> 3;
  const uint32_t skip = (uint32_t)first & 7u;
  if (ALIGNED || skip == 0) {
    drop_block(v, (uint64_t)block, d);
  } else {
    const uint32_t bits = (keep_block((uint64_t)block, d) | keep_block((uint64_t)(block + 1), d) << 8) >> skip;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (bits >> j) & 1u ? v[j] * d.scale : 0.f;
  }
}

// ---- parameter blocks -----------------------------------------------------------------------
struct DropoutParams {
  const void* x;
  const void* residual;  // nullable
  void* out;
  int64_t x_stride, residual_stride, out_stride;
  int64_t rows, cols;
  int lead;     // of row 0
  bool spaced;  // every tensor's rows are at least eight elements apart
  DropParams drop;
};

struct NormForwardParams {
  const void* x;
  const void* residual;
  const float* weight;
  void* y;
  void* z;
  float* rstd;
  int64_t x_stride, residual_stride, y_stride, z_stride;
  int64_t rows;
  int32_t cols;
  int lead;
  bool spaced;
  float eps;
  DropParams drop;
};

struct NormBackwardParams {
  const void* dz;
  const void* dy;  // nullable
  const void* y;
  const float* weight;
  const float* rstd;
  void* dx;         // nullable
  void* dresidual;  // nullable
  float* partial;   // [CTAs][cols]
  int64_t dz_stride, dy_stride, y_stride, dx_stride, dresidual_stride;
  int64_t rows;
  int32_t cols;
  int lead;
  bool spaced;
  DropParams drop;
};

// One [B][T][D] tensor: element (b, t, d) at data + b*batch + t*token + d.
template <typename P>
struct Seq {
  P data;
  int64_t batch, token;
};

struct RecurrenceParams {
  CUtensorMap maps[7];      // x, r, i, dy, dx, dr, di as tiles, where those are used
  Seq<const void*> x, r, i, dy;
  Seq<void*> y, dx, dr, di;
  const float* decay;
  const float* h0;          // nullable
  const uint8_t* reset;     // nullable, [B][T]
  const int32_t* lengths;   // nullable, [B]
  float* h_last;            // nullable
  float* states;            // [B][states of a row][D]; written by the forward pass when not NULL
  const float* dh_last;     // nullable
  float* dh0;               // nullable
  float* partial;           // [B * cluster][D] sums of the decay's gradient
  int64_t B, T, D;
  float c;
  int32_t groups;           // channel groups of a row
  int32_t tile_tries, message_tries;  // of a wait, before it gives up
};
constexpr int32_t kMostTries = 1 << 20;
enum { kMapX, kMapR, kMapI, kMapDy, kMapDx, kMapDr, kMapDi };

struct RecurrenceStepParams {
  const void* x;
  const void* r;
  const void* i;
  void* y;
  int64_t x_stride, r_stride, i_stride, y_stride, state_stride;
  const float* decay;
  float* state;
  const int32_t* slots;  // nullable
  int64_t B, D, n_slots;
  float c;
};

// ---- launchers ------------------------------------------------------------------------------
cudaError_t launch_dropout(const DropoutParams& p, int dtype, Layout layout, cudaStream_t s);

constexpr int kSMs = 152;  // the sizes of grids are rules on it, so that results do not depend on a query
constexpr int kNormMaxCols = 16384;
int norm_backward_most_ctas(int64_t rows, int cols);
cudaError_t launch_norm_forward(const NormForwardParams& p, int dtype, Layout layout, cudaStream_t s);
cudaError_t launch_norm_backward(const NormBackwardParams& p, float* dweight, int dtype, Layout layout, cudaStream_t s);

// out[c] = sum over n rows of partial[row][c]; times -scale sigmoid(decay[c]) where decay is given
cudaError_t launch_column_sums(const float* partial, int64_t n, int64_t cols, const float* decay, float scale,
                               float* out, cudaStream_t s);

struct RecurrenceShape {
  int channels;      // of a CTA
  int cluster;       // CTAs that share a row's time
  int32_t groups;    // CTAs side by side over the channels
  unsigned grid;
};
RecurrenceShape recurrence_shape(int64_t B, int64_t T, int64_t D, int run, bool fp32);
int64_t recurrence_states(int64_t T);  // states kept of a row and channel
int64_t recurrence_partials(int64_t B, int64_t T, int64_t D);
// How the tensors can be moved: by tiles (16, every row starts at a multiple of 16 bytes), by copies of
// 4 bytes with two adjacent channels stored as one, or by single elements (the type's size).
cudaError_t launch_recurrence_forward(RecurrenceParams& p, int dtype, int unit, cudaStream_t s);
cudaError_t launch_recurrence_backward(RecurrenceParams& p, float* ddecay, int dtype, int unit, cudaStream_t s);
cudaError_t launch_recurrence_step(const RecurrenceStepParams& p, int dtype, bool pair, cudaStream_t s);

// launch() with dynamic shared memory and a cluster of `cluster` CTAs along x.
//
// Clusters are launched without programmatic serialization, and do not let the next kernel be
// scheduled early either (begin_cluster): their CTAs stay for the whole kernel where they are first
// put, and put among the last CTAs of another kernel they share SMs unevenly.  Forward and
// backward of 1x65536x1024 bf16 in turn took 481 us with it where 372 us, the sum of both, is right.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_cluster(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, int cluster,
                                  cudaStream_t s, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  if (cluster > 1) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
  } else {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}
// The start of a kernel that may run in clusters.
__device__ __forceinline__ void begin_cluster(int cluster) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (cluster == 1) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Calls f with the layout as a constant.
template <typename F>
inline cudaError_t with_layout(Layout layout, F&& f) {
  switch (layout) {
    case kEven: return f(std::integral_constant<int, kEven>());
    case kTogether: return f(std::integral_constant<int, kTogether>());
    default: return f(std::integral_constant<int, kApart>());
  }
}

// Calls f with a value of the element type that `dtype` names.
template <typename F>
inline cudaError_t with_type(int dtype, F&& f) {
  switch (dtype) {
    case GS_F32: return f(float());
    case GS_F16: return f(__half());
    default: return f(__nv_bfloat16());
  }
}

}  // namespace gs
