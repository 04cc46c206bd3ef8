// C ABI of the recurrent layer's operators: argument checks and parameter blocks.
#include <cmath>
#include <cstring>
#include <initializer_list>
#include <new>
#include <string>

#include "gs_layer.cuh"

namespace {

constexpr int64_t kMaxElements = int64_t(1) << 40;
constexpr int64_t kMaxStride = int64_t(1) << 45;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1;

gs_status bad(const std::string& msg) noexcept { return gs::record_failure(GS_ERR_INVALID_ARG, msg.c_str()); }

#define GS_TRY(expr)                \
  do {                              \
    const gs_status st__ = (expr);  \
    if (st__ != GS_OK) return st__; \
  } while (0)

#define GS_GUARD_BEGIN try {
#define GS_GUARD_END                                                             \
  }                                                                              \
  catch (const std::bad_alloc&) {                                                \
    return gs::record_failure(GS_ERR_OOM, "host allocation failed");             \
  }                                                                              \
  catch (...) {                                                                  \
    return gs::record_failure(GS_ERR_INVALID_ARG, "unexpected host exception");  \
  }

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
cudaStream_t as_stream(gs_stream s) { return reinterpret_cast<cudaStream_t>(s); }
int item(int32_t dtype) { return dtype == GS_F32 ? 4 : 2; }

gs_status check_type(int32_t dtype) {
  if (dtype != GS_F32 && dtype != GS_F16 && dtype != GS_BF16)
    return bad("dtype must be GS_F32, GS_F16 or GS_BF16, got " + std::to_string(dtype));
  return GS_OK;
}

// required: a NULL is refused
gs_status check_data(const void* p, int align, bool required, const char* name) {
  if (!p) return required ? bad(std::string(name) + " is NULL") : GS_OK;
  if (!aligned(p, (uintptr_t)align)) return bad(std::string(name) + " is not " + std::to_string(align) + "-byte aligned");
  return GS_OK;
}

gs_status check_stride(int64_t s, const char* name) {
  if (s < 0 || s > kMaxStride) return bad(std::string(name) + ": strides must lie in [0, 2^45]");
  return GS_OK;
}

gs_status check_matrix(const void* p, int64_t stride, int32_t dtype, bool required, const char* name) {
  GS_TRY(check_data(p, item(dtype), required, name));
  return p ? check_stride(stride, name) : GS_OK;
}

gs_status check_output(const void* p, int64_t stride, int64_t rows, int64_t cols, int32_t dtype, bool required,
                       const char* name) {
  GS_TRY(check_matrix(p, stride, dtype, required, name));
  if (p && rows > 1 && stride < cols) return bad(std::string(name) + ": rows overlap (stride below cols)");
  return GS_OK;
}

// n * unit <= kMaxElements without overflow
bool product_fits(int64_t a, int64_t b) { return a == 0 || b <= kMaxElements / a; }

gs_status check_shape(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0) return bad("rows and cols must not be negative");
  if (rows > kMaxRows || cols > kMaxElements || !product_fits(rows, cols))
    return bad("rows must be below 2^31 and rows * cols at most 2^40");
  return GS_OK;
}

// How the rows of these tensors lie to one another; `lead`: see gs::Layout.  Absent tensors agree
// with everything.
struct Matrix {
  const void* data;
  int64_t stride;
};
gs::Layout layout_of(std::initializer_list<Matrix> all, int64_t rows, int64_t cols, int32_t dtype, int* lead) {
  const Matrix* first = nullptr;
  *lead = 0;
  for (const Matrix& m : all) {
    if (!m.data) continue;
    const int at = (int)(reinterpret_cast<uintptr_t>(m.data) / item(dtype) % 8);
    if (!first) {
      first = &m;
      *lead = at;
    }
    if (at != *lead || (rows > 1 && (m.stride - first->stride) % 8 != 0)) {
      *lead = 0;
      return gs::kApart;
    }
  }
  const bool even = *lead == 0 && cols % 8 == 0 && (rows == 1 || !first || first->stride % 8 == 0);
  return even ? gs::kEven : gs::kTogether;
}

bool spaced(std::initializer_list<Matrix> all) {
  for (const Matrix& m : all)
    if (m.data && m.stride < 8) return false;
  return true;
}

gs_status make_drop(float p, uint64_t seed, uint64_t offset, gs::DropParams& d) {
  if (!(p >= 0.f && p <= 1.f)) return bad("p must lie in [0, 1]");
  d.threshold = (uint32_t)std::floor((double)p * 65536.0 + 0.5);
  d.scale = d.threshold < 65536 ? (float)(65536.0 / (65536 - d.threshold)) : 0.f;
  d.offset = offset;
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  for (int k = 0; k < 10; ++k) {
    d.key[2 * k] = k0;
    d.key[2 * k + 1] = k1;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return GS_OK;
}

gs_status dropout_impl(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, void* out,
                       int64_t out_stride, int64_t rows, int64_t cols, int32_t dtype, float p, uint64_t seed,
                       uint64_t offset, gs_stream stream) {
  GS_TRY(check_type(dtype));
  GS_TRY(check_shape(rows, cols));
  const bool some = rows > 0 && cols > 0;
  gs::DropoutParams q;
  std::memset(&q, 0, sizeof(q));
  GS_TRY(make_drop(p, seed, offset, q.drop));
  GS_TRY(check_matrix(x, x_stride, dtype, some, "x"));
  GS_TRY(check_matrix(residual, residual_stride, dtype, false, "residual"));
  GS_TRY(check_output(out, out_stride, rows, cols, dtype, some, "out"));
  if (!some) return GS_OK;
  q.x = x;
  q.residual = residual;
  q.out = out;
  q.x_stride = x_stride;
  q.residual_stride = residual_stride;
  q.out_stride = out_stride;
  q.rows = rows;
  q.cols = cols;
  // contiguous tensors are one row
  if (x_stride == cols && out_stride == cols && (!residual || residual_stride == cols)) {
    q.rows = 1;
    q.cols = rows * cols;
  }
  const std::initializer_list<Matrix> all = {{x, x_stride}, {residual, residual_stride}, {out, out_stride}};
  const gs::Layout layout = layout_of(all, q.rows, q.cols, dtype, &q.lead);
  // in place, what lies beside a row is being written while it is read
  q.spaced = spaced(all) && out != x && out != residual;
  const cudaError_t e = gs::launch_dropout(q, dtype, layout, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, "dropout launch");
}

gs_status check_norm(int64_t rows, int64_t cols) {
  GS_TRY(check_shape(rows, cols));
  if (cols < 1 || cols > GS_NORM_MAX_COLS)
    return bad("cols must lie in [1, " + std::to_string(GS_NORM_MAX_COLS) + "], got " + std::to_string(cols));
  return GS_OK;
}

size_t norm_ws_bytes(int64_t rows, int64_t cols) {
  const size_t n = (size_t)gs::norm_backward_most_ctas(rows, (int)cols) * (size_t)cols * sizeof(float);
  return n ? (n + 255) & ~size_t(255) : 256;
}

gs_status check_workspace(const void* ws, size_t bytes, size_t need, const char* size_call) {
  if (!ws || !aligned(ws, 256)) return bad("workspace is NULL or not 256-byte aligned");
  if (bytes < need) return bad(std::string("workspace too small: use ") + size_call);
  return GS_OK;
}

gs_status check_sequence_shape(int64_t B, int64_t T, int64_t D) {
  if (B < 0 || T < 0 || D < 0) return bad("B, T and D must not be negative");
  if (B > kMaxElements || T > kMaxRows || D > kMaxElements || !product_fits(B, D) || !product_fits(B * D, T))
    return bad("T must be below 2^31 and B * T * D at most 2^40");
  // one CTA for each row and 64 channels
  if ((D + 63) / 64 >= (int64_t(1) << 28) / (B > 0 ? B : 1)) return bad("B * ceil(D / 64) must be below 2^28");
  return GS_OK;
}

gs_status check_seq(const gs_seq* t, int32_t dtype, bool required, const char* name) {
  if (!t) return bad(std::string(name) + " is NULL");
  GS_TRY(check_data(t->data, item(dtype), required, name));
  GS_TRY(check_stride(t->batch_stride, name));
  return check_stride(t->token_stride, name);
}

// Rows (b, t) of D elements are apart when tokens are apart within a batch and batches from one
// another, or the other way round.
gs_status check_seq_output(const gs_seq* t, int64_t B, int64_t T, int64_t D, int32_t dtype, bool required,
                           const char* name) {
  GS_TRY(check_seq(t, dtype, required, name));
  const int64_t bs = B > 1 ? t->batch_stride : kMaxStride, ts = T > 1 ? t->token_stride : kMaxStride;
  const bool by_batch = ts >= D && (B <= 1 || bs >= (T - 1) * (T > 1 ? ts : 0) + D);
  const bool by_token = bs >= D && (T <= 1 || ts >= (B - 1) * (B > 1 ? bs : 0) + D);
  if (!by_batch && !by_token) return bad(std::string(name) + ": rows overlap");
  return GS_OK;
}

// whether every row starts at a multiple of `bytes`
bool rows_at(const gs_seq* t, int32_t dtype, int bytes) {
  return aligned(t->data, (uintptr_t)bytes) && t->batch_stride * item(dtype) % bytes == 0 &&
         t->token_stride * item(dtype) % bytes == 0;
}

// How the tensors of a call can be moved: 16 (tiles), 4 (with pairs of channels stored as one), or
// the type's size.  Tiles want coordinates that fit 32 bits.
int copy_unit(std::initializer_list<const gs_seq*> in, std::initializer_list<const gs_seq*> out, int64_t B, int64_t T,
              int64_t D, int32_t dtype) {
  bool tiles = D * item(dtype) % 16 == 0 && T < (1 << 30) && D < (1 << 30) && B < (1 << 30), words = true;
  for (const gs_seq* t : in) {
    tiles = tiles && rows_at(t, dtype, 16);
    words = words && rows_at(t, dtype, 4);
  }
  for (const gs_seq* t : out) {
    tiles = tiles && rows_at(t, dtype, 16);
    words = words && rows_at(t, dtype, 2 * item(dtype));
  }
  return tiles ? 16 : words ? 4 : item(dtype);
}

gs::Seq<const void*> in(const gs_seq* t) { return {t->data, t->batch_stride, t->token_stride}; }
gs::Seq<void*> out(const gs_seq* t) { return {t->data, t->batch_stride, t->token_stride}; }

size_t round256(size_t n) { return n ? (n + 255) & ~size_t(255) : 256; }

size_t states_bytes(int64_t B, int64_t T, int64_t D) {
  return round256((size_t)B * (size_t)gs::recurrence_states(T) * (size_t)D * sizeof(float));
}

size_t recurrence_ws_bytes(int64_t B, int64_t T, int64_t D) {
  return round256((size_t)gs::recurrence_partials(B, T, D) * (size_t)D * sizeof(float));
}

// Tries of the recurrence's waits in calls of this thread.
thread_local int32_t tile_tries = gs::kMostTries, message_tries = gs::kMostTries;

void set_tries(gs::RecurrenceParams& p) {
  p.tile_tries = tile_tries;
  p.message_tries = message_tries;
}

gs_status check_c(float c) {
  if (!(c > 0.f) || std::isinf(c)) return bad("c must be positive and finite");
  return GS_OK;
}

}  // namespace

extern "C" {

gs_status gs_dropout(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, void* out,
                     int64_t out_stride, int64_t rows, int64_t cols, int32_t dtype, float p, uint64_t seed,
                     uint64_t offset, gs_stream stream) {
  GS_GUARD_BEGIN
  return dropout_impl(x, x_stride, residual, residual_stride, out, out_stride, rows, cols, dtype, p, seed, offset,
                      stream);
  GS_GUARD_END
}

gs_status gs_dropout_backward(const void* dout, int64_t dout_stride, void* dx, int64_t dx_stride, int64_t rows,
                              int64_t cols, int32_t dtype, float p, uint64_t seed, uint64_t offset,
                              gs_stream stream) {
  GS_GUARD_BEGIN
  return dropout_impl(dout, dout_stride, nullptr, 0, dx, dx_stride, rows, cols, dtype, p, seed, offset, stream);
  GS_GUARD_END
}

gs_status gs_dropout_add_norm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                              const float* weight, void* y, int64_t y_stride, void* z, int64_t z_stride, float* rstd,
                              int64_t rows, int64_t cols, int32_t dtype, float p, uint64_t seed, uint64_t offset,
                              float eps, gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  GS_TRY(check_norm(rows, cols));
  if (!(eps >= 0.f) || std::isinf(eps)) return bad("eps must be finite and not negative");
  gs::NormForwardParams q;
  std::memset(&q, 0, sizeof(q));
  GS_TRY(make_drop(p, seed, offset, q.drop));
  const bool some = rows > 0;
  GS_TRY(check_matrix(x, x_stride, dtype, some, "x"));
  GS_TRY(check_matrix(residual, residual_stride, dtype, some, "residual"));
  GS_TRY(check_data(weight, 4, true, "weight"));
  GS_TRY(check_output(y, y_stride, rows, cols, dtype, some, "y"));
  GS_TRY(check_output(z, z_stride, rows, cols, dtype, some, "z"));
  GS_TRY(check_data(rstd, 4, some, "rstd"));
  if (!some) return GS_OK;
  q.x = x;
  q.residual = residual;
  q.weight = weight;
  q.y = y;
  q.z = z;
  q.rstd = rstd;
  q.x_stride = x_stride;
  q.residual_stride = residual_stride;
  q.y_stride = y_stride;
  q.z_stride = z_stride;
  q.rows = rows;
  q.cols = (int32_t)cols;
  q.eps = eps;
  const std::initializer_list<Matrix> all = {{x, x_stride}, {residual, residual_stride}, {y, y_stride}, {z, z_stride}};
  gs::Layout layout = layout_of(all, rows, cols, dtype, &q.lead);
  q.spaced = spaced(all) && y != x && y != residual;
  if (!aligned(weight, 16)) layout = gs::kApart;
  const cudaError_t e = gs::launch_norm_forward(q, dtype, layout, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, "dropout_add_norm launch");
  GS_GUARD_END
}

gs_status gs_dropout_add_norm_workspace_size(int64_t rows, int64_t cols, size_t* bytes) {
  GS_GUARD_BEGIN
  if (!bytes) return bad("bytes is NULL");
  GS_TRY(check_norm(rows, cols));
  *bytes = norm_ws_bytes(rows, cols);
  return GS_OK;
  GS_GUARD_END
}

gs_status gs_dropout_add_norm_backward(const void* dz, int64_t dz_stride, const void* dy, int64_t dy_stride,
                                       const void* y, int64_t y_stride, const float* weight, const float* rstd,
                                       void* dx, int64_t dx_stride, void* dresidual, int64_t dresidual_stride,
                                       float* dweight, int64_t rows, int64_t cols, int32_t dtype, float p,
                                       uint64_t seed, uint64_t offset, void* workspace, size_t workspace_bytes,
                                       gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  GS_TRY(check_norm(rows, cols));
  gs::NormBackwardParams q;
  std::memset(&q, 0, sizeof(q));
  GS_TRY(make_drop(p, seed, offset, q.drop));
  const bool some = rows > 0;
  GS_TRY(check_matrix(dz, dz_stride, dtype, some, "dz"));
  GS_TRY(check_matrix(dy, dy_stride, dtype, false, "dy"));
  GS_TRY(check_matrix(y, y_stride, dtype, some, "y"));
  GS_TRY(check_data(weight, 4, true, "weight"));
  GS_TRY(check_data(rstd, 4, some, "rstd"));
  GS_TRY(check_output(dx, dx_stride, rows, cols, dtype, false, "dx"));
  GS_TRY(check_output(dresidual, dresidual_stride, rows, cols, dtype, false, "dresidual"));
  GS_TRY(check_data(dweight, 4, true, "dweight"));
  GS_TRY(check_workspace(workspace, workspace_bytes, norm_ws_bytes(rows, cols), "gs_dropout_add_norm_workspace_size"));
  q.dz = dz;
  q.dy = dy;
  q.y = y;
  q.weight = weight;
  q.rstd = rstd;
  q.dx = dx;
  q.dresidual = dresidual;
  q.partial = static_cast<float*>(workspace);
  q.dz_stride = dz_stride;
  q.dy_stride = dy ? dy_stride : 0;
  q.y_stride = y_stride;
  q.dx_stride = dx ? dx_stride : 0;
  q.dresidual_stride = dresidual ? dresidual_stride : 0;
  q.rows = rows;
  q.cols = (int32_t)cols;
  const std::initializer_list<Matrix> all = {
      {dz, dz_stride}, {dy, dy_stride}, {y, y_stride}, {dx, dx_stride}, {dresidual, dresidual_stride}};
  gs::Layout layout = layout_of(all, rows, cols, dtype, &q.lead);
  q.spaced = spaced(all);
  if (!aligned(weight, 16)) layout = gs::kApart;
  const cudaError_t e = gs::launch_norm_backward(q, dweight, dtype, layout, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, "dropout_add_norm_backward launch");
  GS_GUARD_END
}

gs_status gs_recurrence_states_size(int64_t B, int64_t T, int64_t D, size_t* bytes) {
  GS_GUARD_BEGIN
  if (!bytes) return bad("bytes is NULL");
  GS_TRY(check_sequence_shape(B, T, D));
  *bytes = states_bytes(B, T, D);
  return GS_OK;
  GS_GUARD_END
}

gs_status gs_recurrence_workspace_size(int64_t B, int64_t T, int64_t D, size_t* bytes) {
  GS_GUARD_BEGIN
  if (!bytes) return bad("bytes is NULL");
  GS_TRY(check_sequence_shape(B, T, D));
  *bytes = recurrence_ws_bytes(B, T, D);
  return GS_OK;
  GS_GUARD_END
}

gs_status gs_recurrence_forward(const gs_seq* x, const gs_seq* r, const gs_seq* i, const float* decay, const float* h0,
                                const uint8_t* reset, const int32_t* lengths, const gs_seq* y, float* h_last,
                                void* states, int64_t B, int64_t T, int64_t D, int32_t dtype, float c,
                                gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  GS_TRY(check_sequence_shape(B, T, D));
  GS_TRY(check_c(c));
  const bool rows = B > 0 && D > 0, some = rows && T > 0;
  GS_TRY(check_seq(x, dtype, some, "x"));
  GS_TRY(check_seq(r, dtype, some, "r"));
  GS_TRY(check_seq(i, dtype, some, "i"));
  GS_TRY(check_seq_output(y, B, T, D, dtype, some, "y"));
  GS_TRY(check_data(decay, 4, rows, "decay"));
  GS_TRY(check_data(h0, 4, false, "h0"));
  GS_TRY(check_data(lengths, 4, false, "lengths"));
  GS_TRY(check_data(h_last, 4, false, "h_last"));
  GS_TRY(check_data(states, 256, false, "states"));
  if (!rows) return GS_OK;
  gs::RecurrenceParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = in(x);
  p.r = in(r);
  p.i = in(i);
  p.y = out(y);
  p.decay = decay;
  p.h0 = h0;
  p.reset = reset;
  p.lengths = lengths;
  p.h_last = h_last;
  p.states = static_cast<float*>(states);
  p.B = B;
  p.T = T;
  p.D = D;
  p.c = c;
  set_tries(p);
  const int unit = copy_unit({x, r, i}, {y}, B, T, D, dtype);
  const cudaError_t e = gs::launch_recurrence_forward(p, dtype, unit, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, "recurrence_forward launch");
  GS_GUARD_END
}

gs_status gs_recurrence_backward(const gs_seq* dy, const float* dh_last, const gs_seq* x, const gs_seq* r,
                                 const gs_seq* i, const float* decay, const uint8_t* reset, const int32_t* lengths,
                                 const void* states, const gs_seq* dx, const gs_seq* dr, const gs_seq* di,
                                 float* ddecay, float* dh0, int64_t B, int64_t T, int64_t D, int32_t dtype, float c,
                                 void* workspace, size_t workspace_bytes, gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  GS_TRY(check_sequence_shape(B, T, D));
  GS_TRY(check_c(c));
  const bool some = B > 0 && D > 0 && T > 0;
  GS_TRY(check_seq(dy, dtype, some, "dy"));
  GS_TRY(check_seq(x, dtype, some, "x"));
  GS_TRY(check_seq(r, dtype, some, "r"));
  GS_TRY(check_seq(i, dtype, some, "i"));
  GS_TRY(check_seq_output(dx, B, T, D, dtype, some, "dx"));
  GS_TRY(check_seq_output(dr, B, T, D, dtype, some, "dr"));
  GS_TRY(check_seq_output(di, B, T, D, dtype, some, "di"));
  GS_TRY(check_data(decay, 4, D > 0, "decay"));
  GS_TRY(check_data(lengths, 4, false, "lengths"));
  GS_TRY(check_data(states, 256, some, "states"));
  GS_TRY(check_data(dh_last, 4, false, "dh_last"));
  GS_TRY(check_data(ddecay, 4, D > 0, "ddecay"));
  GS_TRY(check_data(dh0, 4, false, "dh0"));
  GS_TRY(check_workspace(workspace, workspace_bytes, recurrence_ws_bytes(B, T, D), "gs_recurrence_workspace_size"));
  if (D == 0) return GS_OK;
  gs::RecurrenceParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = in(x);
  p.r = in(r);
  p.i = in(i);
  p.dy = in(dy);
  p.dx = out(dx);
  p.dr = out(dr);
  p.di = out(di);
  p.decay = decay;
  p.reset = reset;
  p.lengths = lengths;
  p.states = static_cast<float*>(const_cast<void*>(states));
  p.dh_last = dh_last;
  p.dh0 = dh0;
  p.partial = static_cast<float*>(workspace);
  p.B = B;
  p.T = T;
  p.D = D;
  p.c = c;
  set_tries(p);
  const int unit = copy_unit({x, r, i, dy}, {dx, dr, di}, B, T, D, dtype);
  const cudaError_t e = gs::launch_recurrence_backward(p, ddecay, dtype, unit, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, "recurrence_backward launch");
  GS_GUARD_END
}

gs_status gs_recurrence_wait_tries(int32_t tiles, int32_t messages) {
  if (tiles < 0 || tiles > gs::kMostTries || messages < 0 || messages > gs::kMostTries)
    return gs::record_failure(GS_ERR_INVALID_ARG, "tries must lie in [0, 2^20]");
  tile_tries = tiles;
  message_tries = messages;
  return GS_OK;
}

gs_status gs_recurrence_step(const void* x, int64_t x_stride, const void* r, int64_t r_stride, const void* i,
                             int64_t i_stride, const float* decay, float* state, int64_t state_stride, int64_t n_slots,
                             const int32_t* slots, void* y, int64_t y_stride, int64_t B, int64_t D, int32_t dtype,
                             float c, gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  GS_TRY(check_shape(B, D));
  if (D > kMaxRows) return bad("D must be below 2^31");
  GS_TRY(check_c(c));
  if (n_slots < 0) return bad("n_slots must not be negative");
  const bool some = B > 0 && D > 0;
  GS_TRY(check_matrix(x, x_stride, dtype, some, "x"));
  GS_TRY(check_matrix(r, r_stride, dtype, some, "r"));
  GS_TRY(check_matrix(i, i_stride, dtype, some, "i"));
  GS_TRY(check_output(y, y_stride, B, D, dtype, some, "y"));
  GS_TRY(check_data(decay, 4, some, "decay"));
  GS_TRY(check_output(state, state_stride, n_slots, D, GS_F32, some && n_slots > 0, "state"));
  GS_TRY(check_data(slots, 4, false, "slots"));
  if (!slots && n_slots < B) return bad("without slots, n_slots must be at least B");
  if (!some) return GS_OK;
  gs::RecurrenceStepParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = x;
  p.r = r;
  p.i = i;
  p.y = y;
  p.x_stride = x_stride;
  p.r_stride = r_stride;
  p.i_stride = i_stride;
  p.y_stride = y_stride;
  p.state_stride = state_stride;
  p.decay = decay;
  p.state = state;
  p.slots = slots;
  p.B = B;
  p.D = D;
  p.n_slots = n_slots;
  p.c = c;
  const uintptr_t two = 2 * item(dtype);
  const bool pair = D % 2 == 0 && (x_stride | r_stride | i_stride | y_stride | state_stride) % 2 == 0 && aligned(x, two) &&
                    aligned(r, two) && aligned(i, two) && aligned(y, two) && aligned(state, 8);
  const cudaError_t e = gs::launch_recurrence_step(p, dtype, pair, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, "recurrence_step launch");
  GS_GUARD_END
}

}  // extern "C"
