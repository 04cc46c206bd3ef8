// Argument checks shared by the entry points of the layers' operators.
#pragma once

#include <cmath>
#include <cstring>
#include <initializer_list>
#include <new>
#include <string>

#include "gs_layer.cuh"

namespace gs {
namespace args {

constexpr int64_t kMaxElements = int64_t(1) << 40;
constexpr int64_t kMaxStride = int64_t(1) << 45;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1;

inline gs_status bad(const std::string& msg) noexcept { return record_failure(GS_ERR_INVALID_ARG, msg.c_str()); }

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

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline cudaStream_t as_stream(gs_stream s) { return reinterpret_cast<cudaStream_t>(s); }
inline int item(int32_t dtype) { return dtype == GS_F32 ? 4 : 2; }

inline gs_status check_type(int32_t dtype) {
  if (dtype != GS_F32 && dtype != GS_F16 && dtype != GS_BF16)
    return bad("dtype must be GS_F32, GS_F16 or GS_BF16, got " + std::to_string(dtype));
  return GS_OK;
}

// required: a NULL is refused
inline gs_status check_data(const void* p, int align, bool required, const char* name) {
  if (!p) return required ? bad(std::string(name) + " is NULL") : GS_OK;
  if (!aligned(p, (uintptr_t)align)) return bad(std::string(name) + " is not " + std::to_string(align) + "-byte aligned");
  return GS_OK;
}

inline gs_status check_stride(int64_t s, const char* name) {
  if (s < 0 || s > kMaxStride) return bad(std::string(name) + ": strides must lie in [0, 2^45]");
  return GS_OK;
}

inline gs_status check_matrix(const void* p, int64_t stride, int32_t dtype, bool required, const char* name) {
  GS_TRY(check_data(p, item(dtype), required, name));
  return p ? check_stride(stride, name) : GS_OK;
}

inline gs_status check_output(const void* p, int64_t stride, int64_t rows, int64_t cols, int32_t dtype, bool required,
                       const char* name) {
  GS_TRY(check_matrix(p, stride, dtype, required, name));
  if (p && rows > 1 && stride < cols) return bad(std::string(name) + ": rows overlap (stride below cols)");
  return GS_OK;
}

// n * unit <= kMaxElements without overflow
inline bool product_fits(int64_t a, int64_t b) { return a == 0 || b <= kMaxElements / a; }

inline gs_status check_shape(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0) return bad("rows and cols must not be negative");
  if (rows > kMaxRows || cols > kMaxElements || !product_fits(rows, cols))
    return bad("rows must be below 2^31 and rows * cols at most 2^40");
  return GS_OK;
}

// How the rows of these tensors lie to one another; `lead`: see Layout.  Absent tensors agree
// with everything.
struct Matrix {
  const void* data;
  int64_t stride;
};
inline Layout layout_of(std::initializer_list<Matrix> all, int64_t rows, int64_t cols, int32_t dtype, int* lead) {
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
      return kApart;
    }
  }
  const bool even = *lead == 0 && cols % 8 == 0 && (rows == 1 || !first || first->stride % 8 == 0);
  return even ? kEven : kTogether;
}

inline bool spaced(std::initializer_list<Matrix> all) {
  for (const Matrix& m : all)
    if (m.data && m.stride < 8) return false;
  return true;
}

inline gs_status check_workspace(const void* ws, size_t bytes, size_t need, const char* size_call) {
  if (!ws || !aligned(ws, 256)) return bad("workspace is NULL or not 256-byte aligned");
  if (bytes < need) return bad(std::string("workspace too small: use ") + size_call);
  return GS_OK;
}

inline size_t round256(size_t n) { return n ? (n + 255) & ~size_t(255) : 256; }

}  // namespace args
}  // namespace gs
