// C ABI of the linear attention layer's operators: argument checks and parameter blocks.
#include <algorithm>

#include "attention.cuh"
#include "layer_args.cuh"

namespace {

using namespace gs::args;

gs_status check_heads(const gs_heads* t, int32_t dtype, bool required, const char* name) {
  if (!t) return bad(std::string(name) + " is NULL");
  GS_TRY(check_data(t->data, item(dtype), required, name));
  GS_TRY(check_stride(t->batch_stride, name));
  GS_TRY(check_stride(t->token_stride, name));
  return check_stride(t->head_stride, name);
}

// Rows (b, t, h) of D elements are apart when, from the smallest stride to the largest, each steps over
// all that lies within the ones before.
gs_status check_heads_output(const gs_heads* t, int64_t B, int64_t T, int64_t H, int64_t D, int32_t dtype, bool required,
                             const char* name) {
  GS_TRY(check_heads(t, dtype, required, name));
  struct Way {
    int64_t stride, n;
  } way[3] = {{t->batch_stride, B}, {t->token_stride, T}, {t->head_stride, H}};
  std::sort(way, way + 3, [](const Way& a, const Way& b) { return a.stride < b.stride; });
  int64_t span = D;
  for (const Way& w : way) {
    if (w.n <= 1) continue;
    if (w.stride < span) return bad(std::string(name) + ": rows overlap");
    if (w.n - 1 > (int64_t(1) << 60) / w.stride) return bad(std::string(name) + ": strides are too large for its sizes");
    span += w.stride * (w.n - 1);
  }
  return GS_OK;
}

// Where a tensor's elements are: rows of D adjacent ones, at multiples of up to three strides from the first.
struct Place {
  const void* data;
  int64_t item, D;
  struct {
    int64_t n, stride;
  } way[3];
};
Place place(const gs_heads* t, int64_t B, int64_t T, int64_t H, int64_t D, int32_t dtype) {
  return {t->data, item(dtype), D, {{B, t->batch_stride}, {T, t->token_stride}, {H, t->head_stride}}};
}
Place place(const Matrix& m, int64_t rows, int64_t cols, int32_t dtype) { return {m.data, item(dtype), cols, {{rows, m.stride}, {1, 0}, {1, 0}}}; }

// Whether two tensors of one type share an element.  With d the distance of their first ones, one of a and one of b are the
// same where d + sum of i_k stride_k - sum of j_k stride_k lies in (-D of a, D of b).  Equal strides count once, with i_k - j_k;
// from the largest stride to the smallest only those multiples are followed from which the rest can still get there.
bool overlap(const Place& a, const Place& b) {
  typedef __int128 Wide;  // strides and sizes are bounded each, their products are not
  struct Way {
    Wide stride, least, most;
  } way[6];
  int ways = 0;
  if (!a.data || !b.data) return false;
  const auto span = [](const Place& t) {
    Wide n = t.D;
    for (const auto& w : t.way) n += (Wide)(w.n > 1 ? w.n - 1 : 0) * w.stride;
    return n;
  };
  const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(a.data) - reinterpret_cast<uintptr_t>(b.data)) / a.item;
  if (d >= span(b) || -d >= span(a)) return false;
  for (const auto& w : a.way)
    if (w.n > 1 && w.stride > 0) way[ways++] = {w.stride, 0, w.n - 1};
  for (const auto& w : b.way) {
    if (w.n <= 1 || w.stride <= 0) continue;
    int k = 0;
    while (k < ways && (way[k].stride != w.stride || way[k].least < 0)) ++k;
    if (k < ways)
      way[k].least = 1 - w.n;
    else
      way[ways++] = {w.stride, 1 - w.n, 0};
  }
  std::sort(way, way + ways, [](const Way& x, const Way& y) { return x.stride > y.stride; });
  Wide low[7], high[7];  // of what the ways from k on add
  low[ways] = high[ways] = 0;
  for (int k = ways; k-- > 0;) {
    low[k] = low[k + 1] + way[k].stride * way[k].least;
    high[k] = high[k + 1] + way[k].stride * way[k].most;
  }
  const auto down = [](Wide x, Wide s) { return x / s - (x % s != 0 && x < 0); };
  int tries = 1 << 12;  // strides that are not multiples of one another might need more; what is not found is the caller's to know
  const auto find = [&](const auto& self, int k, Wide at) -> bool {
    if (k == ways) return at > -a.D && at < b.D;
    const Wide s = way[k].stride;
    const Wide first = std::max(way[k].least, -down(at + high[k + 1] + a.D - 1, s)), last = std::min(way[k].most, down(b.D - 1 - low[k + 1] - at, s));
    for (Wide v = first; v <= last && tries-- > 0; ++v)
      if (self(self, k + 1, at + v * s)) return true;
    return false;
  };
  return find(find, 0, d);
}

// Other CTAs read inputs while one writes its output: no output may share an element with an input or another output.
gs_status check_apart(std::initializer_list<Place> outputs, std::initializer_list<Place> inputs, const char* what) {
  for (auto o = outputs.begin(); o != outputs.end(); ++o) {
    for (const Place& i : inputs)
      if (overlap(*o, i)) return bad(std::string(what) + " may not be an input, nor overlap one");
    for (auto other = outputs.begin(); other != o; ++other)
      if (overlap(*o, *other)) return bad(std::string(what) + " may not be the same tensor, nor overlap");
  }
  return GS_OK;
}

// Of two states of `n` floats, `to` may be `from` itself (where that is said) or apart from it.
gs_status check_states(const float* to, const float* from, int64_t n, bool itself, const char* what) {
  if (!to || !from || (itself && to == from)) return GS_OK;
  const uintptr_t a = reinterpret_cast<uintptr_t>(to), b = reinterpret_cast<uintptr_t>(from), bytes = (uintptr_t)n * sizeof(float);
  return a < b + bytes && b < a + bytes ? bad(what) : GS_OK;
}

gs_status check_fraction(float f, const char* name) {
  if (!std::isfinite(f)) return bad(std::string(name) + " must be finite");
  return GS_OK;
}

// ---- linear attention ----------------------------------------------------------------------

// A walk counts tokens in 32 bits, up to a block past the last one.
constexpr int64_t kMaxTokens = (int64_t(1) << 31) - (int64_t(1) << 10);

gs_status check_attention(int64_t B, int64_t T, int64_t H, int64_t K, int64_t Dk, int64_t Dv) {
  if (B < 0 || T < 0 || H < 0 || K < 0) return bad("B, T, H and K must not be negative");
  if (Dk < 1 || Dv < 1 || Dk > GS_ATTENTION_MAX_HEAD || Dv > GS_ATTENTION_MAX_HEAD)
    return bad("Dk and Dv must lie in [1, " + std::to_string(GS_ATTENTION_MAX_HEAD) + "]");
  if (H > 0 && (K < 1 || H % K != 0)) return bad("H must be a multiple of K");
  const int64_t most = Dk > Dv ? Dk : Dv;
  if (T > kMaxTokens || B > kMaxRows || H > kMaxRows || !product_fits(B, T) || !product_fits(B * T, H) || !product_fits(B * T * H, most) ||
      !product_fits(B, H) || !product_fits(B * H, Dk * Dv))
    return bad("T must be at most 2^31 - 2^10, B and H below 2^31, B * T * H * D and B * H * Dk * Dv at most 2^40");
  return GS_OK;
}

struct Sizes {
  int64_t B, T, H, K, Dk, Dv;
  bool packed;
  int32_t dtype;
};

// A walk with C contracted rows and D columns; false where its grid would be too large.
bool shape_fits(const Sizes& z, const gs::AttentionShape& shape, int64_t C, int64_t D) {
  const int64_t most = ((int64_t(1) << 31) - 1) / 3;  // three walks may run at once
  return shape.items < most && shape.items * z.H <= most / ((D + 31) / 32) && z.B * z.H <= most / ((C * D + 255) / 256);
}

size_t carry_bytes(const Sizes& z, int64_t C, int64_t D) {
  const gs::AttentionShape shape = gs::attention_shape(z.B, z.T, z.H, (int)C, (int)D, z.dtype, z.packed);
  return shape.segments > 1 ? round256((size_t)shape.items * z.H * C * D * sizeof(float)) : 0;
}

// For heads that are summed after, of D elements.
size_t part_bytes(const Sizes& z, int64_t D) {
  return z.H > z.K ? round256((size_t)(z.packed ? 1 : z.B) * z.T * z.H * D * sizeof(float)) : 0;
}

gs_status attention_bytes(const Sizes& z, bool backward, size_t* carry, size_t* bytes) {
  for (const auto& w : {std::pair<int64_t, int64_t>{z.Dk, z.Dv}, {z.Dv, z.Dk}})
    if (z.H > 0 && !shape_fits(z, gs::attention_shape(z.B, z.T, z.H, (int)w.first, (int)w.second, z.dtype, z.packed), w.first, w.second))
      return bad("B * T * H is too large for one call");
  *carry = carry_bytes(z, z.Dk, z.Dv);
  if (backward) *carry = std::max(*carry, carry_bytes(z, z.Dv, z.Dk));
  *bytes = backward ? 3 * *carry + part_bytes(z, z.Dk) + part_bytes(z, z.Dv) : *carry;
  if (*bytes == 0) *bytes = 256;
  return GS_OK;
}

gs_status check_sequences(const int32_t* lengths, const int32_t* offsets) {
  GS_TRY(check_data(lengths, 4, false, "lengths"));
  GS_TRY(check_data(offsets, 4, false, "offsets"));
  if (lengths && offsets) return bad("lengths and offsets cannot both be given");
  return GS_OK;
}

gs::HeadsIn in(const gs_heads* t, int64_t share) {
  return {t->data, t->batch_stride, t->token_stride, t->head_stride, (int32_t)share};
}
gs::HeadsOut out(const gs_heads* t) { return {t->data, t->batch_stride, t->token_stride, t->head_stride}; }

thread_local int32_t issue_tries = gs::kMostTries, find_tries = gs::kMostTries, work_tries = gs::kMostTries;

// Walks of the same C and D, at once.
gs_status run_walks(const Sizes& z, gs::AttentionWalks& walks, gs_stream stream, const char* what) {
  for (int k = 0; k < walks.count; ++k) {
    gs::AttentionParams& p = walks.of[k];
    const gs::AttentionShape shape = gs::attention_shape(z.B, z.T, z.H, p.C, p.D, z.dtype, z.packed);
    p.B = z.B;
    p.T = z.T;
    p.H = (int32_t)z.H;
    p.segment = shape.segment;
    p.segments = shape.segments;
    p.items = (int32_t)shape.items;
    p.issue_tries = issue_tries;
    p.find_tries = find_tries;
    p.work_tries = work_tries;
    p.chained = shape.segments > 1 && shape.segments <= gs::kChainedPieces && (!p.first || p.first != p.last);
  }
  const cudaError_t e = gs::launch_attention(walks, z.dtype, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, what);
}

}  // namespace

extern "C" {

gs_status gs_rotary(const gs_heads* x, const gs_heads* o, const double* frequencies, const int32_t* positions,
                    int64_t first, int64_t B, int64_t T, int64_t H, int64_t D, int64_t R, int32_t dtype,
                    int32_t interleaved, int32_t inverse, float magnitude, gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  if (B < 0 || T < 0 || H < 0) return bad("B, T and H must not be negative");
  if (D < 1 || D > GS_ROTARY_MAX_HEAD) return bad("D must lie in [1, " + std::to_string(GS_ROTARY_MAX_HEAD) + "]");
  if (R < 0 || R > D || R % 2 != 0) return bad("R must be even and lie in [0, D]");
  if (B > kMaxRows || T > kMaxRows || H > kMaxRows || !product_fits(B, T) || !product_fits(B * T, H) || !product_fits(B * T * H, D))
    return bad("B, T and H must be below 2^31 and B * T * H * D at most 2^40");
  // one CTA for each token at most, and sixteen of heads; 1024 units of a CTA stay in 32 bits
  if (B * T >= int64_t(1) << 31 || H * D >= int64_t(1) << 26) return bad("B * T must be below 2^31 and H * D below 2^26");
  GS_TRY(check_fraction(magnitude, "magnitude"));
  const bool some = B > 0 && T > 0 && H > 0;
  GS_TRY(check_heads(x, dtype, some, "x"));
  GS_TRY(check_heads_output(o, B, T, H, D, dtype, some, "out"));
  GS_TRY(check_data(frequencies, 8, some && R > 0, "frequencies"));
  GS_TRY(check_data(positions, 4, false, "positions"));
  if (!some) return GS_OK;
  gs::RotaryParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = in(x, 1);
  p.out = out(o);
  p.frequencies = frequencies;
  p.positions = positions;
  p.first = first;
  p.B = B;
  p.T = T;
  p.H = (int32_t)H;
  p.D = (int32_t)D;
  p.R = (int32_t)R;
  p.magnitude = magnitude;
  p.sign = inverse ? -1.f : 1.f;
  p.copy = x->data != o->data && R < D;
  const bool alike = (B <= 1 || x->batch_stride == o->batch_stride) && (T <= 1 || x->token_stride == o->token_stride) &&
                     (H <= 1 || x->head_stride == o->head_stride);
  if (x->data == o->data ? !alike : overlap(place(o, B, T, H, D, dtype), place(x, B, T, H, D, dtype)))
    return bad("out may be x itself only with the same strides, and may not overlap it otherwise");
  if (R == 0 && !p.copy) return GS_OK;
  bool vec = R % (interleaved ? 8 : 16) == 0 && (!p.copy || (D - R) % 8 == 0);
  for (const gs_heads* t : {x, o})
    vec = vec && aligned(t->data, 16) && ((t->batch_stride | t->token_stride | t->head_stride) * item(dtype)) % 16 == 0;
  const cudaError_t e = gs::launch_rotary(p, dtype, interleaved != 0, vec, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, "rotary launch");
  GS_GUARD_END
}

gs_status gs_rotary_frequencies(int64_t R, double base, double factor, double original, double low, double high,
                                double* result) {
  GS_GUARD_BEGIN
  if (R < 0 || R % 2 != 0 || R > GS_ROTARY_MAX_HEAD) return bad("R must be even and lie in [0, " + std::to_string(GS_ROTARY_MAX_HEAD) + "]");
  if (!(base > 0) || std::isinf(base)) return bad("base must be positive and finite");
  if (!(factor >= 1) || std::isinf(factor)) return bad("factor must be finite and at least 1");
  if (!(original >= 0) || std::isinf(original)) return bad("original must be finite and not negative");
  if (!(low >= 0) || !(high > low) || std::isinf(high)) return bad("low and high must be finite with 0 <= low < high");
  if (!result && R > 0) return bad("out is NULL");
  for (int64_t j = 0; j < R / 2; ++j) {
    const double f = std::pow(base, -2.0 * (double)j / (double)R);
    const double stay = original > 0 ? std::min(std::max((original * f / 6.283185307179586 - low) / (high - low), 0.0), 1.0) : 0.0;
    result[j] = f * (stay + (1 - stay) / factor);
  }
  return GS_OK;
  GS_GUARD_END
}

gs_status gs_linear_attention_workspace_size(int64_t B, int64_t T, int64_t H, int64_t K, int64_t Dk, int64_t Dv,
                                             int32_t dtype, int32_t backward, int32_t packed, size_t* bytes) {
  GS_GUARD_BEGIN
  if (!bytes) return bad("bytes is NULL");
  GS_TRY(check_type(dtype));
  GS_TRY(check_attention(B, T, H, K, Dk, Dv));
  size_t carry;
  return attention_bytes({B, T, H, K, Dk, Dv, packed != 0, dtype}, backward != 0, &carry, bytes);
  GS_GUARD_END
}

gs_status gs_linear_attention_forward(const gs_heads* q, const gs_heads* k, const gs_heads* v, const float* log_decay,
                                      const float* s0, const int32_t* lengths, const int32_t* offsets, const gs_heads* o,
                                      float* s_last, int64_t B, int64_t T, int64_t H, int64_t K, int64_t Dk, int64_t Dv,
                                      int32_t dtype, float scale, void* workspace, size_t workspace_bytes,
                                      gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  GS_TRY(check_attention(B, T, H, K, Dk, Dv));
  GS_TRY(check_fraction(scale, "scale"));
  const Sizes z = {B, T, H, K, Dk, Dv, offsets != nullptr, dtype};
  const bool rows = B > 0 && H > 0, some = rows && T > 0;
  GS_TRY(check_heads(q, dtype, some, "q"));
  GS_TRY(check_heads(k, dtype, some, "k"));
  GS_TRY(check_heads(v, dtype, some, "v"));
  GS_TRY(check_heads_output(o, z.packed ? 1 : B, T, H, Dv, dtype, some, "o"));
  if (some) {
    const int64_t batch = z.packed ? 1 : B;
    GS_TRY(check_apart({place(o, batch, T, H, Dv, dtype)},
                       {place(q, batch, T, H, Dk, dtype), place(k, batch, T, K, Dk, dtype), place(v, batch, T, K, Dv, dtype)}, "o"));
  }
  GS_TRY(check_data(log_decay, 4, rows, "log_decay"));
  GS_TRY(check_data(s0, 4, false, "s0"));
  GS_TRY(check_data(s_last, 4, false, "s_last"));
  GS_TRY(check_states(s_last, s0, B * H * Dk * Dv, true, "s_last may be s0 itself, but not overlap it"));
  GS_TRY(check_sequences(lengths, offsets));
  size_t carry, need;
  GS_TRY(attention_bytes(z, false, &carry, &need));
  GS_TRY(check_workspace(workspace, workspace_bytes, need, "gs_linear_attention_workspace_size"));
  if (!rows) return GS_OK;
  gs::AttentionWalks walks;
  std::memset(&walks, 0, sizeof(walks));
  walks.count = 1;
  gs::AttentionParams& p = walks.of[0];
  p.q = in(q, 1);
  p.k = in(k, H / K);
  p.v = in(v, H / K);
  p.o = out(o);
  p.log_decay = log_decay;
  p.first = s0;
  p.last = s_last;
  p.carry = static_cast<float*>(workspace);
  p.state_row = Dv;
  p.state_col = 1;
  p.lengths = lengths;
  p.offsets = offsets;
  p.C = (int32_t)Dk;
  p.D = (int32_t)Dv;
  p.in_scale = 1.f;
  p.out_scale = scale;
  return run_walks(z, walks, stream, "linear_attention_forward launch");
  GS_GUARD_END
}

gs_status gs_linear_attention_backward(const gs_heads* d_o, const gs_heads* q, const gs_heads* k, const gs_heads* v,
                                       const float* log_decay, const float* s0, const float* ds_last,
                                       const int32_t* lengths, const int32_t* offsets, const gs_heads* dq,
                                       const gs_heads* dk, const gs_heads* dv, float* ds0, int64_t B, int64_t T,
                                       int64_t H, int64_t K, int64_t Dk, int64_t Dv, int32_t dtype, float scale,
                                       void* workspace, size_t workspace_bytes, gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  GS_TRY(check_attention(B, T, H, K, Dk, Dv));
  GS_TRY(check_fraction(scale, "scale"));
  const Sizes z = {B, T, H, K, Dk, Dv, offsets != nullptr, dtype};
  const int64_t batch = z.packed ? 1 : B;
  const bool rows = B > 0 && H > 0, some = rows && T > 0;
  GS_TRY(check_heads(d_o, dtype, some, "d_o"));
  GS_TRY(check_heads(q, dtype, some, "q"));
  GS_TRY(check_heads(k, dtype, some, "k"));
  GS_TRY(check_heads(v, dtype, some, "v"));
  GS_TRY(check_heads_output(dq, batch, T, H, Dk, dtype, some, "dq"));
  GS_TRY(check_heads_output(dk, batch, T, K, Dk, dtype, some, "dk"));
  GS_TRY(check_heads_output(dv, batch, T, K, Dv, dtype, some, "dv"));
  if (some)
    GS_TRY(check_apart({place(dq, batch, T, H, Dk, dtype), place(dk, batch, T, K, Dk, dtype), place(dv, batch, T, K, Dv, dtype)},
                       {place(d_o, batch, T, H, Dv, dtype), place(q, batch, T, H, Dk, dtype), place(k, batch, T, K, Dk, dtype),
                        place(v, batch, T, K, Dv, dtype)}, "dq, dk and dv"));
  GS_TRY(check_data(log_decay, 4, rows, "log_decay"));
  GS_TRY(check_data(s0, 4, false, "s0"));
  GS_TRY(check_data(ds_last, 4, false, "ds_last"));
  GS_TRY(check_data(ds0, 4, false, "ds0"));
  for (const float* other : {s0, ds_last}) GS_TRY(check_states(ds0, other, B * H * Dk * Dv, false, "ds0 may not be s0 or ds_last, nor overlap them"));
  GS_TRY(check_sequences(lengths, offsets));
  size_t carry, need;
  GS_TRY(attention_bytes(z, true, &carry, &need));
  GS_TRY(check_workspace(workspace, workspace_bytes, need, "gs_linear_attention_workspace_size"));
  if (!rows) return GS_OK;
  const int64_t share = H / K;
  const char* what = "linear_attention_backward launch";
  char* ws = static_cast<char*>(workspace);
  float* const part_k = reinterpret_cast<float*>(ws + 3 * carry);
  float* const part_v = reinterpret_cast<float*>(ws + 3 * carry + part_bytes(z, Dk));
  gs::AttentionWalks first, second;
  std::memset(&first, 0, sizeof(first));
  for (int k = 0; k < 3; ++k) {
    gs::AttentionParams& p = first.of[k];
    p.log_decay = log_decay;
    p.lengths = lengths;
    p.offsets = offsets;
    p.carry = reinterpret_cast<float*>(ws + k * carry);
    p.in_scale = k > 0 ? scale : 1.f;
    p.out_scale = k > 0 ? 1.f : scale;
    p.back = k > 0;
  }
  const auto shared = [&](const gs_heads* to, float* part, int64_t D) {
    return share == 1 ? out(to) : gs::HeadsOut{part, T * H * D, H * D, D};
  };
  // dq: do reads the transposed state that v and k make up
  gs::AttentionParams& p = first.of[0];
  p.q = in(d_o, 1);
  p.k = in(v, share);
  p.v = in(k, share);
  p.o = out(dq);
  p.first = s0;
  // dk: v reads the transposed gradient of the state, which do and q make up
  gs::AttentionParams& r = first.of[1];
  r.q = in(v, share);
  r.k = in(d_o, 1);
  r.v = in(q, 1);
  r.o = shared(dk, part_k, Dk);
  r.wide = share > 1;
  r.first = ds_last;
  for (int n = 0; n < 2; ++n) {
    first.of[n].state_row = 1;
    first.of[n].state_col = Dv;
    first.of[n].C = (int32_t)Dv;
    first.of[n].D = (int32_t)Dk;
  }
  // dv: k reads the gradient of the state, which q and do make up
  gs::AttentionParams& t = first.of[2];
  t.q = in(k, share);
  t.k = in(q, 1);
  t.v = in(d_o, 1);
  t.o = shared(dv, part_v, Dv);
  t.wide = share > 1;
  t.first = ds_last;
  t.last = ds0;
  t.state_row = Dv;
  t.state_col = 1;
  t.C = (int32_t)Dk;
  t.D = (int32_t)Dv;
  // all at once, where they are of one kind: the heads' sizes, the outputs' type, whether there is a last state
  const bool alike = Dk == Dv && !ds0;
  second = first;
  second.of[0] = first.of[2];
  second.count = 1;
  first.count = alike && share == 1 ? 3 : share == 1 ? 2 : 1;
  GS_TRY(run_walks(z, first, stream, what));
  if (share > 1) {
    first.of[0] = first.of[1];
    first.of[1] = first.of[2];
    first.count = alike ? 2 : 1;
    GS_TRY(run_walks(z, first, stream, what));
  }
  if (!alike) GS_TRY(run_walks(z, second, stream, what));
  if (share == 1 || T == 0) return GS_OK;
  gs::HeadSumParams sum;
  std::memset(&sum, 0, sizeof(sum));
  sum.offsets = offsets;
  sum.B = batch;
  sum.T = T;
  sum.sequences = (int32_t)B;
  sum.K = (int32_t)K;
  sum.share = (int32_t)share;
  for (const bool keys : {true, false}) {
    sum.part = keys ? part_k : part_v;
    sum.out = out(keys ? dk : dv);
    sum.D = (int32_t)(keys ? Dk : Dv);
    const cudaError_t e = gs::launch_head_sums(sum, dtype, as_stream(stream));
    if (e != cudaSuccess) return gs::record_cuda_failure(e, what);
  }
  return GS_OK;
  GS_GUARD_END
}

gs_status gs_linear_attention_wait_tries(int32_t issue, int32_t find, int32_t work) {
  for (const int32_t tries : {issue, find, work})
    if (tries < 0 || tries > gs::kMostTries) return gs::record_failure(GS_ERR_INVALID_ARG, "tries must lie in [0, 2^20]");
  issue_tries = issue;
  find_tries = find;
  work_tries = work;
  return GS_OK;
}

gs_status gs_linear_attention_step(const gs_heads* q, const gs_heads* k, const gs_heads* v, const float* log_decay,
                                   float* state, int64_t state_stride, int64_t n_slots, const int32_t* slots,
                                   const gs_heads* o, int64_t B, int64_t H, int64_t K, int64_t Dk, int64_t Dv,
                                   int32_t dtype, float scale, gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  GS_TRY(check_attention(B, 1, H, K, Dk, Dv));
  GS_TRY(check_fraction(scale, "scale"));
  const bool some = B > 0 && H > 0;
  if (n_slots < 0 || n_slots > kMaxRows) return bad("n_slots must lie in [0, 2^31)");
  GS_TRY(check_heads(q, dtype, some, "q"));
  GS_TRY(check_heads(k, dtype, some, "k"));
  GS_TRY(check_heads(v, dtype, some, "v"));
  GS_TRY(check_heads_output(o, B, 1, H, Dv, dtype, some, "o"));
  if (some)
    GS_TRY(check_apart({place(o, B, 1, H, Dv, dtype)}, {place(q, B, 1, H, Dk, dtype), place(k, B, 1, K, Dk, dtype), place(v, B, 1, K, Dv, dtype)},
                       "o"));
  GS_TRY(check_data(log_decay, 4, some, "log_decay"));
  GS_TRY(check_output(state, state_stride, n_slots, H * Dk * Dv, GS_F32, some && n_slots > 0, "state"));
  GS_TRY(check_data(slots, 4, false, "slots"));
  if (!slots && n_slots < B) return bad("without slots, n_slots must be at least B");
  if (B > 0 && H > ((int64_t(1) << 31) - 1) / ((Dv + 31) / 32) / B) return bad("B * H is too large for one call");
  if (!some) return GS_OK;
  gs::AttentionStepParams p;
  std::memset(&p, 0, sizeof(p));
  p.q = in(q, 1);
  p.k = in(k, H / K);
  p.v = in(v, H / K);
  p.o = out(o);
  p.log_decay = log_decay;
  p.state = state;
  p.state_stride = state_stride;
  p.n_slots = n_slots;
  p.slots = slots;
  p.B = B;
  p.H = (int32_t)H;
  p.Dk = (int32_t)Dk;
  p.Dv = (int32_t)Dv;
  p.scale = scale;
  const bool vec = Dv % 4 == 0 && state_stride % 4 == 0 && aligned(state, 16);
  const cudaError_t e = gs::launch_attention_step(p, dtype, vec, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, "linear_attention_step launch");
  GS_GUARD_END
}

}  // extern "C"

namespace {

// ---- the norms around a block ----------------------------------------------------------------

gs_status check_gated(int64_t rows, int64_t cols, int64_t groups, int32_t act) {
  GS_TRY(check_shape(rows, cols));
  if (groups < 1 || cols < 1 || cols % groups != 0) return bad("groups must divide cols, which must be positive");
  if (cols / groups > GS_NORM_MAX_COLS) return bad("a group must have at most " + std::to_string(GS_NORM_MAX_COLS) + " columns");
  if (cols > int64_t(1) << 20) return bad("cols must be at most 2^20");
  // a CTA takes two groups or more where they are narrow
  if (rows > kMaxRows / groups) return bad("rows * groups must be below 2^31");
  if (act != GS_GATE_NONE && act != GS_GATE_SIGMOID && act != GS_GATE_SILU)
    return bad("act must be GS_GATE_NONE, GS_GATE_SIGMOID or GS_GATE_SILU, got " + std::to_string(act));
  return GS_OK;
}

size_t gated_ws_bytes(int64_t rows, int64_t cols, int64_t groups) {
  const int64_t width = cols / groups;
  return round256((size_t)gs::gated_norm_most_sums(rows * groups, (int)groups, (int)width) * width * sizeof(float) * (groups == 1 ? 2 : 1));
}

// How the groups of these tensors lie; makes evenly spaced groups rows of their own.
struct Lie {
  gs::Layout layout;
  int lead, outer;
  bool spaced;
};
Lie lie_of(std::initializer_list<Matrix> all, int64_t rows, int64_t cols, int64_t groups, int32_t dtype) {
  Lie l = {gs::kApart, 0, 1, spaced(all)};
  if (groups == 1) {
    l.layout = layout_of(all, rows, cols, dtype, &l.lead);
    return l;
  }
  bool even = true;  // all groups of all rows at one distance
  for (const Matrix& m : all) even = even && (!m.data || rows <= 1 || m.stride == cols);
  const int64_t width = cols / groups;
  if (even) {
    bool first = true;
    l.layout = gs::kTogether;
    for (const Matrix& m : all) {
      if (!m.data) continue;
      const int at = (int)(reinterpret_cast<uintptr_t>(m.data) / item(dtype) % 8);
      if (first) l.lead = at;
      first = false;
      if (at != l.lead) l.layout = gs::kApart;
    }
    if (l.layout == gs::kApart)
      l.lead = 0;
    else if (l.lead == 0 && width % 8 == 0)
      l.layout = gs::kEven;
    l.spaced = l.spaced && width >= 8;
    return l;
  }
  l.outer = (int)groups;
  if (layout_of(all, rows, cols, dtype, &l.lead) == gs::kEven && width % 8 == 0) l.layout = gs::kEven;
  l.lead = 0;
  return l;
}

int64_t step_of(const Lie& l, int64_t stride, int64_t cols, int64_t groups) { return groups > 1 && l.outer == 1 ? cols / groups : stride; }

}  // namespace

extern "C" {

gs_status gs_gated_norm(const void* x, int64_t x_stride, const void* gate, int64_t gate_stride, const void* residual,
                        int64_t residual_stride, const float* weight, const float* next_weight, void* y,
                        int64_t y_stride, void* z, int64_t z_stride, float* rstd, float* next_rstd, int64_t rows,
                        int64_t cols, int64_t groups, int32_t dtype, int32_t act, float scale, float eps,
                        gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  GS_TRY(check_gated(rows, cols, groups, act));
  GS_TRY(check_fraction(scale, "scale"));
  if (!(eps >= 0.f) || std::isinf(eps)) return bad("eps must be finite and not negative");
  const bool some = rows > 0, follow = next_weight != nullptr;
  if (follow && groups != 1) return bad("groups must be 1 with next_weight");
  GS_TRY(check_matrix(x, x_stride, dtype, some, "x"));
  GS_TRY(check_matrix(gate, gate_stride, dtype, some && act != GS_GATE_NONE, "gate"));
  if (gate && act == GS_GATE_NONE) return bad("gate is given, but act is GS_GATE_NONE");
  GS_TRY(check_matrix(residual, residual_stride, dtype, false, "residual"));
  GS_TRY(check_data(weight, 4, true, "weight"));
  GS_TRY(check_data(next_weight, 4, false, "next_weight"));
  GS_TRY(check_output(y, y_stride, rows, cols, dtype, some, "y"));
  GS_TRY(check_output(z, z_stride, rows, cols, dtype, some && follow, "z"));
  GS_TRY(check_data(rstd, 4, some, "rstd"));
  GS_TRY(check_data(next_rstd, 4, some && follow, "next_rstd"));
  if (!follow && (z || next_rstd)) return bad("z and next_rstd go with next_weight");
  if (!some) return GS_OK;
  const auto at = [&](const void* t, int64_t stride) { return place(Matrix{t, stride}, rows, cols, dtype); };
  GS_TRY(check_apart({at(z, z_stride)}, {at(x, x_stride), at(gate, gate_stride), at(residual, residual_stride), at(y, y_stride)}, "z"));
  for (const Matrix& m : {Matrix{x, x_stride}, Matrix{gate, gate_stride}, Matrix{residual, residual_stride}})
    if (m.data == y ? rows > 1 && m.stride != y_stride : overlap(at(y, y_stride), at(m.data, m.stride)))
      return bad("y may be an input itself only with the same stride, and may not overlap it otherwise");
  gs::GatedNormParams q;
  std::memset(&q, 0, sizeof(q));
  q.x = x;
  q.gate = gate;
  q.residual = residual;
  q.weight = weight;
  q.next_weight = next_weight;
  q.y = y;
  q.z = z;
  q.rstd = rstd;
  q.next_rstd = next_rstd;
  const std::initializer_list<Matrix> all = {
      {x, x_stride}, {gate, gate_stride}, {residual, residual_stride}, {y, y_stride}, {z, z_stride}};
  Lie l = lie_of(all, rows, cols, groups, dtype);
  q.x_stride = step_of(l, x_stride, cols, groups);
  q.gate_stride = step_of(l, gate_stride, cols, groups);
  q.residual_stride = step_of(l, residual_stride, cols, groups);
  q.y_stride = step_of(l, y_stride, cols, groups);
  q.z_stride = z_stride;
  q.rows = rows * groups;
  q.groups = (int32_t)groups;
  q.width = (int32_t)(cols / groups);
  q.lead = l.lead;
  // in place, what lies beside a row is being written while it is read
  q.spaced = l.spaced && y != x && y != gate && y != residual;
  q.act = act;
  q.scale = scale;
  q.eps = eps;
  if (!aligned(weight, 16) || !aligned(next_weight, 16)) l.layout = gs::kApart;
  const cudaError_t e = gs::launch_gated_norm(q, l.outer, dtype, l.layout, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, "gated_norm launch");
  GS_GUARD_END
}

gs_status gs_gated_norm_workspace_size(int64_t rows, int64_t cols, int64_t groups, size_t* bytes) {
  GS_GUARD_BEGIN
  if (!bytes) return bad("bytes is NULL");
  GS_TRY(check_gated(rows, cols, groups, GS_GATE_NONE));
  *bytes = gated_ws_bytes(rows, cols, groups);
  return GS_OK;
  GS_GUARD_END
}

gs_status gs_gated_norm_backward(const void* dy, int64_t dy_stride, const void* dz, int64_t dz_stride, const void* x,
                                 int64_t x_stride, const void* gate, int64_t gate_stride, const void* y,
                                 int64_t y_stride, const float* weight, const float* next_weight, const float* rstd,
                                 const float* next_rstd, void* dx, int64_t dx_stride, void* dgate,
                                 int64_t dgate_stride, void* dresidual, int64_t dresidual_stride, float* dweight,
                                 float* dnext_weight, int64_t rows, int64_t cols, int64_t groups, int32_t dtype,
                                 int32_t act, float scale, void* workspace, size_t workspace_bytes, gs_stream stream) {
  GS_GUARD_BEGIN
  GS_TRY(check_type(dtype));
  GS_TRY(check_gated(rows, cols, groups, act));
  GS_TRY(check_fraction(scale, "scale"));
  const bool some = rows > 0, follow = next_weight != nullptr;
  if (follow && groups != 1) return bad("groups must be 1 with next_weight");
  GS_TRY(check_matrix(dy, dy_stride, dtype, some && !follow, "dy"));
  GS_TRY(check_matrix(dz, dz_stride, dtype, some && follow, "dz"));
  GS_TRY(check_matrix(x, x_stride, dtype, some, "x"));
  GS_TRY(check_matrix(gate, gate_stride, dtype, some && act != GS_GATE_NONE, "gate"));
  if ((gate || dgate) && act == GS_GATE_NONE) return bad("gate or dgate is given, but act is GS_GATE_NONE");
  GS_TRY(check_matrix(y, y_stride, dtype, some && follow, "y"));
  GS_TRY(check_data(weight, 4, true, "weight"));
  GS_TRY(check_data(next_weight, 4, false, "next_weight"));
  GS_TRY(check_data(rstd, 4, some, "rstd"));
  GS_TRY(check_data(next_rstd, 4, some && follow, "next_rstd"));
  if (!follow && (dz || y || next_rstd || dnext_weight)) return bad("dz, y, next_rstd and dnext_weight go with next_weight");
  GS_TRY(check_output(dx, dx_stride, rows, cols, dtype, false, "dx"));
  GS_TRY(check_output(dgate, dgate_stride, rows, cols, dtype, false, "dgate"));
  GS_TRY(check_output(dresidual, dresidual_stride, rows, cols, dtype, false, "dresidual"));
  if (some) {
    const auto at = [&](const void* t, int64_t stride) { return place(Matrix{t, stride}, rows, cols, dtype); };
    GS_TRY(check_apart({at(dx, dx_stride), at(dgate, dgate_stride), at(dresidual, dresidual_stride)},
                       {at(dy, dy_stride), at(dz, dz_stride), at(x, x_stride), at(gate, gate_stride), at(y, y_stride)},
                       "dx, dgate and dresidual"));
  }
  GS_TRY(check_data(dweight, 4, true, "dweight"));
  GS_TRY(check_data(dnext_weight, 4, follow, "dnext_weight"));
  GS_TRY(check_workspace(workspace, workspace_bytes, gated_ws_bytes(rows, cols, groups), "gs_gated_norm_workspace_size"));
  gs::GatedNormBackParams q;
  std::memset(&q, 0, sizeof(q));
  q.dy = dy;
  q.dz = some ? dz : nullptr;
  q.x = x;
  q.gate = gate;
  q.y = y;
  q.weight = weight;
  q.next_weight = next_weight;
  q.rstd = rstd;
  q.next_rstd = next_rstd;
  q.dx = dx;
  q.dgate = dgate;
  q.dresidual = dresidual;
  q.partial = static_cast<float*>(workspace);
  const std::initializer_list<Matrix> all = {{dy, dy_stride}, {dz, dz_stride}, {x, x_stride},         {gate, gate_stride},
                                             {y, y_stride},   {dx, dx_stride}, {dgate, dgate_stride}, {dresidual, dresidual_stride}};
  Lie l = lie_of(all, rows, cols, groups, dtype);
  q.dy_stride = step_of(l, dy_stride, cols, groups);
  q.dz_stride = dz_stride;
  q.x_stride = step_of(l, x_stride, cols, groups);
  q.gate_stride = step_of(l, gate_stride, cols, groups);
  q.y_stride = y_stride;
  q.dx_stride = step_of(l, dx_stride, cols, groups);
  q.dgate_stride = step_of(l, dgate_stride, cols, groups);
  q.dresidual_stride = step_of(l, dresidual_stride, cols, groups);
  q.rows = rows * groups;
  q.groups = (int32_t)groups;
  q.width = (int32_t)(cols / groups);
  q.lead = l.lead;
  q.spaced = l.spaced;
  q.act = act;
  q.scale = scale;
  if (!aligned(weight, 16) || !aligned(next_weight, 16)) l.layout = gs::kApart;
  const cudaError_t e = gs::launch_gated_norm_backward(q, l.outer, dweight, dnext_weight, dtype, l.layout, as_stream(stream));
  return e == cudaSuccess ? GS_OK : gs::record_cuda_failure(e, "gated_norm_backward launch");
  GS_GUARD_END
}

}  // extern "C"
