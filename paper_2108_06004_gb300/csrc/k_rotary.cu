// Rotary positions.  A position's turn is exact: with u = frequency / 2 pi as a fraction of 2^64, the low 64 bits
// of position * u are the fraction of a turn, of which the upper 32 go into the sine and cosine (a
// quarter of 2^-32 turns is far below an fp32 rounding of either).  u itself is right to the 53 bits of
// the frequency: position 2^31 is off by 4e-8 turns at most.
//
// Bound by memory: every element that moves is read and written once.  A CTA works out the sines and cosines of its
// tokens once, for all heads, and then moves units of eight pairs (16-byte words) or single pairs.
#include "attention.cuh"

namespace gs {
namespace {

constexpr int kRotaryThreads = 256, kRotaryPairs = 1024;  // sines and cosines that a CTA holds

template <typename E>
__device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], const float2* cs) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 t = cs[j];
    const float x = a[j] * t.x - b[j] * t.y;
    b[j] = a[j] * t.y + b[j] * t.x;
    a[j] = x;
  }
}

// VEC: all rows start at 16-byte boundaries, R is a multiple of 16 and what is copied of 8.
template <typename E, bool INTERLEAVED, bool VEC>
__global__ void __launch_bounds__(kRotaryThreads)
k_rotary(const __grid_constant__ RotaryParams p, int tokens, int parts) {
  grid_begin();
  __shared__ __align__(16) float2 cs[kRotaryPairs];
  const int half = p.R / 2, part = blockIdx.x % parts;
  const int64_t n0 = (int64_t)(blockIdx.x / parts) * tokens, all = p.B * p.T;
  const int here = (int)(all - n0 < tokens ? all - n0 : tokens);
  for (int at = threadIdx.x; at < here * half; at += kRotaryThreads) {
    const int64_t n = n0 + at / half;
    const int j = at % half;
    const int32_t position = p.positions ? p.positions[n] : (int32_t)(p.first + n % p.T);
    const double turns = p.frequencies[j] * 0.15915494309189533577;
    // the fraction in [0, 1] as 2^64ths; 2^64 itself is no turn at all
    const double share = (turns - floor(turns)) * 18446744073709551616.0;
    const uint64_t u = share < 18446744073709551616.0 ? (uint64_t)share : 0;
    const int32_t angle = (int32_t)(((uint64_t)(int64_t)position * u) >> 32);
    float s, c;
    sincospif((float)angle * 0x1p-31f, &s, &c);
    cs[at] = make_float2(c * p.magnitude, s * p.magnitude * p.sign);
  }
  __syncthreads();
  const int h0 = (int)((int64_t)p.H * part / parts), heads = (int)((int64_t)p.H * (part + 1) / parts) - h0;
  if constexpr (VEC) {
    const int rot = p.R / 16, units = rot + (p.copy ? (p.D - p.R) / 8 : 0);
    for (int at = threadIdx.x; at < here * heads * units; at += kRotaryThreads) {
      const int u = at % units, row = at / units, t = row / heads;
      const int64_t n = n0 + t, batch = n / p.T, token = n % p.T, head = h0 + row % heads;
      const E* x = static_cast<const E*>(p.x.data) + batch * p.x.batch + token * p.x.token + head * p.x.head;
      E* out = static_cast<E*>(p.out.data) + batch * p.out.batch + token * p.out.token + head * p.out.head;
      const Span g = {0, 0, 8};
      if (u >= rot) {
        const int c = p.R + (u - rot) * 8;
        const Raw8<E> raw = fetch8<E, kEven>(x + c, g);
#pragma unroll
        for (int k = 0; k < (int)(sizeof(E) / 2); ++k) reinterpret_cast<uint4*>(out + c)[k] = raw.q[k];
        continue;
      }
      const int ca = INTERLEAVED ? u * 16 : u * 8, cb = INTERLEAVED ? ca + 8 : ca + half;
      const Raw8<E> ra = fetch8<E, kEven>(x + ca, g), rb = fetch8<E, kEven>(x + cb, g);
      float a[8], b[8];
      unpack8<E, kEven>(ra, g, a);
      unpack8<E, kEven>(rb, g, b);
      const float2* t8 = cs + t * half + u * 8;
      if constexpr (INTERLEAVED) {
        float e[8], o[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          e[j] = a[2 * j], o[j] = a[2 * j + 1];
          e[4 + j] = b[2 * j], o[4 + j] = b[2 * j + 1];
        }
        turn<E>(e, o, t8);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          a[2 * j] = e[j], a[2 * j + 1] = o[j];
          b[2 * j] = e[4 + j], b[2 * j + 1] = o[4 + j];
        }
      } else {
        turn<E>(a, b, t8);
      }
      store8<E, kEven>(out + ca, g, a);
      store8<E, kEven>(out + cb, g, b);
    }
  } else {
    const int units = half + (p.copy ? p.D - p.R : 0);
    for (int at = threadIdx.x; at < here * heads * units; at += kRotaryThreads) {
      const int u = at % units, row = at / units, t = row / heads;
      const int64_t n = n0 + t, batch = n / p.T, token = n % p.T, head = h0 + row % heads;
      const E* x = static_cast<const E*>(p.x.data) + batch * p.x.batch + token * p.x.token + head * p.x.head;
      E* out = static_cast<E*>(p.out.data) + batch * p.out.batch + token * p.out.token + head * p.out.head;
      if (u >= half) {
        out[p.R + u - half] = x[p.R + u - half];
        continue;
      }
      const int ca = INTERLEAVED ? 2 * u : u, cb = INTERLEAVED ? ca + 1 : u + half;
      const float a = to_f32(x[ca]), b = to_f32(x[cb]);
      const float2 t2 = cs[t * half + u];
      out[ca] = from_f32<E>(a * t2.x - b * t2.y);
      out[cb] = from_f32<E>(a * t2.y + b * t2.x);
    }
  }
}

}  // namespace

cudaError_t launch_rotary(const RotaryParams& p, int dtype, bool interleaved, bool vec, cudaStream_t s) {
  const int64_t all = p.B * p.T;
  const int half = p.R / 2;
  // as many tokens as the table holds, up to eight, and fewer while there are fewer than four CTAs an SM;
  // the heads of few tokens are shared out
  int tokens = half > 0 ? kRotaryPairs / half : 8;
  tokens = tokens > 8 ? 8 : tokens;
  while (tokens > 1 && (all + tokens - 1) / tokens < 4 * kSMs) tokens /= 2;
  const int64_t groups = (all + tokens - 1) / tokens;
  int parts = 1;
  while (groups * parts < 4 * kSMs && parts * 8 <= p.H) parts *= 2;
  return with_type(dtype, [&](auto e) {
    using E = decltype(e);
    const auto go = [&](auto kernel) { return launch(kernel, dim3((unsigned)(groups * parts)), dim3(kRotaryThreads), s, p, tokens, parts); };
    return interleaved ? (vec ? go(k_rotary<E, true, true>) : go(k_rotary<E, true, false>))
                       : (vec ? go(k_rotary<E, false, true>) : go(k_rotary<E, false, false>));
  });
}

}  // namespace gs
