// Rotary positions.  A position's turn is exact: with u = frequency / 2 pi as a fraction of 2^64, the low 64 bits
// of position * u are the fraction of a turn, of which the upper 32 go into the sine and cosine.  What they have
// beyond the nearest quarter of a turn, an eighth at most, is rounded to fp32, which moves the angle by 2^-28 turns at
// most (2.3e-8; the whole turn rounded to fp32 moved it by four times that, more than a sine's own rounding).  u itself is
// right to the 53 bits of the frequency: position 2^31 is off by 4e-8 turns at most.
//
// Bound by memory: every element that moves is read and written once.  A CTA works out the sines and cosines of its
// tokens once; a thread then has one place of a head (pairs of one 16-byte word, or of two, or one pair, or words that
// are copied) of one token, whose sines and cosines stay in its registers, in every so many heads.  8x4096x40x128 bf16 in
// place takes 126 us (78 % of the copy rate), half of each head turned out of place 121 us (81 %; 148 us with sines and
// cosines read again for every head).  Registers for four CTAs an SM, or six where elements move one by one: 8x4096x8x128
// in rows that start anywhere takes 57 us, 70 with four.
#include "attention.cuh"

namespace gs {
namespace {

constexpr int kRotaryThreads = 256, kRotaryPairs = 1024;  // sines and cosines that a CTA holds

// VEC: all rows start at 16-byte boundaries, R is a multiple of 16 (interleaved: 8) and what is copied of 8.
template <typename E, bool INTERLEAVED, bool VEC>
__global__ void __launch_bounds__(kRotaryThreads, VEC ? 4 : 6)
k_rotary(const __grid_constant__ RotaryParams p, int tokens, int parts) {
  grid_begin();
  __shared__ __align__(16) float2 cs[kRotaryPairs];
  const int half = p.R / 2, part = blockIdx.x % parts;
  const uint32_t all = (uint32_t)(p.B * p.T), n0 = blockIdx.x / parts * (uint32_t)tokens;
  const int here = (int)min(all - n0, (uint32_t)tokens);
  for (int at = threadIdx.x; at < here * half; at += kRotaryThreads) {
    const uint32_t n = n0 + at / half;
    const int j = at % half;
    const int32_t position = p.positions ? p.positions[n] : (int32_t)(p.first + n % (uint32_t)p.T);
    const double turns = p.frequencies[j] * 0.15915494309189533577;
    // the fraction in [0, 1] as 2^64ths; 2^64 itself is no turn at all
    const double share = (turns - floor(turns)) * 18446744073709551616.0;
    const uint64_t u = share < 18446744073709551616.0 ? (uint64_t)share : 0;
    const uint32_t turn = (uint32_t)(((uint64_t)(int64_t)position * u) >> 32);
    // an eighth of a turn either way of the nearest quarter
    const uint32_t quarters = (turn + 0x20000000u) >> 30;
    float s, c;
    sincospif((float)(int32_t)(turn - (quarters << 30)) * 0x1p-31f, &s, &c);
    if (quarters & 1) {
      const float t = c;
      c = -s;
      s = t;
    }
    if (quarters & 2) {
      c = -c;
      s = -s;
    }
    cs[at] = make_float2(c * p.magnitude, s * p.magnitude * p.sign);
  }
  __syncthreads();
  const int first = (int)((int64_t)p.H * part / parts), last = (int)((int64_t)p.H * (part + 1) / parts);
  const int turned = !VEC ? half : INTERLEAVED ? p.R / 8 : p.R / 16, units = turned + (!p.copy ? 0 : VEC ? (p.D - p.R) / 8 : p.D - p.R);
  // threads side by side: places of a head, tokens, heads
  const int wide = units < kRotaryThreads ? units : kRotaryThreads, lane = threadIdx.x / wide;
  const int lanes = kRotaryThreads / wide, side = min(tokens, lanes), heads = lanes / side, h0 = first + lane / side;
  if (lane / side >= heads) return;
  for (int t = lane % side; t < here; t += side) {
    const uint32_t n = n0 + t, batch = n / (uint32_t)p.T, token = n - batch * (uint32_t)p.T;
    const E* const x = static_cast<const E*>(p.x.data) + batch * p.x.batch + token * p.x.token;
    E* const out = static_cast<E*>(p.out.data) + batch * p.out.batch + token * p.out.token;
    for (int u = threadIdx.x % wide; u < units; u += wide) {
      if constexpr (VEC) {
        const Span g = {0, 0, 8};
        constexpr int AHEAD = 4;
        if (u >= turned) {
          const int c = p.R + (u - turned) * 8;
          for (int h = h0; h < last; h += AHEAD * heads) {
            Raw8<E> raw[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a)
              if (h + a * heads < last) raw[a] = fetch8<E, kEven>(x + (h + a * heads) * p.x.head + c, g);
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
              if (h + a * heads >= last) continue;
#pragma unroll
              for (int k = 0; k < (int)(sizeof(E) / 2); ++k) reinterpret_cast<uint4*>(out + (h + a * heads) * p.out.head + c)[k] = raw[a].q[k];
            }
          }
          continue;
        }
        constexpr int WORDS = INTERLEAVED ? 1 : 2, PAIRS = 4 * WORDS, N = AHEAD / WORDS;
        const int ca = u * 8;
        float2 f[PAIRS];
#pragma unroll
        for (int j = 0; j < PAIRS; ++j) f[j] = cs[t * half + u * PAIRS + j];
        for (int h = h0; h < last; h += N * heads) {
          Raw8<E> raw[N][WORDS];
#pragma unroll
          for (int a = 0; a < N; ++a)
#pragma unroll
            for (int k = 0; k < WORDS; ++k)
              if (h + a * heads < last) raw[a][k] = fetch8<E, kEven>(x + (h + a * heads) * p.x.head + ca + k * half, g);
#pragma unroll
          for (int a = 0; a < N; ++a) {
            if (h + a * heads >= last) continue;
            float v[WORDS][8];
#pragma unroll
            for (int k = 0; k < WORDS; ++k) unpack8<E, kEven>(raw[a][k], g, v[k]);
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) {
              float &first_one = INTERLEAVED ? v[0][j * 2 % 8] : v[0][j], &other = INTERLEAVED ? v[0][(j * 2 + 1) % 8] : v[WORDS - 1][j];
              const float one = first_one, two = other;
              first_one = one * f[j].x - two * f[j].y;
              other = one * f[j].y + two * f[j].x;
            }
#pragma unroll
            for (int k = 0; k < WORDS; ++k) store8<E, kEven>(out + (h + a * heads) * p.out.head + ca + k * half, g, v[k]);
          }
        }
      } else {
        const bool turns = u < half;
        const int ca = !turns ? p.R + u - half : INTERLEAVED ? 2 * u : u, cb = INTERLEAVED ? ca + 1 : u + half;
        const float2 f = turns ? cs[t * half + u] : make_float2(0.f, 0.f);
#pragma unroll 4
        for (int h = h0; h < last; h += heads) {
          const E* from = x + h * p.x.head;
          E* to = out + h * p.out.head;
          if (!turns) {
            to[ca] = from[ca];
            continue;
          }
          const float a = to_f32(from[ca]), b = to_f32(from[cb]);
          to[ca] = from_f32<E>(a * f.x - b * f.y);
          to[cb] = from_f32<E>(a * f.y + b * f.x);
        }
      }
    }
  }
}

}  // namespace

cudaError_t launch_rotary(const RotaryParams& p, int dtype, bool interleaved, bool vec, cudaStream_t s) {
  const int64_t all = p.B * p.T;
  const int half = p.R / 2;
  const int units = (!vec ? half : interleaved ? p.R / 8 : p.R / 16) + (!p.copy ? 0 : vec ? (p.D - p.R) / 8 : p.D - p.R);
  // Tokens of a CTA: enough for eight places a thread, as far as the table goes, and fewer while there are fewer than four
  // CTAs an SM; the heads of few tokens are shared out.  (104678 tokens of 2 heads of 64, 16 of them turned, in rows that start
  // anywhere: 109 us with the four tokens that 256 threads hold at once.)
  const int64_t places = (int64_t)units * p.H;
  int64_t most = half > 0 ? kRotaryPairs / half : 64;
  most = most > 64 ? 64 : most;
  int tokens = (int)(8 * kRotaryThreads / places);
  tokens = tokens < 8 ? 8 : tokens;
  tokens = tokens > most ? (int)most : tokens;
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
