// Rotary positions of rows of heads: pair i of head h of token t turns by
// pos[t] * f_i, in the half or the interleaved layout, over the first r
// elements of the head; the others are copied.
//
// Angles are kept in turns, as 64-bit fixed point fractions: pos * turns[i] modulo
// 2^64 is the angle without its whole turns, exactly, at any position, so far
// positions lose nothing and nothing needs 64-bit floating point.  The two top bits
// (rounded) are the quarter, and what is left, within an eighth of a turn,
// goes through the Taylor polynomials of sine and cosine in float32: both are within 2^-23
// of the exact angle's (2^-23.2 at worst, most of it the 24 bits of what is left).
//
// The floor is one read and one write of the rows: 3000 tokens of 72 heads of 128 (111 MB)
// 22 us, 16,000 (590 MB) 115 us, 5.0 and 5.1 TB/s with the launch; one token 2.8 us.
#include "common.h"
#include "kernels.h"

namespace pallas {

namespace {

constexpr int kThreads = 256;   // at most
constexpr int kPasses = 3;      // units of a thread whose loads are in flight together

// Outputs from this many bytes on are stored non-temporally (111 MB read and written: 21.1
// us, 26.8 with plain stores; 164 MB: 34.1, 38.4); smaller ones stay in the caches for what
// reads them next.
constexpr int64_t kNtStoreBytes = int64_t(4) << 20;

template <bool kNt, class V>
__device__ __forceinline__ void put(V v, void* at) {
  if constexpr (kNt) __builtin_nontemporal_store(v, static_cast<V*>(at));
  else *static_cast<V*>(at) = v;
}

// (cos, sin) of an angle of `a` 2^-64 turns, times m.  |rest| <= pi / 4: the first
// terms left out are below 2^-29 (sine, x^11 / 11!) and 2^-32 (cosine, x^12 / 12!)
// of a radian.
__device__ __forceinline__ void turn_cos_sin(uint64_t a, float m, float& c, float& s) {
  const uint64_t quarter = (a + (uint64_t(1) << 61)) >> 62;
  const int32_t rest = static_cast<int32_t>(static_cast<int64_t>(a - (quarter << 62)) >> 32);
  const float x = static_cast<float>(rest) * 1.46291807926715968e-9f;   // 2 pi 2^-32
  const float z = x * x;
  float sp = __builtin_fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
  sp = __builtin_fmaf(z, sp, 8.33333333e-3f);
  sp = __builtin_fmaf(z, sp, -1.66666667e-1f);
  sp = __builtin_fmaf(z * x, sp, x);
  float cp = __builtin_fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
  cp = __builtin_fmaf(z, cp, -1.38888889e-3f);
  cp = __builtin_fmaf(z, cp, 4.16666667e-2f);
  cp = __builtin_fmaf(z, cp, -0.5f);
  cp = __builtin_fmaf(z, cp, 1.0f);
  const bool odd = quarter & 1;
  const float cm = (quarter + 1) & 2 ? -m : m, sm = quarter & 2 ? -m : m;
  c = (odd ? sp : cp) * cm;
  s = (odd ? cp : sp) * sm;
}

__device__ __forceinline__ uint64_t turned(const RopeParams& p, int pos, int i) {
  const uint64_t a = static_cast<uint64_t>(static_cast<int64_t>(pos)) * p.turns[i];
  return p.negate ? 0 - a : a;
}

// A unit is 16 bytes of a head: four pairs (half layout: two 8-byte halves), or
// 8 elements behind the rotated ones.  `units` of a head are worked on (the
// copied ones only where y is not x).  A thread keeps its unit, and so its four
// angles, for all the heads that it takes: `slots` heads of a token go side by
// side (several tokens where a token has fewer), kPasses times.  The first loads are
// issued before the angles are worked out.
template <bool kNt>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeParams p, int units, int slots, int tokens_per, int heads_per) {
  const int j = threadIdx.x % units, slot = threadIdx.x / units;
  const int t = blockIdx.x * tokens_per + (tokens_per > 1 ? slot / p.heads : 0);
  int h = tokens_per > 1 ? slot % p.heads : slot + blockIdx.y * heads_per;
  const int h1 = tokens_per > 1 ? p.heads : min(p.heads, static_cast<int>(blockIdx.y + 1) * heads_per);
  if (slot >= (tokens_per > 1 ? tokens_per * p.heads : slots) || t >= p.tokens) return;
  const bool turn = 8 * j < p.r;
  const bool half = !p.interleaved && turn;
  const int lo = half ? 4 * j : 8 * j, hi = half ? p.r / 2 + 4 * j : 8 * j + 4;
  const uint16_t* x = p.x + t * p.x_token;
  uint16_t* y = p.y + t * p.y_token;
  u32x2 a[kPasses], b[kPasses];
  auto read = [&] {
#pragma unroll
    for (int k = 0; k < kPasses; ++k) {
      if (h + k * slots >= h1) continue;
      const uint16_t* src = x + (h + k * slots) * p.x_head;
      a[k] = *reinterpret_cast<const u32x2*>(src + lo);
      b[k] = *reinterpret_cast<const u32x2*>(src + hi);
    }
  };
  read();
  float c[4], s[4];
  if (turn) {
    const int pos = p.pos[t];
#pragma unroll
    for (int e = 0; e < 4; ++e) turn_cos_sin(turned(p, pos, 4 * j + e), p.magnitude, c[e], s[e]);
  }
  for (;;) {
#pragma unroll
    for (int k = 0; k < kPasses; ++k) {
      if (h + k * slots >= h1) continue;
      if (turn) {
        // half: a = x0 of pairs 0 .. 3, b = x1; interleaved: a, b = pairs 0, 1 and 2, 3
        const float v[8] = {bflo(a[k].x), bfhi(a[k].x), bflo(a[k].y), bfhi(a[k].y),
                            bflo(b[k].x), bfhi(b[k].x), bflo(b[k].y), bfhi(b[k].y)};
        float w[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x0 = half ? v[e] : v[2 * e], x1 = half ? v[e + 4] : v[2 * e + 1];
          const float y0 = x0 * c[e] - x1 * s[e], y1 = x1 * c[e] + x0 * s[e];
          if (half) {
            w[e] = y0;
            w[e + 4] = y1;
          } else {
            w[2 * e] = y0;
            w[2 * e + 1] = y1;
          }
        }
        a[k] = u32x2{pack_bf2(w[0], w[1]), pack_bf2(w[2], w[3])};
        b[k] = u32x2{pack_bf2(w[4], w[5]), pack_bf2(w[6], w[7])};
      }
      uint16_t* dst = y + (h + k * slots) * p.y_head;
      put<kNt>(a[k], dst + lo);
      put<kNt>(b[k], dst + hi);
    }
    h += kPasses * slots;
    if (h >= h1) return;
    read();
  }
}

// The same with units of a pair (or of two copied elements, the last alone in an odd
// head), for any alignment; heads of more units than threads take them in turns.
__global__ __launch_bounds__(kThreads) void rope_any_kernel(RopeParams p, int units, int slots, int heads_per) {
  const int t = blockIdx.x, slot = threadIdx.x / units;
  const int h0 = blockIdx.y * heads_per, h1 = min(p.heads, h0 + heads_per);
  if (slot >= slots) return;
  const int pos = p.pos[t];
  for (int i = threadIdx.x % units; i < units; i += kThreads) {
    const bool turn = 2 * i < p.r;
    const int lo = !turn || p.interleaved ? 2 * i : i, hi = !turn || p.interleaved ? 2 * i + 1 : i + p.r / 2;
    float c = 1.f, s = 0.f;
    if (turn) turn_cos_sin(turned(p, pos, i), p.magnitude, c, s);
    for (int h = h0 + slot; h < h1; h += slots) {
      const uint16_t* x = p.x + t * p.x_token + h * p.x_head;
      uint16_t* y = p.y + t * p.y_token + h * p.y_head;
      const uint16_t a = x[lo], b = hi < p.d ? x[hi] : 0;
      y[lo] = turn ? f2bf(bf2f(a) * c - bf2f(b) * s) : a;
      if (hi < p.d) y[hi] = turn ? f2bf(bf2f(b) * c + bf2f(a) * s) : b;
    }
  }
}

}  // namespace

hipError_t launch_rope(const RopeParams& p, hipStream_t s) {
  if (p.tokens == 0) return hipSuccess;
  auto by = [](const void* q, int64_t a, int64_t b) {
    return (reinterpret_cast<uintptr_t>(q) & 15) == 0 && a % 8 == 0 && b % 8 == 0;
  };
  const bool copy = p.x != p.y;
  if (p.r % 8 != 0 || p.d % 8 != 0 || p.d > 8 * kThreads || !by(p.x, p.x_token, p.x_head) ||
      !by(p.y, p.y_token, p.y_head)) {
    const int units = p.r / 2 + (copy ? (p.d - p.r + 1) / 2 : 0);
    const int slots = std::max(kThreads / units, 1);
    const int heads_per = p.tokens < 512 ? slots : p.heads;
    rope_any_kernel<<<dim3(p.tokens, (p.heads + heads_per - 1) / heads_per), kThreads, 0, s>>>(p, units, slots, heads_per);
    return hipGetLastError();
  }
  // Workgroups as wide as a token's heads fill evenly.
  const int units = copy ? p.d / 8 : p.r / 8;
  const int most = kThreads / units, passes = (p.heads + most - 1) / most;
  const int tokens_per = std::max(most / p.heads, 1);
  const int slots = tokens_per > 1 ? tokens_per * p.heads : (p.heads + passes - 1) / passes;
  // Few tokens: a token's heads over several workgroups.
  const int heads_per = p.tokens < 512 ? slots : p.heads;
  const dim3 grid((p.tokens + tokens_per - 1) / tokens_per, tokens_per > 1 ? 1 : (p.heads + heads_per - 1) / heads_per);
  const int threads = (units * slots + 63) / 64 * 64;
  if (int64_t(p.tokens) * p.heads * units * 16 >= kNtStoreBytes)
    rope_kernel<true><<<grid, threads, 0, s>>>(p, units, slots, tokens_per, heads_per);
  else
    rope_kernel<false><<<grid, threads, 0, s>>>(p, units, slots, tokens_per, heads_per);
  return hipGetLastError();
}

}  // namespace pallas
