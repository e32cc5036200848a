// Device helpers that quantise rows of a cache (quant_kv.hip, append.hip): a row's
// elements lie over neighbouring lanes, a few to each.
#pragma once

#include <type_traits>

#include "common.h"

namespace pallas {

constexpr uint32_t kInfBits = 0x7F80;        // of a bf16 magnitude
constexpr uint32_t kNanScale = 0x7FC00000;
constexpr uint32_t kNanUnit = 0xFF;          // of an E2M1 group

// Larger magnitude of each half of two packed pairs of bf16 (signs cleared).
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_word(uint32_t v) { return __builtin_amdgcn_mov_dpp(v, CTRL, 0xF, 0xF, false); }
constexpr int kDppHalfMirror = 0x141;   // lane i of 8 reads lane 7 - i: the other quad
constexpr int kDppMirror = 0x140;       // lane i of 16 reads lane 15 - i: the other eight

// Largest bf16 magnitude (as its bits, which order as the values do) of the elements that
// kLanes neighbouring lanes hold, given the largest of each half of a lane's pairs.  All
// lanes of the group are active.
template <int kLanes>
__device__ __forceinline__ uint32_t lanes_top(uint32_t top) {
  if constexpr (kLanes >= 2) top = max_u16x2(top, dpp_word<kDppXor1>(top));
  if constexpr (kLanes >= 4) top = max_u16x2(top, dpp_word<kDppXor2>(top));
  if constexpr (kLanes >= 8) top = max_u16x2(top, dpp_word<kDppHalfMirror>(top));
  if constexpr (kLanes >= 16) top = max_u16x2(top, dpp_word<kDppMirror>(top));
  return max(top & 0xFFFFu, top >> 16);
}

// A lane's part of a quantised row: N / 4 words of 8-bit codes or N / 8 of 4-bit ones, and
// the scale of the row (8 bits: a float32's bits) or of the lane's group (E2M1: its byte).
template <int N>
struct RowCodes {
  uint32_t codes[N / 4];
  uint32_t scale;
};

// N bf16 values of a row of D (packed pairs, in the row's order), D / N lanes to the row.
template <int kFormat, int D, int N>
__device__ __forceinline__ RowCodes<N> quantise_row(const uint32_t (&w)[N / 2]) {
  RowCodes<N> out{};
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < N / 2; ++e) top = max_u16x2(top, w[e] & 0x7FFF7FFFu);
  if constexpr (kFormat == PALLAS_QUANT_E2M1) {
    static_assert((D / 4) % N == 0, "a lane's values are of one group");
    const uint32_t a = lanes_top<D / 4 / N>(top);
    if (a >= kInfBits) {
      out.scale = kNanUnit;
    } else if (a >= (27u << 7)) {      // 2^-100
      // a = 1.f 2^(E - 127): at most 6 = 1.5 2^2 times the scale
      const uint32_t unit = min((a >> 7) - 2 + ((a & 0x7F) > 0x40 ? 1 : 0), 252u);
      out.scale = unit;
      const float scale = __uint_as_float(unit << 23);
#pragma unroll
      for (int e = 0; e < N / 8; ++e) {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[4 * e]), scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[4 * e + 1]), scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[4 * e + 2]), scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[4 * e + 3]), scale, 3);
        out.codes[e] = c;
      }
    }
    return out;
  }
  const uint32_t a = lanes_top<D / N>(top);
  float up = 0.f, scale = 0.f;
  if (a >= kInfBits) {
    scale = __uint_as_float(kNanScale);
  } else if constexpr (kFormat == PALLAS_QUANT_INT8) {
    const float amax = __uint_as_float(a << 16);
    if (amax >= 0x1p-100f) {
      up = 127.0f / amax;
      scale = amax / 127.0f;
    }
  } else if (a != 0) {
    // a = 1.f 2^(E - 127): at most 448 = 1.75 2^8 times the scale
    const int biased = max(1, static_cast<int>(a >> 7) - 8 + ((a & 0x7F) > 0x60 ? 1 : 0));
    scale = __uint_as_float(static_cast<uint32_t>(biased) << 23);
    up = __uint_as_float(static_cast<uint32_t>(254 - biased) << 23);
  }
  out.scale = __float_as_uint(scale);
  if (up != 0.f) {
#pragma unroll
    for (int e = 0; e < N / 4; ++e) {
      const float f0 = bflo(w[2 * e]) * up, f1 = bfhi(w[2 * e]) * up;
      const float f2 = bflo(w[2 * e + 1]) * up, f3 = bfhi(w[2 * e + 1]) * up;
      if constexpr (kFormat == PALLAS_QUANT_INT8) {
        auto code = [](float f) {
          return static_cast<uint32_t>(static_cast<int>(fminf(fmaxf(__builtin_rintf(f), -127.f), 127.f))) & 0xFFu;
        };
        out.codes[e] = code(f0) | code(f1) << 8 | code(f2) << 16 | code(f3) << 24;
      } else {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(f0, f1, 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(f2, f3, c, true);
        out.codes[e] = static_cast<uint32_t>(c);
      }
    }
  }
  return out;
}

// Four 8-bit codes of a row as the numbers they are, without its scale.
template <int kFormat>
__device__ __forceinline__ f32x4 code_values(uint32_t c) {
  if constexpr (kFormat == PALLAS_QUANT_INT8) {
    return f32x4{static_cast<float>(static_cast<int8_t>(c)), static_cast<float>(static_cast<int8_t>(c >> 8)),
                 static_cast<float>(static_cast<int8_t>(c >> 16)), static_cast<float>(static_cast<int8_t>(c >> 24))};
  } else {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c), false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c), true);
    return f32x4{lo.x, lo.y, hi.x, hi.y};
  }
}

// Eight E2M1 codes as bf16, times their scale (the exponent of `unit`, a float32; the
// conversion looks at no other bit of it).
__device__ __forceinline__ u32x4 e2m1_bf16(uint32_t c, float unit) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 3))};
}

// f(std::integral_constant) of a run-time format.
template <class F>
auto for_format(int format, F f) {
  if (format == PALLAS_QUANT_E2M1) return f(std::integral_constant<int, PALLAS_QUANT_E2M1>());
  if (format == PALLAS_QUANT_INT8) return f(std::integral_constant<int, PALLAS_QUANT_INT8>());
  return f(std::integral_constant<int, PALLAS_QUANT_E4M3>());
}

}  // namespace pallas
