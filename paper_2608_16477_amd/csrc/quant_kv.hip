// An 8-bit KV cache: rows (one token's K or V of one head, d values) quantised as
// they are written into their page slots, and read back as bf16.
//
//   E4M3  scale = 2^e, the least with a <= 448 * 2^e (a: the row's largest
//         magnitude).  A power of two costs a floating-point code no precision and
//         makes both directions exact but for the code's own rounding (and for 2^128,
//         which the last 8 of bf16's magnitudes round to).
//   INT8  scale = a / 127: a power of two would cost up to one of seven bits.
//
// Both are bound by memory: 2 d bytes and d + 4 bytes per row (34,708 tokens of 8 heads of
// 128, E4M3, 217 MB each way: 42 us written, 42 read back, 5.2 TB/s).  Codes are stored
// plainly (with non-temporal stores 87 us for both, and loads 86, in place of 84).  A lane takes 16
// elements (two 16-byte vectors of bf16, one of codes), d / 16 neighbouring lanes a
// row, and neighbouring rows are the heads of a token, contiguous on both sides.
#include "common.h"
#include "kernels.h"

namespace pallas {

namespace {

constexpr int kThreads = 256;
constexpr int kPage = 16;
// Rows read back are stored non-temporally from this many bytes on (34,708 tokens of 8
// heads of 128 written and read back: 84 us, 97 with plain stores; 256 written and 3000 read:
// 8.0, 9.3); fewer stay in the caches for what reads them next.
constexpr int64_t kNtStoreBytes = int64_t(4) << 20;
constexpr uint32_t kInfBits = 0x7F80;
constexpr uint32_t kNanScale = 0x7FC00000;

// Row `row` of the call (token-major, K heads then V heads): a token, its plane and head.
struct Row {
  int t, h, h2;
  bool v;
};
__device__ __forceinline__ Row row_of(const QuantParams& p, uint32_t row) {
  Row r;
  r.t = static_cast<int>(row / static_cast<uint32_t>(2 * p.Hkv));
  r.h2 = static_cast<int>(row) - r.t * (2 * p.Hkv);
  r.v = r.h2 >= p.Hkv;
  r.h = r.v ? r.h2 - p.Hkv : r.h2;
  return r;
}
// Its element offset in the caller's K (or V) rows.
__device__ __forceinline__ int64_t at_of(const QuantParams& p, const Row& r) {
  return r.t * (r.v ? p.v_stride : p.k_stride) + static_cast<int64_t>(r.h) * p.d;
}
// Its place in the pool, among the rows of both planes; negative: skipped.
__device__ __forceinline__ int64_t slot_of(const QuantParams& p, const Row& r, bool flag) {
  const int pos = p.pos[r.t], s = p.seq ? p.seq[r.t] : r.t;
  if (pos < 0) return -1;
  int pg = -1;
  if (s >= 0 && s < p.seqs && pos / kPage < p.max_pages) pg = p.bt[static_cast<int64_t>(s) * p.max_pages + pos / kPage];
  if (pg < 0 || pg >= p.num_pages) {
    if (flag && r.h2 == 0 && p.err) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
    return -1;
  }
  return ((static_cast<int64_t>(r.v ? p.num_pages : 0) + pg) * kPage + pos % kPage) * p.Hkv + r.h;
}

// Larger magnitude of each half of two packed pairs of bf16 (signs cleared).
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ uint32_t dpp_xor1(uint32_t v) { return __builtin_amdgcn_mov_dpp(v, kDppXor1, 0xF, 0xF, false); }
__device__ __forceinline__ uint32_t dpp_xor2(uint32_t v) { return __builtin_amdgcn_mov_dpp(v, kDppXor2, 0xF, 0xF, false); }
constexpr int kDppHalfMirror = 0x141;   // lane i of 8 reads lane 7 - i: the other quad

template <int D, bool kInt8>
__global__ __launch_bounds__(kThreads) void quant_store_kernel(QuantParams p, uint32_t rows) {
  constexpr int kLanes = D / 16;
  const uint32_t row = blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  const int part = threadIdx.x % kLanes;
  // Every lane stays for the row's reduction: rows past the end repeat the last one.
  const bool in = row < rows;
  const Row r = row_of(p, in ? row : rows - 1);
  const u32x4* src = reinterpret_cast<const u32x4*>((r.v ? p.v : p.k) + at_of(p, r) + part * 16);
  const u32x4 x0 = src[0], x1 = src[1];
  const int64_t slot = slot_of(p, r, in && part == 0);
  const uint32_t w[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
  uint32_t top = 0;   // bf16 magnitudes order as their bit patterns
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max_u16x2(top, w[e] & 0x7FFF7FFFu);
  top = max_u16x2(top, dpp_xor1(top));
  top = max_u16x2(top, dpp_xor2(top));
  if constexpr (kLanes == 8) top = max_u16x2(top, __builtin_amdgcn_mov_dpp(top, kDppHalfMirror, 0xF, 0xF, false));
  const uint32_t a = max(top & 0xFFFFu, top >> 16);
  float up = 0.f, scale = 0.f;
  if (a >= kInfBits) {
    scale = __uint_as_float(kNanScale);
  } else if constexpr (kInt8) {
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
  u32x4 codes = {};
  if (up != 0.f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float f0 = bflo(w[2 * e]) * up, f1 = bfhi(w[2 * e]) * up;
      const float f2 = bflo(w[2 * e + 1]) * up, f3 = bfhi(w[2 * e + 1]) * up;
      if constexpr (kInt8) {
        auto code = [](float f) {
          return static_cast<uint32_t>(static_cast<int>(fminf(fmaxf(__builtin_rintf(f), -127.f), 127.f))) & 0xFFu;
        };
        codes[e] = code(f0) | code(f1) << 8 | code(f2) << 16 | code(f3) << 24;
      } else {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(f0, f1, 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(f2, f3, c, true);
        codes[e] = static_cast<uint32_t>(c);
      }
    }
  }
  if (!in || slot < 0) return;
  *reinterpret_cast<u32x4*>(p.codes + slot * D + part * 16) = codes;
  if (part == 0) p.scales[slot] = scale;
}

template <int D, bool kInt8, bool kNt>
__global__ __launch_bounds__(kThreads) void quant_load_kernel(QuantParams p, uint32_t rows) {
  constexpr int kLanes = D / 16;
  const uint32_t row = blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  const int part = threadIdx.x % kLanes;
  if (row >= rows) return;
  const Row r = row_of(p, row);
  const int64_t slot = slot_of(p, r, part == 0);
  if (slot < 0) return;
  const u32x4 codes = *reinterpret_cast<const u32x4*>(p.codes + slot * D + part * 16);
  const float scale = p.scales[slot];
  uint32_t w[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float f[4];
    if constexpr (kInt8) {
#pragma unroll
      for (int b = 0; b < 4; ++b) f[b] = static_cast<float>(static_cast<int8_t>(codes[e] >> (8 * b)));
    } else {
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes[e]), false);
      const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes[e]), true);
      f[0] = lo.x, f[1] = lo.y, f[2] = hi.x, f[3] = hi.y;
    }
    w[2 * e] = pack_bf2(f[0] * scale, f[1] * scale);
    w[2 * e + 1] = pack_bf2(f[2] * scale, f[3] * scale);
  }
  u32x4* dst = reinterpret_cast<u32x4*>((r.v ? p.v_out : p.k_out) + at_of(p, r) + part * 16);
  const u32x4 lo = {w[0], w[1], w[2], w[3]}, hi = {w[4], w[5], w[6], w[7]};
  if constexpr (kNt) {
    __builtin_nontemporal_store(lo, dst);
    __builtin_nontemporal_store(hi, dst + 1);
  } else {
    dst[0] = lo;
    dst[1] = hi;
  }
}

uint32_t row_count(const QuantParams& p) { return static_cast<uint32_t>(p.tokens) * 2 * p.Hkv; }
unsigned groups(const QuantParams& p) {
  const uint32_t per = kThreads / (p.d / 16);
  return (row_count(p) + per - 1) / per;
}

}  // namespace

hipError_t launch_quant_store(const QuantParams& p, hipStream_t s) {
  if (p.tokens == 0) return hipSuccess;
  const uint32_t rows = row_count(p);
  const unsigned grid = groups(p);
  if (p.d == 128 && p.int8) quant_store_kernel<128, true><<<grid, kThreads, 0, s>>>(p, rows);
  else if (p.d == 128) quant_store_kernel<128, false><<<grid, kThreads, 0, s>>>(p, rows);
  else if (p.d == 64 && p.int8) quant_store_kernel<64, true><<<grid, kThreads, 0, s>>>(p, rows);
  else if (p.d == 64) quant_store_kernel<64, false><<<grid, kThreads, 0, s>>>(p, rows);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

namespace {

template <int D, bool kInt8>
void load(const QuantParams& p, hipStream_t s) {
  const uint32_t rows = row_count(p);
  if (int64_t(rows) * D * 2 >= kNtStoreBytes) quant_load_kernel<D, kInt8, true><<<groups(p), kThreads, 0, s>>>(p, rows);
  else quant_load_kernel<D, kInt8, false><<<groups(p), kThreads, 0, s>>>(p, rows);
}

}  // namespace

hipError_t launch_quant_load(const QuantParams& p, hipStream_t s) {
  if (p.tokens == 0) return hipSuccess;
  if (p.d == 128 && p.int8) load<128, true>(p, s);
  else if (p.d == 128) load<128, false>(p, s);
  else if (p.d == 64 && p.int8) load<64, true>(p, s);
  else if (p.d == 64) load<64, false>(p, s);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pallas
