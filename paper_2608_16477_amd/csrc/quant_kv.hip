// An 8- or 4-bit KV cache: rows (one token's K or V of one head, d values) quantised as
// they are written into their page slots, and read back as bf16.
//
//   E4M3  scale = 2^e, the least with a <= 448 * 2^e (a: the row's largest
//         magnitude).  A power of two costs a floating-point code no precision and
//         makes both directions exact but for the code's own rounding (and for 2^128,
//         which the last 8 of bf16's magnitudes round to).
//   INT8  scale = a / 127: a power of two would cost up to one of seven bits.
//   E2M1  a scale 2^e for each quarter of the row, the least with a <= 6 * 2^e (a: the
//         quarter's): with two significant bits to a code a large value costs its
//         neighbours theirs, so fewer share a scale, and a power of two is one byte and
//         goes into the conversion instruction.
//
// All are bound by memory: 2 d bytes and d + 4 (E2M1: d / 2 + 4) bytes per row (34,708
// tokens of 8 heads of 128, E4M3, 217 MB each way: 42 us written, 42 read back, 5.2 TB/s;
// E2M1, 180 MB: 37 and 37, 4.8 TB/s).
// Codes are stored plainly (with non-temporal stores 87 us for both, and loads 86, in place
// of 84).  A lane takes 16 elements (two 16-byte vectors of bf16, one of 8-bit codes), d / 16
// neighbouring lanes a row, and neighbouring rows are the heads of a token, contiguous on
// both sides.
#include "common.h"
#include "kernels.h"
#include "quant_rows.h"

namespace pallas {

namespace {

constexpr int kThreads = 256;
constexpr int kPage = 16;
// Rows read back are stored non-temporally from this many bytes on (34,708 tokens of 8
// heads of 128 written and read back: 84 us, 97 with plain stores; 256 written and 3000 read:
// 8.0, 9.3); fewer stay in the caches for what reads them next.
constexpr int64_t kNtStoreBytes = int64_t(4) << 20;

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

template <int D, int kFormat>
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
  const RowCodes<16> q = quantise_row<kFormat, D, 16>(w);
  if (!in || slot < 0) return;
  if constexpr (kFormat == PALLAS_QUANT_E2M1) {
    constexpr int kGroup = D / 64;      // lanes of a group
    *reinterpret_cast<u32x2*>(p.codes + slot * (D / 2) + part * 8) = u32x2{q.codes[0], q.codes[1]};
    if (part % kGroup == 0) reinterpret_cast<uint8_t*>(p.scales)[slot * 4 + part / kGroup] = static_cast<uint8_t>(q.scale);
  } else {
    *reinterpret_cast<u32x4*>(p.codes + slot * D + part * 16) = u32x4{q.codes[0], q.codes[1], q.codes[2], q.codes[3]};
    if (part == 0) p.scales[slot] = __uint_as_float(q.scale);
  }
}

template <int D, int kFormat, bool kNt>
__global__ __launch_bounds__(kThreads) void quant_load_kernel(QuantParams p, uint32_t rows) {
  constexpr int kLanes = D / 16;
  const uint32_t row = blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  const int part = threadIdx.x % kLanes;
  if (row >= rows) return;
  const Row r = row_of(p, row);
  const int64_t slot = slot_of(p, r, part == 0);
  if (slot < 0) return;
  u32x4 lo, hi;
  if constexpr (kFormat == PALLAS_QUANT_E2M1) {
    const u32x2 codes = *reinterpret_cast<const u32x2*>(p.codes + slot * (D / 2) + part * 8);
    const uint32_t byte = reinterpret_cast<const uint8_t*>(p.scales)[slot * 4 + part / (D / 64)];
    const float unit = __uint_as_float(byte << 23);
    lo = e2m1_bf16(codes.x, unit);
    hi = e2m1_bf16(codes.y, unit);
  } else {
    const u32x4 codes = *reinterpret_cast<const u32x4*>(p.codes + slot * D + part * 16);
    const float scale = p.scales[slot];
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4 f = code_values<kFormat>(codes[e]);
      w[2 * e] = pack_bf2(f[0] * scale, f[1] * scale);
      w[2 * e + 1] = pack_bf2(f[2] * scale, f[3] * scale);
    }
    lo = u32x4{w[0], w[1], w[2], w[3]};
    hi = u32x4{w[4], w[5], w[6], w[7]};
  }
  u32x4* dst = reinterpret_cast<u32x4*>((r.v ? p.v_out : p.k_out) + at_of(p, r) + part * 16);
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

template <int D>
void store(const QuantParams& p, hipStream_t s) {
  for_format(p.format, [&](auto f) { quant_store_kernel<D, f.value><<<groups(p), kThreads, 0, s>>>(p, row_count(p)); });
}

template <int D>
void load(const QuantParams& p, hipStream_t s) {
  const uint32_t rows = row_count(p);
  for_format(p.format, [&](auto f) {
    if (int64_t(rows) * D * 2 >= kNtStoreBytes) quant_load_kernel<D, f.value, true><<<groups(p), kThreads, 0, s>>>(p, rows);
    else quant_load_kernel<D, f.value, false><<<groups(p), kThreads, 0, s>>>(p, rows);
  });
}

}  // namespace

hipError_t launch_quant_store(const QuantParams& p, hipStream_t s) {
  if (p.tokens == 0) return hipSuccess;
  if (p.d == 128) store<128>(p, s);
  else if (p.d == 64) store<64>(p, s);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_quant_load(const QuantParams& p, hipStream_t s) {
  if (p.tokens == 0) return hipSuccess;
  if (p.d == 128) load<128>(p, s);
  else if (p.d == 64) load<64>(p, s);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pallas
