// Which blocks of a long context a query attends to: bounds of the keys of each 16-position
// block (one page of a block table), and the blocks that score highest against them.
//
// Bounds are the elementwise largest and smallest key of a block, INT8 with one scale: for a
// query q, sum_i max(q_i, 0) top_i + min(q_i, 0) low_i is at least every q . k of the block,
// up to the rounding of both.  Queries are INT8 too, with a scale each, so that the sums are
// whole numbers (below 2^24 in magnitude, so exact in float32 as well) and v_mfma_i32_16x16x64_i8
// takes them: which blocks are selected depends on no order of summation.
//
// Bounds of many keys are bound by reading them (8 sequences of 1505 to 6441 keys, bf16, 53 MB of K, 11.6
// us, 4.6 TB/s; those of one new token a sequence are a chain of loads, 2.6 to 3.1).  A score reads 260
// bytes of a block (head of 128) in place of its keys' 8192 (64 sequences of 2000 to 16,000 keys, 56 MB,
// 14.6, 3.8 TB/s); selection works in LDS on what one workgroup reads of a row, 7 us up to
// 2048 blocks and 10 for 8192, most of it barriers.
#include "common.h"
#include "kernels.h"
#include "paged_attn.h"
#include "quant_rows.h"

namespace pallas {

namespace {

constexpr int kPage = 16;
constexpr int kThreads = 256;
typedef int i32x4 __attribute__((ext_vector_type(4)));

// The step that `top` takes 127 of, and what turns values into steps (0: all count as zero).
struct Step {
  float step, up;
};
__device__ __forceinline__ Step step_of(float top) {
  if (!(top < INFINITY)) return {__uint_as_float(kNanScale), 0.f};      // an infinity or a NaN
  if (top < 0x1p-100f) return {0.f, 0.f};
  return {top / 127.0f, 127.0f / top};
}
__device__ __forceinline__ uint32_t step_codes(const float* x, float up) {
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = up == 0.f ? 0 : static_cast<int>(fminf(fmaxf(__builtin_rintf(x[e] * up), -127.f), 127.f));
    w |= (static_cast<uint32_t>(c) & 0xFFu) << (8 * e);
  }
  return w;
}

// What the lanes of one part of a row hold: lanes l, l ^ 32, l ^ 16 and, of 64 dimensions, l ^ 8.
template <int kLanes, class F>
__device__ __forceinline__ uint32_t over_rows(uint32_t v, F f) {
  auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = f(r[0], r[1]);
  r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = f(r[0], r[1]);
  if constexpr (kLanes == 8) v = f(v, dpp_word<kDppRor8>(v));
  return v;
}

typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_i16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
}
__device__ __forceinline__ uint32_t min_i16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
}
// Two bf16 values as signed integers of the same order (NaN outside all others), and back.
__device__ __forceinline__ uint32_t ordered_bf2(uint32_t w) {
  const i16x2 sign = __builtin_bit_cast(i16x2, w) >> 15;
  return w ^ (__builtin_bit_cast(uint32_t, sign) & 0x7FFF7FFFu);
}

// A wave per block and KV head, of each sequence: where two hold a page their waves write the same, or
// the caller keeps them apart (codes and step are two stores, which nothing orders between workgroups).
// D / 8 lanes take a row, eight values each.  Rows of bf16 and
// E2M1 are (these, with their scales, exactly, but for magnitudes too small to be of a block that
// is not zero) bf16 values, which order as integers: two to an instruction, and infinities and
// NaN show at the end.  8-bit rows are products in float32.
template <int D, CacheType T>
__global__ __launch_bounds__(kThreads) void bounds_kernel(BoundsParams p, int per_seq) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes, kReads = kPage / kRows;
  const int item = static_cast<int>(blockIdx.x) * (kThreads / 64) + static_cast<int>(threadIdx.x >> 6);   // heads of a block side by side
  const int lane = threadIdx.x & 63, part = lane % kLanes, sub = lane / kLanes;
  const int nth = item / p.Hkv, h = item - nth * p.Hkv, s = blockIdx.y;
  if (nth >= per_seq) return;
  const int from = p.start[s], len = p.lengths[s];
  if (from < 0 || from >= len) return;              // padding, or nothing due
  if (p.err && item == 0 && lane == 0) {
    // (No wave has a block that lies behind `per_seq`, a table's width at most.)
    const int last = min((len - 1) / kPage, from / kPage + bounds_blocks(p.most) - 1);
    if (len - from > p.most) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_LENGTH));
    if (last >= p.max_pages) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
  }
  const int64_t j = from / kPage + nth;
  if (j * kPage >= len) return;
  const int pg = j < p.max_pages ? p.bt[static_cast<int64_t>(s) * p.max_pages + j] : -1;
  if (pg < 0 || pg >= p.num_pages) {
    if (p.err && h == 0 && lane == 0) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
    return;
  }
  const int keys = static_cast<int>(min(len - j * kPage, static_cast<int64_t>(kPage)));
  // (Rows behind the last key read it again.)
  auto row = [&](int n) { return (static_cast<int64_t>(pg) * kPage + min(n * kRows + sub, keys - 1)) * p.Hkv + h; };
  float x[8];           // of the largest (lanes of the first row) or the smallest key
  float a;              // the largest magnitude of both, over the row
  if constexpr (T == kCacheInt8 || T == kCacheE4m3) {
    constexpr int kFormat = T == kCacheInt8 ? PALLAS_QUANT_INT8 : PALLAS_QUANT_E4M3;
    u32x2 c[kReads];
    float scale[kReads], top[8], low[8];
#pragma unroll
    for (int n = 0; n < kReads; ++n) {
      c[n] = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(p.k) + row(n) * D + part * 8);
      scale[n] = p.scales[row(n)];
    }
    bool odd = false;
#pragma unroll
    for (int n = 0; n < kReads; ++n) {
      odd |= !(scale[n] < INFINITY);
      const f32x4 lo = code_values<kFormat>(c[n].x), hi = code_values<kFormat>(c[n].y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = (e < 4 ? lo[e % 4] : hi[e % 4]) * scale[n];
        if constexpr (T == kCacheE4m3) odd |= v != v;      // (a code, too, can be NaN)
        top[e] = n == 0 ? v : fmaxf(top[e], v);
        low[e] = n == 0 ? v : fminf(low[e], v);
      }
    }
    a = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      auto larger = [](uint32_t u, uint32_t v) { return __float_as_uint(fmaxf(__uint_as_float(u), __uint_as_float(v))); };
      const float hi = __uint_as_float(over_rows<kLanes>(__float_as_uint(top[e]), larger));
      const float lo = -__uint_as_float(over_rows<kLanes>(__float_as_uint(-low[e]), larger));
      a = fmaxf(a, fmaxf(fabsf(hi), fabsf(lo)));
      x[e] = sub == 0 ? hi : lo;
    }
    a = row16_max(a);      // (of 64: both halves hold the same)
    if (__builtin_amdgcn_ballot_w64(odd) != 0) a = INFINITY;
  } else {
    u32x4 w[kReads];
#pragma unroll
    for (int n = 0; n < kReads; ++n) {
      if constexpr (T == kCacheBf16) {
        w[n] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.k) + row(n) * D + part * 8);
      } else if constexpr (T == kCacheE2m1) {
        w[n].x = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(p.k) + row(n) * (D / 2) + part * 4);
        w[n].y = static_cast<uint32_t>(reinterpret_cast<const uint8_t*>(p.scales)[row(n) * 4 + part / (D / 32)]);
      }
    }
    uint32_t top[4], low[4];
#pragma unroll
    for (int n = 0; n < kReads; ++n) {
      if constexpr (T == kCacheE2m1) {
        w[n] = e2m1_bf16(w[n].x, __uint_as_float(w[n].y << 23));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t o = ordered_bf2(w[n][e]);
        top[e] = n == 0 ? o : max_i16x2(top[e], o);
        low[e] = n == 0 ? o : min_i16x2(low[e], o);
      }
    }
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t hi = ordered_bf2(over_rows<kLanes>(top[e], max_i16x2)), lo = ordered_bf2(over_rows<kLanes>(low[e], min_i16x2));
      most = max_u16x2(most, max_u16x2(hi & 0x7FFF7FFFu, lo & 0x7FFF7FFFu));
      x[2 * e] = bflo(sub == 0 ? hi : lo), x[2 * e + 1] = bfhi(sub == 0 ? hi : lo);
    }
    a = __uint_as_float(lanes_top<16>(most) << 16);
  }
  const Step st = step_of(a);
  const int64_t to = static_cast<int64_t>(pg) * p.Hkv + h;
  if (sub < 2) *reinterpret_cast<u32x2*>(p.bounds + (to * 2 + sub) * D + part * 8) = u32x2{step_codes(x, st.up), step_codes(x + 4, st.up)};
  if (lane == 0) p.bound_scales[to] = st.step;
}

// Over all lanes of a wave, and inclusive sums.
template <class F>
__device__ __forceinline__ uint32_t over_wave(uint32_t v, F f) {
  v = over_rows<16>(v, f);
  v = f(v, dpp_word<kDppRor8>(v));
  v = f(v, dpp_word<kDppRor4>(v));
  v = f(v, dpp_word<kDppXor2>(v));
  return f(v, dpp_word<kDppXor1>(v));
}
__device__ __forceinline__ uint32_t wave_sums(uint32_t v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // row_bcast:31 into rows 2 and 3
  return v;
}

// ------------------------------------------------------------ scores
// Scores order as these: negative numbers turned over, NaN above all, and what is always
// selected above that.
constexpr uint32_t kAlways = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return kAlways - 1;
  const uint32_t b = __float_as_uint(x + 0.0f);      // (-0 is 0)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A wave takes up to kRuns runs of 16 blocks of one KV head and up to 16 of its query heads (others
// in further passes): Q as the MFMA's rows, blocks as its columns, so that lane l holds heads 4 (l /
// 16) + r against block l mod 16.  `runs` runs of a row of `blocks`: first, first + step, ..;
// put(block, score, pass) keeps a score, or the larger of two passes'.  Pages of all runs are read
// together, bounds a run ahead, and the first of both before the query is worked on.
constexpr int kRun = 16;
constexpr int kHeads = 16;
constexpr int kRuns = 4;
template <int D>
struct Ahead {
  int pages[kRuns];
  u32x4 w[D / 64][2];      // 16 elements of each 64 of head l16 (the last again where there are fewer)

  // (Entries behind the row's: no use, but within the table.)
  __device__ __forceinline__ void read_pages(const SelectParams& p, int s, int first, int step) {
#pragma unroll
    for (int n = 0; n < kRuns; ++n)
      pages[n] = p.bt[static_cast<int64_t>(s) * p.max_pages + min((first + n * step) * kRun + static_cast<int>(threadIdx.x & 15), p.max_pages - 1)];
  }
  __device__ __forceinline__ void read_q(const SelectParams& p, int s, int kh, int g0) {
    const int lane = threadIdx.x & 63, q4 = lane >> 4, l16 = lane & 15;
    const uint16_t* q = p.q + s * p.q_stride + static_cast<int64_t>(kh * p.G + g0 + min(l16, min(kHeads, p.G - g0) - 1)) * D;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) w[c][i] = *reinterpret_cast<const u32x4*>(q + 64 * c + 16 * q4 + 8 * i);
  }
};
template <int D, class Put>
__device__ __forceinline__ void score_runs(const SelectParams& p, Ahead<D>& a, int s, int kh, int blocks, int first, int step, int runs, Put put) {
  const int lane = threadIdx.x & 63, q4 = lane >> 4, l16 = lane & 15;
  for (int g0 = 0; g0 < p.G; g0 += kHeads) {
    if (g0 > 0) {
      a.read_pages(p, s, first, step);
      a.read_q(p, s, kh, g0);
    }
    i32x4 top[2][D / 64], low[2][D / 64];
    float scale[2];
    auto inside = [&](int pg) { return pg >= 0 && pg < p.num_pages; };
    auto read = [&](int pg, int to) {
      const int64_t at = static_cast<int64_t>(inside(pg) ? pg : 0) * p.Hkv + kh;
      const int8_t* b = p.bounds + at * 2 * D + 16 * q4;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        top[to][c] = *reinterpret_cast<const i32x4*>(b + 64 * c);
        low[to][c] = *reinterpret_cast<const i32x4*>(b + D + 64 * c);
      }
      scale[to] = p.bound_scales[at];
    };
    read(a.pages[0], 0);
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) most = max_u16x2(most, a.w[c][i][e] & 0x7FFF7FFFu);
    // (As bits, in which a NaN is larger than any number.)
    most = over_rows<16>(max(most & 0xFFFFu, most >> 16), [](uint32_t u, uint32_t v) { return max(u, v); });
    const Step st = step_of(__uint_as_float(most << 16));
    i32x4 up[D / 64], down[D / 64];      // positive codes, negative codes
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo = a.w[c][e / 2][e % 2 * 2], hi = a.w[c][e / 2][e % 2 * 2 + 1];
        const float x[4] = {bflo(lo), bfhi(lo), bflo(hi), bfhi(hi)};
        const uint32_t codes = step_codes(x, st.up), sign = (codes >> 7 & 0x01010101u) * 255u;
        up[c][e] = static_cast<int>(codes & ~sign);
        down[c][e] = static_cast<int>(codes & sign);
      }
    float unit[4];      // steps of heads 4 q4 + r
#pragma unroll
    for (int r = 0; r < 4; ++r) unit[r] = __shfl(st.step, 4 * q4 + r, 64);
#pragma unroll
    for (int n = 0; n < kRuns; ++n) {
      if (n >= runs) break;
      if (n + 1 < kRuns) read(a.pages[n + 1], (n + 1) % 2);
      i32x4 dot = {0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(up[c], top[n % 2][c], dot, 0, 0, 0);
        dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(down[c], low[n % 2][c], dot, 0, 0, 0);
      }
      uint32_t best = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r) best = max(best, order_of(static_cast<float>(dot[r]) * scale[n % 2] * unit[r]));
      best = over_rows<16>(best, [](uint32_t u, uint32_t v) { return max(u, v); });
      const bool bad = !inside(a.pages[n]);
      if (bad) best = 0;      // (the keys of such a block are masked)
      const int b = (first + n * step) * kRun + l16;
      if (b < p.first || b >= blocks - p.last) best = kAlways;
      if (q4 == 0 && b < blocks) {
        put(b, best, g0);
        if (p.err && bad && kh == 0 && g0 == 0) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
      }
    }
  }
}

__device__ __forceinline__ int row_blocks(const SelectParams& p, int s) {
  return (min(max(p.lengths[s], 0), p.max_length) + kPage - 1) / kPage;      // (max_length: at most 2^30)
}

// Scores of long rows, spread over the chip: waves of a workgroup take the heads of the same
// blocks, which are neighbours in memory.
template <int D>
__global__ __launch_bounds__(kThreads) void score_kernel(SelectParams p, int per_wave) {
  const int s = blockIdx.y;
  // (Rotated from row to row: else an XCD takes the same blocks of all rows, and the one with the first
  // blocks has more than that with the last; 64 rows of 2000 to 16,000 keys 29.1 us, 22.4.)
  const int unit = static_cast<int>((blockIdx.x + blockIdx.y) % gridDim.x) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kh = unit % p.Hkv, first = unit / p.Hkv * per_wave;
  Ahead<D> a;
  a.read_pages(p, s, first, 1);
  a.read_q(p, s, kh, 0);
  const int blocks = row_blocks(p, s);
  if (blocks <= p.budget || first * kRun >= blocks) return;      // all are selected, or none here
  uint32_t* out = p.order + (static_cast<int64_t>(s) * p.Hkv + kh) * p.stride;
  score_runs<D>(p, a, s, kh, blocks, first, 1, min((blocks + kRun - 1) / kRun - first, per_wave), [&](int b, uint32_t x, int pass) { out[b] = pass == 0 ? x : max(x, out[b]); });
}

// ------------------------------------------------------------ selection
// One workgroup per (sequence, KV head).  Of the scores that are not selected in any case, those
// between a least and a largest one hold the last that is selected, the `want`-th of them: they are
// counted in kBins equal steps, the step it is in becomes the new range, until all of a step are
// selected, or a step is one score (of which the earliest are).  (Steps of what is left of the
// range, not digits: scores lie within a few powers of two, whose high digits are one.)  Then what is
// selected is listed in order.  Counts are whole numbers: the same in every run.
//   kScored: the scores of the row are worked out here first, into LDS.
constexpr int kBins = 2048;
constexpr int kEach = 8;        // scores that a thread keeps
constexpr int kShortBlocks = 128;   // of a row that is scored where it is selected: two runs a wave
template <int D, int kWide, bool kScored>
__global__ __launch_bounds__(kWide) void select_kernel(SelectParams p) {
  constexpr int kWaves = kWide / 64, kPass = kWide * kEach;
  static_assert(!kScored || kShortBlocks <= kWaves * kRuns * kRun, "a wave's runs");
  __shared__ uint32_t bins[kBins];
  __shared__ uint32_t scored[kScored ? kShortBlocks : 1];
  __shared__ uint32_t lows[kWaves], highs[kWaves], sums[kWaves], found[3];
  __shared__ uint32_t counts[2][kEach * kWaves];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int kh = blockIdx.x, s = blockIdx.y;
  Ahead<D> a;
  if constexpr (kScored) {
    a.read_pages(p, s, wave, kWaves);
    a.read_q(p, s, kh, 0);
  }
  // (Scores of the first pass are read beside the length; those behind the row count as none.)
  const uint32_t* in = p.order + (static_cast<int64_t>(s) * p.Hkv + kh) * p.stride;
  uint32_t x[kEach];
  if constexpr (!kScored) {
#pragma unroll
    for (int k = 0; k < kEach; ++k) x[k] = in[min(k * kWide + t, static_cast<int>(p.stride) - 1)];
  }
  const int full = p.lengths[s], blocks = row_blocks(p, s);
  if (p.err && kh == 0 && t == 0 && full != min(max(full, 0), p.max_length)) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_LENGTH));
  int32_t* out = p.blocks + (static_cast<int64_t>(s) * p.Hkv + kh) * p.budget;
  if (blocks <= p.budget) {
    for (int i = t; i < p.budget; i += kWide) out[i] = i < blocks ? i : -1;
    return;
  }
  if constexpr (kScored) {
    const int runs = ((blocks + kRun - 1) / kRun - wave + kWaves - 1) / kWaves;
    if (runs > 0) score_runs<D>(p, a, s, kh, blocks, wave, kWaves, runs, [&](int b, uint32_t x, int pass) { scored[b] = pass == 0 ? x : max(x, scored[b]); });
    in = scored;
    __syncthreads();
  }
  // Score k of the thread in a pass is of block k kWide + t of it; those behind the row are 0.
  const int passes = (blocks + kPass - 1) / kPass;
  auto load = [&](int pass) {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int i = pass * kPass + k * kWide + t;
      x[k] = i < blocks ? in[i] : 0;
    }
  };
  if constexpr (kScored) load(0);
#pragma unroll
  for (int k = 0; k < kEach; ++k) x[k] = k * kWide + t < blocks ? x[k] : 0;
  uint32_t low = kAlways, high = 0;
  for (int pass = 0; pass < passes; ++pass) {
    if (pass > 0) load(pass);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const bool open = pass * kPass + k * kWide + t < blocks && x[k] != kAlways;
      low = min(low, open ? x[k] : kAlways);
      high = max(high, open ? x[k] : 0u);
    }
  }
  auto least = [](uint32_t u, uint32_t v) { return min(u, v); };
  auto largest = [](uint32_t u, uint32_t v) { return max(u, v); };
  low = over_wave(low, least);
  high = over_wave(high, largest);
  if (lane == 0) lows[wave] = low, highs[wave] = high;
  for (int i = t; i < kBins; i += kWide) bins[i] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) low = min(low, lows[w]), high = max(high, highs[w]);
  uint32_t want = p.budget - p.first - p.last;
  bool all = want == 0;      // all of [low, high] are selected (none: it lies above every score)
  if (all) low = high = kAlways;
  // (Four rounds at most, 2^32 of 2^21 to begin with; counted, so that scores that another call changes
  // meanwhile end too.)
  for (int round = 0; round < 4 && !all && low < high; ++round) {
    // Of 2^shift scores each, at most kBins.
    const int shift = max(32 - __builtin_clz(high - low) - 11, 0);
    for (int pass = 0; pass < passes; ++pass) {
      if (passes > 1) load(pass);
#pragma unroll
      for (int k = 0; k < kEach; ++k)
        if (pass * kPass + k * kWide + t < blocks && x[k] >= low && x[k] <= high) atomicAdd(&bins[(x[k] - low) >> shift], 1u);
    }
    __syncthreads();
    // Thread t: bins from the top, kBins / kWide of them.
    constexpr int kMine = kBins / kWide;
    uint32_t n[kMine], sum = 0;
#pragma unroll
    for (int e = 0; e < kMine; ++e) sum += n[e] = bins[kBins - 1 - kMine * t - e];
    const uint32_t upto = wave_sums(sum);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    uint32_t above = upto - sum;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) above += w < wave ? sums[w] : 0;
    if (above < want && above + sum >= want) {
      bool here = false;
#pragma unroll
      for (int e = 0; e < kMine; ++e) {
        if (!here && above + n[e] >= want) {
          here = true;
          found[0] = kBins - 1 - kMine * t - e;
          found[1] = want - above;
          found[2] = n[e];
        }
        above += n[e];
      }
    }
#pragma unroll
    for (int e = 0; e < kMine; ++e) bins[kBins - 1 - kMine * t - e] = 0;
    __syncthreads();
    low += found[0] << shift;
    high = low + min(high - low, (1u << shift) - 1);      // (the topmost step can end behind 2^32)
    want = found[1];
    all = found[2] == want;
  }
  // In order: what is above `high`, and of [low, high] all, or the first `want`.
  uint32_t more0 = 0, same0 = 0;      // before this pass
  for (int pass = 0; pass < passes; ++pass) {
    if (passes > 1) {
      load(pass);
      __syncthreads();
    }
    uint64_t more[kEach], same[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const bool in_row = pass * kPass + k * kWide + t < blocks;
      const bool mid = in_row && x[k] >= low && x[k] <= high;
      more[k] = __builtin_amdgcn_ballot_w64(in_row && (x[k] > high || x[k] == kAlways || (all && mid)));
      same[k] = __builtin_amdgcn_ballot_w64(!all && mid && x[k] != kAlways);
      if (lane == 0) {
        counts[0][k * kWaves + wave] = __builtin_popcountll(more[k]);
        counts[1][k * kWaves + wave] = __builtin_popcountll(same[k]);
      }
    }
    __syncthreads();
    // Exclusive sums over (k, wave), in order; the whole behind them.
    if (wave < 2) {
      constexpr int kMine = (kEach * kWaves + 63) / 64;
      uint32_t n[kMine], sum = 0;
#pragma unroll
      for (int e = 0; e < kMine; ++e) {
        const int i = lane * kMine + e;
        n[e] = i < kEach * kWaves ? counts[wave][i] : 0;
        sum += n[e];
      }
      uint32_t before = wave_sums(sum) - sum;
      if (lane == 63) found[wave] = before + sum;
#pragma unroll
      for (int e = 0; e < kMine; ++e) {
        const int i = lane * kMine + e;
        if (i < kEach * kWaves) counts[wave][i] = before;
        before += n[e];
      }
    }
    __syncthreads();
    const uint64_t below = (uint64_t(1) << lane) - 1;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const bool m = more[k] >> lane & 1, e = same[k] >> lane & 1;
      const uint32_t ms = more0 + counts[0][k * kWaves + wave] + __builtin_popcountll(more[k] & below);
      const uint32_t es = same0 + counts[1][k * kWaves + wave] + __builtin_popcountll(same[k] & below);
      const uint32_t to = ms + (all ? 0 : min(es, want));
      if ((m || (e && es < want)) && to < static_cast<uint32_t>(p.budget)) out[to] = pass * kPass + k * kWide + t;
    }
    more0 += found[0], same0 += found[1];
    if (pass + 1 < passes) __syncthreads();
  }
}

// Short rows are scored where they are selected, one launch (us; in two: 1 row of 2000 keys, 8 KV
// heads, 8.0 (10.7), 64 of them 10.8 (12.9), 128 of 1000 12.8 (13.7)); a workgroup that scores longer ones
// is longer than the chip's way to the second launch (1 row of 4000 12.0 (10.8), 64 of 2000 to 16,000 31
// (28.5)).
template <int D>
hipError_t launch_selection(const SelectParams& p, hipStream_t s) {
  const int most = (p.max_length + kPage - 1) / kPage;
  const dim3 grid(p.Hkv, p.seqs);
  if (most > p.budget && most <= kShortBlocks) {
    select_kernel<D, 256, true><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
  }
  if (most > p.budget) {
    // Runs of a wave, whose work on its queries is once: as many as leave waves for the chip (us with 1,
    // 2 and 4: 1 row of 8000 keys 9.7, 10.0, 11.0; 8 of 1000 to 8000 11.0, 10.3, 11.3; 1 of 131,071 18.1,
    // 16.2, 15.3; 64 of 32,000 99, 80, 67, with 8 and 16 the same).
    const int64_t runs = (int64_t(most) + kRun - 1) / kRun, all = runs * p.Hkv * p.seqs;
    const int per_wave = all < 2048 ? 1 : all < 4096 ? 2 : kRuns;
    const int64_t units = (runs + per_wave - 1) / per_wave * p.Hkv;
    score_kernel<D><<<dim3(static_cast<unsigned>((units + 3) / 4), p.seqs), kThreads, 0, s>>>(p, per_wave);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (most <= 256 * kEach) select_kernel<D, 256, false><<<grid, 256, 0, s>>>(p);
  else select_kernel<D, 1024, false><<<grid, 1024, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_bounds(const BoundsParams& p, CacheType type, hipStream_t s) {
  const int per_seq = std::min(bounds_blocks(p.most), p.max_pages);
  const dim3 grid((static_cast<unsigned>(per_seq) * p.Hkv + 3) / 4, p.seqs);
  auto run = [&](auto d, auto t) { bounds_kernel<d.value, t.value><<<grid, kThreads, 0, s>>>(p, per_seq); };
  auto of = [&](auto d) {
    if (type == kCacheBf16) run(d, std::integral_constant<CacheType, kCacheBf16>());
    else if (type == kCacheE4m3) run(d, std::integral_constant<CacheType, kCacheE4m3>());
    else if (type == kCacheInt8) run(d, std::integral_constant<CacheType, kCacheInt8>());
    else run(d, std::integral_constant<CacheType, kCacheE2m1>());
  };
  if (p.d == 128) of(std::integral_constant<int, 128>());
  else if (p.d == 64) of(std::integral_constant<int, 64>());
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_select(const SelectParams& p, hipStream_t s) {
  if (p.d == 128) return launch_selection<128>(p, s);
  if (p.d == 64) return launch_selection<64>(p, s);
  return hipErrorInvalidValue;
}

}  // namespace pallas
