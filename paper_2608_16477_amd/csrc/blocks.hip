// Which blocks of a long context a query attends to: bounds of the keys of each 16-position
// block (one page of a block table), and the blocks that score highest against them.
//
// Bounds are the elementwise largest and smallest key of a block, INT8 with one scale: for a
// query q, sum_i max(q_i, 0) top_i + min(q_i, 0) low_i is at least every q . k of the block,
// up to the rounding of both.  Queries are INT8 too, with a scale each, so that the sums are
// whole numbers (below 2^24 in magnitude, so exact in float32 as well) and v_mfma_i32_16x16x64_i8
// takes them: which blocks are selected depends on no order of summation.
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

// Eight values of a cached K row.
template <CacheType T, int D>
__device__ __forceinline__ void read_row8(const BoundsParams& p, int64_t row, int part, float (&x)[8]) {
  if constexpr (T == kCacheBf16 || T == kCacheE2m1) {
    u32x4 w;
    if constexpr (T == kCacheBf16) {
      w = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.k) + row * D + part * 8);
    } else {
      const uint32_t c = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(p.k) + row * (D / 2) + part * 4);
      const uint32_t unit = reinterpret_cast<const uint8_t*>(p.scales)[row * 4 + part / (D / 32)];
      w = e2m1_bf16(c, __uint_as_float(unit << 23));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[2 * e] = bflo(w[e]), x[2 * e + 1] = bfhi(w[e]);
  } else {
    constexpr int kFormat = T == kCacheInt8 ? PALLAS_QUANT_INT8 : PALLAS_QUANT_E4M3;
    const u32x2 c = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(p.k) + row * D + part * 8);
    const float scale = p.scales[row];
    const f32x4 lo = code_values<kFormat>(c.x), hi = code_values<kFormat>(c.y);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = lo[e] * scale, x[4 + e] = hi[e] * scale;
  }
}

// A wave per block and KV head: D / 8 lanes take a row, eight values each.
template <int D, CacheType T>
__global__ __launch_bounds__(kThreads) void bounds_kernel(BoundsParams p, int per_seq) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes;
  const int item = static_cast<int>(blockIdx.x) * (kThreads / 64) + static_cast<int>(threadIdx.x >> 6);   // heads of a block side by side
  const int lane = threadIdx.x & 63, part = lane % kLanes, sub = lane / kLanes;
  const int nth = item / p.Hkv, h = item - nth * p.Hkv, s = blockIdx.y;
  if (nth >= per_seq) return;
  const int from = p.start[s], len = p.lengths[s];
  if (from < 0 || from >= len) return;              // padding, or nothing due
  if (p.err && item == 0 && lane == 0 && len - from > p.most) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_LENGTH));
  const int64_t j = from / kPage + nth;
  if (j * kPage >= len) return;
  const int pg = j < p.max_pages ? p.bt[static_cast<int64_t>(s) * p.max_pages + j] : -1;
  if (pg < 0 || pg >= p.num_pages) {
    if (p.err && h == 0 && lane == 0) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
    return;
  }
  const int keys = static_cast<int>(min(len - j * kPage, static_cast<int64_t>(kPage)));
  float top[8], low[8];
  bool odd = false;      // an infinity or a NaN
#pragma unroll
  for (int e = 0; e < 8; ++e) top[e] = -INFINITY, low[e] = INFINITY;
#pragma unroll
  for (int n = 0; n < kPage / kRows; ++n) {
    const int r = n * kRows + sub;
    // (Rows behind the last key read it again.)
    float x[8];
    read_row8<T, D>(p, (static_cast<int64_t>(pg) * kPage + min(r, keys - 1)) * p.Hkv + h, part, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      odd |= !(fabsf(x[e]) < INFINITY);
      top[e] = fmaxf(top[e], x[e]);
      low[e] = fminf(low[e], x[e]);
    }
  }
  // Over the rows: lanes l, l ^ 32, l ^ 16 and, of 64, l ^ 8.
  float a = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    top[e] = rows_max(top[e]);
    low[e] = -rows_max(-low[e]);
    if constexpr (kLanes == 8) {
      top[e] = fmaxf(top[e], dpp_read<kDppRor8>(top[e]));
      low[e] = fminf(low[e], dpp_read<kDppRor8>(low[e]));
    }
    a = fmaxf(a, fmaxf(fabsf(top[e]), fabsf(low[e])));
  }
  a = row16_max(a);      // (of 64: both halves hold the same)
  const Step st = step_of(__builtin_amdgcn_ballot_w64(odd) != 0 ? INFINITY : a);
  const int64_t to = static_cast<int64_t>(pg) * p.Hkv + h;
  if (sub < 2) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = sub == 0 ? top[e] : low[e];
    *reinterpret_cast<u32x2*>(p.bounds + (to * 2 + sub) * D + part * 8) = u32x2{step_codes(y, st.up), step_codes(y + 4, st.up)};
  }
  if (lane == 0) p.bound_scales[to] = st.step;
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

// A wave takes runs of 16 blocks of one KV head and up to 16 of its query heads (others in
// further passes): Q as the MFMA's rows, blocks as its columns, so that lane l holds heads 4 (l /
// 16) + r against block l mod 16.
constexpr int kRun = 16;
constexpr int kHeads = 16;
template <int D>
__global__ __launch_bounds__(kThreads) void score_kernel(SelectParams p, int per_wave) {
  const int lane = threadIdx.x & 63, q4 = lane >> 4, l16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // A workgroup's waves take the heads of the same blocks, which are neighbours in memory.
  const int s = blockIdx.y;
  const int unit = static_cast<int>(blockIdx.x) * (kThreads / 64) + wave;
  const int kh = unit % p.Hkv, first = unit / p.Hkv * per_wave * kRun;
  const int len = min(max(p.lengths[s], 0), p.max_length), blocks = (len + kPage - 1) / kPage;
  if (blocks <= p.budget || first >= blocks) return;      // all are selected, or none here
  const int stop = min(first + per_wave * kRun, blocks);
  for (int g0 = 0; g0 < p.G; g0 += kHeads) {
    // Lane: 16 elements of each 64 of head l16 (the last again where there are fewer).
    const int nh = min(kHeads, p.G - g0);
    const uint16_t* q = p.q + s * p.q_stride + static_cast<int64_t>(kh * p.G + g0 + min(l16, nh - 1)) * D;
    float x[D / 64][16];
    float a = 0.f;
    bool odd = false;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(q + 64 * c + 16 * q4 + 8 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[c][8 * i + 2 * e] = bflo(w[e]), x[c][8 * i + 2 * e + 1] = bfhi(w[e]);
          odd |= (w[e] & 0x7F80u) == 0x7F80u || (w[e] & 0x7F800000u) == 0x7F800000u;
          a = fmaxf(a, fmaxf(fabsf(bflo(w[e])), fabsf(bfhi(w[e]))));
        }
      }
    a = rows_max(odd ? INFINITY : a);
    const Step st = step_of(a);
    i32x4 up[D / 64], down[D / 64];      // positive codes, negative codes
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float pos[4], neg[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) pos[b] = fmaxf(x[c][4 * e + b], 0.f), neg[b] = fminf(x[c][4 * e + b], 0.f);
        up[c][e] = static_cast<int>(step_codes(pos, st.up));
        down[c][e] = static_cast<int>(step_codes(neg, st.up));
      }
    float step[4];      // of heads 4 q4 + r
#pragma unroll
    for (int r = 0; r < 4; ++r) step[r] = __shfl(st.step, 4 * q4 + r, 64);
    for (int b0 = first; b0 < stop; b0 += kRun) {
      const int j = min(b0 + l16, blocks - 1);
      const int pg = p.bt[static_cast<int64_t>(s) * p.max_pages + j];
      const bool bad = pg < 0 || pg >= p.num_pages;
      const int64_t at = static_cast<int64_t>(bad ? 0 : pg) * p.Hkv + kh;
      const int8_t* b = p.bounds + at * 2 * D + 16 * q4;
      i32x4 dot = {0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(up[c], *reinterpret_cast<const i32x4*>(b + 64 * c), dot, 0, 0, 0);
        dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(down[c], *reinterpret_cast<const i32x4*>(b + D + 64 * c), dot, 0, 0, 0);
      }
      const float scale = p.bound_scales[at];
      uint32_t best = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r) best = max(best, order_of(static_cast<float>(dot[r]) * scale * step[r]));
      best = max(best, static_cast<uint32_t>(__shfl_xor(static_cast<int>(best), 16, 64)));
      best = max(best, static_cast<uint32_t>(__shfl_xor(static_cast<int>(best), 32, 64)));
      if (bad) best = 0;      // (the keys of such a block are masked)
      if (b0 + l16 < p.first || b0 + l16 >= blocks - p.last) best = kAlways;
      uint32_t* out = p.order + (static_cast<int64_t>(s) * p.Hkv + kh) * p.stride + b0 + l16;
      if (q4 == 0 && b0 + l16 < blocks) *out = g0 == 0 ? best : max(best, *out);
      if (p.err && bad && kh == 0 && g0 == 0 && q4 == 0 && b0 + l16 < blocks) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
    }
  }
}

// ------------------------------------------------------------ selection
// One workgroup per (sequence, KV head): the budget-th largest of its scores, found eight
// bits at a time from the histogram of those that share the bits above, then all larger
// scores and the first of the equal ones, in order.  Integer counts: the same in every run.
template <int kWide>
__global__ __launch_bounds__(kWide) void select_kernel(SelectParams p) {
  constexpr int kWaves = kWide / 64;
  __shared__ uint32_t hist[256];
  __shared__ uint32_t found[2];       // the digit, and how many are still wanted of those with it
  __shared__ uint32_t sums[2][kWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int kh = blockIdx.x, s = blockIdx.y;
  const int full = p.lengths[s], len = min(max(full, 0), p.max_length), blocks = (len + kPage - 1) / kPage;
  if (p.err && kh == 0 && t == 0 && full != len) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_LENGTH));
  int32_t* out = p.blocks + (static_cast<int64_t>(s) * p.Hkv + kh) * p.budget;
  if (blocks <= p.budget) {
    for (int i = t; i < p.budget; i += kWide) out[i] = i < blocks ? i : -1;
    return;
  }
  const uint32_t* in = p.order + (static_cast<int64_t>(s) * p.Hkv + kh) * p.stride;
  uint32_t prefix = 0, want = p.budget;      // bits known of the score that is looked for; its rank among those that share them
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = t; i < 256; i += kWide) hist[i] = 0;
    __syncthreads();
    for (int i = t; i < blocks; i += kWide) {
      const uint32_t x = in[i];
      if (shift == 24 || (x >> (shift + 8)) == prefix) atomicAdd(&hist[(x >> shift) & 255], 1u);
    }
    __syncthreads();
    if (wave == 0) {
      // Lane l: digits 255 - 4 l .. 252 - 4 l, from the top.
      uint32_t n[4], sum = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += n[e] = hist[255 - 4 * lane - e];
      uint32_t above = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(above, o, 64);
        if (lane >= o) above += v;
      }
      above -= sum;
      if (above < want && above + sum >= want) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (above < want && above + n[e] >= want) {
            found[0] = 255 - 4 * lane - e;
            found[1] = want - above;
          }
          above += n[e];
        }
      }
    }
    __syncthreads();
    prefix = prefix << 8 | found[0];
    want = found[1];
    __syncthreads();
  }
  // In order: everything above `prefix`, and the first `want` of those equal to it.
  uint32_t larger = 0, equal = 0;      // before this round
  for (int i0 = 0; i0 < blocks; i0 += kWide) {
    const uint32_t x = i0 + t < blocks ? in[i0 + t] : 0;
    const bool in_range = i0 + t < blocks, more = in_range && x > prefix, same = in_range && x == prefix;
    const uint64_t mb = __builtin_amdgcn_ballot_w64(more), sb = __builtin_amdgcn_ballot_w64(same);
    if (lane == 0) sums[0][wave] = __builtin_popcountll(mb), sums[1][wave] = __builtin_popcountll(sb);
    __syncthreads();
    uint32_t m = larger, e = equal;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) m += sums[0][w], e += sums[1][w];
      larger += sums[0][w], equal += sums[1][w];
    }
    const uint64_t below = (uint64_t(1) << lane) - 1;
    m += __builtin_popcountll(mb & below), e += __builtin_popcountll(sb & below);
    if (more || (same && e < want)) out[m + min(e, want)] = i0 + t;
    __syncthreads();
  }
}

template <int D>
hipError_t launch_score(const SelectParams& p, hipStream_t s) {
  const int most = (p.max_length + kPage - 1) / kPage;
  const int64_t runs = (most + kRun - 1) / kRun;
  const int per_wave = static_cast<int>(std::min<int64_t>(std::max<int64_t>(runs * p.Hkv * p.seqs / 4096, 1), 8));
  const int64_t units = (runs + per_wave - 1) / per_wave * p.Hkv;
  score_kernel<D><<<dim3(static_cast<unsigned>((units + 3) / 4), p.seqs), kThreads, 0, s>>>(p, per_wave);
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
  const int most = (p.max_length + kPage - 1) / kPage;
  if (most > p.budget) {
    if (hipError_t e = p.d == 128 ? launch_score<128>(p, s) : p.d == 64 ? launch_score<64>(p, s) : hipErrorInvalidValue; e != hipSuccess)
      return e;
  }
  const dim3 grid(p.Hkv, p.seqs);
  if (most > 2048) select_kernel<1024><<<grid, 1024, 0, s>>>(p);
  else select_kernel<256><<<grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace pallas
