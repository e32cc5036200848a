// Attention of one new token per sequence over a paged KV cache (bf16, E4M3 or
// INT8): a row's keys are cut into splits, each a softmax of its own with a running
// maximum and sum, and joined by a second launch where a row can have several.
#include "common.h"
#include "kernels.h"

namespace pallas {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kPage = 16;

// Two neighbouring elements of a cached row.
template <CacheType T>
__device__ __forceinline__ f32x2 pair_at(const void* plane, int64_t e) {
  if constexpr (T == kCacheBf16) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(plane) + e);
    return f32x2{bflo(w), bfhi(w)};
  } else {
    const uint32_t w = *reinterpret_cast<const uint16_t*>(static_cast<const uint8_t*>(plane) + e);
    if constexpr (T == kCacheE4m3) return __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
    return f32x2{static_cast<float>(static_cast<int8_t>(w)), static_cast<float>(static_cast<int8_t>(w >> 8))};
  }
}

__device__ __forceinline__ int row_length(const AttendParams& p, int s) { return min(max(p.lengths[s], 0), p.max_length); }

__device__ __forceinline__ void write_row(const AttendParams& p, int s, int h, int i, float o, float m, float l) {
  p.out[s * p.out_stride + int64_t(h) * p.d + i] = f2bf(l > 0.f ? o / l : l);
  if (i == 0 && p.lse) p.lse[int64_t(s) * p.Hq + h] = l == 0.f ? -INFINITY : (m + __log2f(l)) * 0.693147180559945309f;
}

// One workgroup per (split, query head, sequence): a wave takes every fourth key, a
// lane D / 32 elements of it (half the lanes when D is 64).
template <int D, CacheType T>
__global__ __launch_bounds__(kThreads) void attend_kernel(AttendParams p, int rows) {
  const int split = blockIdx.x, h = blockIdx.y, s = blockIdx.z;
  const int len = row_length(p, s), per = attend_split_keys(len, rows);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (split == 0 && h == 0 && threadIdx.x == 0 && len != p.lengths[s] && p.err)
    atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_LENGTH));
  if (split > 0 && split * int64_t(per) >= len) return;
  const int j0 = split * per, j1 = min(len, j0 + per);
  const bool mine = lane < D / 2;
  f32x2 q{0.f, 0.f}, acc{0.f, 0.f};
  if (mine) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(p.q + s * p.q_stride + int64_t(h) * D + 2 * lane);
    q = f32x2{bflo(w), bfhi(w)};
  }
  const int kh = h / (p.Hq / p.Hkv);
  float m = -INFINITY, l = 0.f;
  for (int j = j0 + wave; j < j1; j += kWaves) {
    const int pg = p.bt[int64_t(s) * p.max_pages + j / kPage];
    if (pg < 0 || pg >= p.num_pages) {
      if (lane == 0 && p.err) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
      continue;
    }
    const int64_t row = (int64_t(pg) * kPage + j % kPage) * p.Hkv + kh;
    const f32x2 k = mine ? pair_at<T>(p.k, row * D + 2 * lane) : f32x2{0.f, 0.f};
    const f32x2 v = mine ? pair_at<T>(p.v, row * D + 2 * lane) : f32x2{0.f, 0.f};
    const float ks = T == kCacheBf16 ? 1.f : p.k_scale[row], vs = T == kCacheBf16 ? 1.f : p.v_scale[row];
    const float z = wave_sum(q.x * k.x + q.y * k.y) * ks * p.scale_log2;
    const float top = fmaxf(m, z);
    const float keep = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top);
    const float w = z == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(z - top);   // (NaN: stays)
    m = top;
    l = l * keep + w;
    acc.x = acc.x * keep + w * vs * v.x;
    acc.y = acc.y * keep + w * vs * v.y;
  }
  __shared__ float om[kWaves][D], ml[kWaves][2];
  if (mine) {
    om[wave][2 * lane] = acc.x;
    om[wave][2 * lane + 1] = acc.y;
  }
  if (lane == 0) {
    ml[wave][0] = m;
    ml[wave][1] = l;
  }
  __syncthreads();
  if (threadIdx.x >= D) return;
  float top = ml[0][0];
  for (int w = 1; w < kWaves; ++w) top = fmaxf(top, ml[w][0]);
  float o = 0.f, sum = 0.f;
  for (int w = 0; w < kWaves; ++w) {
    const float f = ml[w][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[w][0] - top);
    o += f * om[w][threadIdx.x];
    sum += f * ml[w][1];
  }
  if (len <= per) {
    write_row(p, s, h, threadIdx.x, o, top, sum);
  } else {
    const int64_t rec = (int64_t(s) * p.Hq + h) * p.splits + split;
    p.part_o[rec * D + threadIdx.x] = o;
    if (threadIdx.x < 2) p.part_ml[rec * 2 + threadIdx.x] = threadIdx.x ? sum : top;
  }
}

// Joins a row's splits: one workgroup per (query head, sequence).
__global__ void join_kernel(AttendParams p, int rows) {
  const int h = blockIdx.x, s = blockIdx.y, i = threadIdx.x;
  const int len = row_length(p, s), per = attend_split_keys(len, rows);
  if (len <= per) return;
  const int n = (len + per - 1) / per;
  const int64_t rec = (int64_t(s) * p.Hq + h) * p.splits;
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int k = 0; k < n; ++k) {
    const float mk = p.part_ml[(rec + k) * 2], lk = p.part_ml[(rec + k) * 2 + 1];
    const float top = fmaxf(m, mk);
    const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    const float w = mk == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mk - top);
    o = o * keep + w * p.part_o[(rec + k) * p.d + i];
    l = l * keep + w * lk;
    m = top;
  }
  write_row(p, s, h, i, o, m, l);
}

template <int D>
hipError_t launch(const AttendParams& p, CacheType type, int rows, hipStream_t s) {
  const dim3 grid(p.splits, p.Hq, p.seqs);
  if (type == kCacheBf16) attend_kernel<D, kCacheBf16><<<grid, kThreads, 0, s>>>(p, rows);
  else if (type == kCacheE4m3) attend_kernel<D, kCacheE4m3><<<grid, kThreads, 0, s>>>(p, rows);
  else attend_kernel<D, kCacheInt8><<<grid, kThreads, 0, s>>>(p, rows);
  if (p.splits > 1) join_kernel<<<dim3(p.Hq, p.seqs), D, 0, s>>>(p, rows);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(const AttendParams& p, CacheType type, hipStream_t s) {
  const int rows = static_cast<int>(attend_rows(p.seqs, p.Hq, p.Hkv));
  if (p.d == 128) return launch<128>(p, type, rows, s);
  if (p.d == 64) return launch<64>(p, type, rows, s);
  return hipErrorInvalidValue;
}

}  // namespace pallas
