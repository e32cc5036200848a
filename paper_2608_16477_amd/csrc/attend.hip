// Attention of one new token per sequence over a paged KV cache (bf16, E4M3 or
// INT8 rows).
//
// A row's keys are cut into splits of a length that its own length and the call's
// size give (attend_split_keys); a workgroup takes one split of one (sequence, KV head)
// and up to 16 query heads that share it.  Its waves take equal runs of the split's
// 32-key blocks, each an online softmax of its own; they are merged through LDS, and
// the splits of a row, where it has several, by a second launch.  Every order is
// fixed, nothing is counted or accumulated across workgroups.
//
// The kernel is bound by the K/V stream.  Each wave moves its own blocks from memory
// straight into a private two-stage LDS ring, with the rows' scales.  Scores are
// S^T = K Q^T with v_mfma_f32_16x16x32_bf16 (the query heads are the columns): lane l
// holds keys 4 (l / 16) + r of head l mod 16.  O^T = V^T P^T takes those registers as
// its B operand as they are, with V read transposed from LDS.  8-bit codes are turned
// into bf16, which holds them exactly, between LDS and the MFMAs; a row's scale
// multiplies the score of its key (K) or its weight (V), in float32.  Weights go into
// the MFMA as two bf16 parts, 2^-17 of their value off: below what the sums lose.
#include "common.h"
#include "kernels.h"
#include "paged_attn.h"

namespace pallas {

namespace {

constexpr int kPage = 16;
constexpr int kBlk = 32;                 // keys per block: two pages
constexpr int kStages = 2;               // blocks in flight per wave
constexpr int kBoundThreads = 512;       // (256 registers a wave, no accumulation registers)
constexpr int kAuxStream = 2;            // nt: K and V are read once
constexpr uint32_t kRsrcFlags = 0x00020000;
constexpr uint32_t kOutside = 0xFFFFFFF0u;   // a buffer offset past any range: reads zero

template <int D, CacheType T>
struct Shape {
  static constexpr int kElem = T == kCacheBf16 ? 2 : 1;
  static constexpr int kRow = D * kElem;              // bytes of a head row
  static constexpr int kCh = kRow / 16;               // 16-byte chunks of it
  static constexpr int kRowsPerLoad = 64 / kCh;       // rows per load instruction
  static constexpr int kPerPage = kPage / kRowsPerLoad;
  static constexpr int kScaleSlots = T == kCacheBf16 ? 0 : 16;   // 32 K scales, 32 V scales
  static constexpr int kSlots = 2 * kBlk * kCh + kScaleSlots;    // 16-byte slots of a stage
  static constexpr int kLoads = 4 * kPerPage + (T == kCacheBf16 ? 0 : 1);   // instructions per block
  // bf16 rows of 128: two waves, so that two workgroups (128 KiB of ring) share a CU.
  static constexpr int kWaves = kRow == 256 ? 2 : 4;
  static constexpr int kRing = kWaves * kStages * kSlots;
  static constexpr int kOut = kWaves * kAttendGroup * D / 4;     // the waves' outputs, over the ring
};

// Chunk swizzles of 8-bit rows of CH chunks (8 rows of 128 bytes, or 16 of 64, fill the
// banks four times): as the bf16 ones, the 16 rows of a K read at one chunk, and the 16
// rows x 16 bytes of half a transposed V read (rows 8 i + 0 .. 7 of both pages), fall on
// 16 distinct 4-bank groups.
template <int CH>
__device__ __forceinline__ int swz8_k(int row) { return CH == 8 ? (row >> 1) & 7 : (row >> 2) & 3; }
template <int CH>
__device__ __forceinline__ int swz8_v(int row) {
  return CH == 8 ? ((row >> 1) & 3) | ((row >> 2) & 4) : ((row >> 2) & 1) | ((row >> 3) & 2);
}
template <CacheType T, int CH>
__device__ __forceinline__ int k_slot(int row) {
  if constexpr (T == kCacheBf16) return swz_k<CH>(row);
  else return swz8_k<CH>(row);
}
template <CacheType T, int CH>
__device__ __forceinline__ int v_slot(int row) {
  if constexpr (T == kCacheBf16) return swz_v<CH>(row);
  else return swz8_v<CH>(row);
}

// 8 codes as bf16.
template <CacheType T>
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t a, uint32_t b) {
  u32x4 w;
  if constexpr (T == kCacheE4m3) {
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true));
  } else {
    auto f = [](uint32_t x, int i) { return static_cast<float>(static_cast<int8_t>(x >> (8 * i))); };
    w[0] = pack_bf2(f(a, 0), f(a, 1));
    w[1] = pack_bf2(f(a, 2), f(a, 3));
    w[2] = pack_bf2(f(b, 0), f(b, 1));
    w[3] = pack_bf2(f(b, 2), f(b, 3));
  }
  return __builtin_bit_cast(bf16x8, w);
}

// Four output tiles of the PV operand from a block of 8-bit V rows.  In each 16-lane
// group, ds_read_b64_tr_b8 hands lane i byte i % 8 of the 64-bit words read by lanes
// i / 8, i / 8 + 2, .. i / 8 + 14: with lanes 2 r and 2 r + 1 at the halves of a 16-byte
// chunk of row r, eight rows of one dimension.  `vb` is the lane's address at tile 0;
// tiles are chunks, XOR 16 each.  (One statement with its wait: see read_pv4.)
__device__ __forceinline__ void read_pv8(uint32_t vb, int dt0, u32x2* a) {
  const uint32_t x0 = vb ^ ((dt0 + 0) * 16u), x1 = vb ^ ((dt0 + 1) * 16u);
  const uint32_t x2 = vb ^ ((dt0 + 2) * 16u), x3 = vb ^ ((dt0 + 3) * 16u);
  u32x2 r0, r1, r2, r3;
  asm volatile(
      "ds_read_b64_tr_b8 %0, %4\n\t"
      "ds_read_b64_tr_b8 %1, %5\n\t"
      "ds_read_b64_tr_b8 %2, %6\n\t"
      "ds_read_b64_tr_b8 %3, %7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r0), "=&v"(r1), "=&v"(r2), "=&v"(r3)
      : "v"(x0), "v"(x1), "v"(x2), "v"(x3)
      : "memory");
  a[0] = r0, a[1] = r1, a[2] = r2, a[3] = r3;
}

__device__ __forceinline__ int row_length(const AttendParams& p, int s) { return min(max(p.lengths[s], 0), p.max_length); }

// Four outputs of a row, of weight sum l (0: no key; NaN stays), and at the first its
// log-sum-exp.
__device__ __forceinline__ void write_row(const AttendParams& p, int s, int h, int i, f32x4 o, float m, float l) {
  const float inv = l > 0.f ? 1.f / l : l;
  u32x2 w;
  w.x = pack_bf2(o[0] * inv, o[1] * inv);
  w.y = pack_bf2(o[2] * inv, o[3] * inv);
  *reinterpret_cast<u32x2*>(p.out + s * p.out_stride + int64_t(h) * p.d + i) = w;
  if (i == 0 && p.lse) p.lse[int64_t(s) * p.Hq + h] = l == 0.f ? -INFINITY : (m + __log2f(l)) * 0.693147180559945309f;
}

// Weight, beside the maximum `top`, of a sum l of exponentials relative to m.  A part
// without keys (m -infinity, l 0) has none; one of nothing but NaN keeps its NaN.
__device__ __forceinline__ float join_weight(float m, float l, float top) {
  return m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - top);
}

// What a wave needs to load blocks of its split.
struct Source {
  const char* k;        // layer planes, at this KV head
  const char* v;
  uint32_t rs;          // bytes between tokens of a page
  int64_t page_bytes;
  int keys;             // keys of the split
  int entry;            // lane: page of the split, or -1
};

// Loads of block `blk` of the split into a stage: rows that exist, on pages of the
// pool; everything else reads zeros.  Every wave issues the loads of every step, so
// that those in flight can be counted.
template <int D, CacheType T>
__device__ __forceinline__ void issue_block(const AttendParams& p, const Source& src, __amdgpu_buffer_rsrc_t scales, int kh,
                                            int blk, bool in, const uint32_t* koff, const uint32_t* voff, u32x4* st) {
  using S = Shape<D, T>;
  int pg[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    pg[h] = in ? __builtin_amdgcn_readlane(src.entry, blk * 2 + h) : -1;
    const int nv = min(kPage, src.keys - (blk * kBlk + h * kPage));
    const uint32_t range = pg[h] >= 0 && nv > 0 ? static_cast<uint32_t>(nv - 1) * src.rs + S::kRow : 0;
    const int64_t base = max(pg[h], 0) * src.page_bytes;
    const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void*)(src.k + base), 0, range, kRsrcFlags);
    const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void*)(src.v + base), 0, range, kRsrcFlags);
#pragma unroll
    for (int v = 0; v < S::kPerPage; ++v)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void*)(st + (h * S::kPerPage + v) * 64), 16, koff[v], 0, 0, kAuxStream);
#pragma unroll
    for (int v = 0; v < S::kPerPage; ++v)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void*)(st + kBlk * S::kCh + (h * S::kPerPage + v) * 64), 16,
                                               voff[h * S::kPerPage + v], 0, 0, kAuxStream);
  }
  if constexpr (T != kCacheBf16) {
    // Lane l: the K (below 32) or V scale of key l % 32.
    const int lane = threadIdx.x & 63, key = lane & 31;
    const int page = key < kPage ? pg[0] : pg[1];
    const uint32_t row = (static_cast<uint32_t>(lane < 32 ? page : page + p.num_pages) * kPage + key % kPage) * p.Hkv + kh;
    const bool live = page >= 0 && blk * kBlk + key < src.keys;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(scales, (lds_void*)(st + 2 * kBlk * S::kCh), 4, live ? row * 4 : kOutside, 0, 0, 0);
  }
}

template <int D, CacheType T>
__global__ __launch_bounds__(kBoundThreads) void attend_kernel(AttendParams p, int rows, int items, int groups) {
  using S = Shape<D, T>;
  constexpr int CH = S::kCh, kWaves = S::kWaves, kThreads = kWaves * 64;
  constexpr int DT = D / 16;
  // One array: with several, the compiler's alias scopes make LDS reads of a
  // stage wait for the loads in flight into the other.
  __shared__ __attribute__((aligned(256))) u32x4 lds[(S::kRing > S::kOut ? S::kRing : S::kOut) + kWaves * kAttendGroup / 2];
  f32x2(*wave_ml)[kAttendGroup] = reinterpret_cast<f32x2(*)[kAttendGroup]>(lds + (S::kRing > S::kOut ? S::kRing : S::kOut));

  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int q4 = lane >> 4, l16 = lane & 15;
  // Workgroups b, b + 8, .. go to one XCD and share an L2: there the heads of one
  // (split, sequence) follow each other, which share its table entries and the lines of
  // its scales.  The splits of a sequence go round the XCDs, which otherwise end up with
  // unequal sequences: few sequences split by split, others a split of all of them at a
  // time, each time turned so that a sequence moves on by one XCD; the last splits, which
  // only long sequences have, first.
  const int heads = p.Hkv * groups;
  const int y = static_cast<int>(blockIdx.x) >> 3;
  const int item = y / heads * 8 + (blockIdx.x & 7);
  if (item >= items) return;
  int split, s;
  if (p.seqs < 8) {
    s = item / p.splits;
    split = item - s * p.splits;
  } else {
    const int turn = item / p.seqs;
    s = (item - turn * p.seqs + static_cast<int>(int64_t(turn) * ((p.seqs - 1) & 7) % p.seqs)) % p.seqs;
    split = p.splits - 1 - turn;
  }
  const int kh = (y % heads) / groups, group = (y % heads) % groups;
  const int G = p.Hq / p.Hkv;
  const int h0 = kh * G + group * kAttendGroup, nh = min(kAttendGroup, G - group * kAttendGroup);
  // The split's table entries, one per lane.  Those of a split of the least length are
  // read while the row's length is on its way: a short call is a chain of loads.
  const int32_t* bt = p.bt + int64_t(s) * p.max_pages;
  const int first = split * (kAttendMinSplit / kPage) + lane;
  int entry = lane < kAttendMinSplit / kPage && first < p.max_pages ? bt[first] : -1;
  const int len = row_length(p, s), per = attend_split_keys(len, rows);
  if (split > 0 && int64_t(split) * per >= len) return;
  const int j0 = split * per;

  Source src;
  src.keys = min(len - j0, per);
  src.rs = static_cast<uint32_t>(p.Hkv) * S::kRow;
  src.page_bytes = int64_t(kPage) * src.rs;
  src.k = static_cast<const char*>(p.k) + int64_t(kh) * S::kRow;
  src.v = static_cast<const char*>(p.v) + int64_t(kh) * S::kRow;
  {
    const bool page = lane * kPage < src.keys;
    if (per != kAttendMinSplit && page) entry = bt[j0 / kPage + lane];
    src.entry = page && entry >= 0 && entry < p.num_pages ? entry : -1;
    if (p.err && wave == 0 && kh == 0 && group == 0) {
      if (page && src.entry < 0) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
      if (split == 0 && lane == 0 && len != p.lengths[s]) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_LENGTH));
    }
  }
  // Q: the MFMA's B operand, column l16 = a head (repeated where there are fewer).  Its
  // dimensions follow what a lane reads of K: bf16, chunk 4 kk + q4; 8 bits, half kk % 2
  // of chunk 4 (kk / 2) + q4.
  u32x4 qf[D / 32];
  {
    const uint16_t* q = p.q + s * p.q_stride + int64_t(h0 + l16 % nh) * D;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk)
      qf[kk] = *reinterpret_cast<const u32x4*>(q + (T == kCacheBf16 ? 32 * kk + 8 * q4 : 64 * (kk / 2) + 16 * q4 + 8 * (kk % 2)));
  }
  // Loaded, and waited for, before the K/V stream (loads return in order).
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) asm volatile("" : "+v"(qf[kk]));
  asm volatile("" : "+v"(src.entry));

  const int blocks = (src.keys + kBlk - 1) / kBlk, each = (blocks + kWaves - 1) / kWaves;
  const int blk0 = wave * each, blk1 = min(blk0 + each, blocks);
  u32x4* const ring = lds + wave * kStages * S::kSlots;
  __amdgpu_buffer_rsrc_t scales = __builtin_amdgcn_make_buffer_rsrc(
      (void*)p.scales, 0, static_cast<uint32_t>(p.num_pages) * (2 * kPage * 4) * p.Hkv, kRsrcFlags);
  // Byte offset in a page of what this lane loads in instruction v of it.
  uint32_t koff[S::kPerPage], voff[2 * S::kPerPage];
#pragma unroll
  for (int v = 0; v < S::kPerPage; ++v) {
    const int r = v * S::kRowsPerLoad + lane / CH, c = lane % CH;
    koff[v] = r * src.rs + static_cast<uint32_t>((c ^ k_slot<T, CH>(r)) * 16);
    voff[v] = r * src.rs + static_cast<uint32_t>((c ^ v_slot<T, CH>(r)) * 16);
    voff[S::kPerPage + v] = r * src.rs + static_cast<uint32_t>((c ^ v_slot<T, CH>(kPage + r)) * 16);
  }
#pragma unroll
  for (int i = 0; i < kStages; ++i)
    issue_block<D, T>(p, src, scales, kh, blk0 + i, blk0 + i < blk1, koff, voff, ring + i * S::kSlots);

  // Where this lane reads: a K block at (row l16, chunk q4), a V block transposed.
  const uint32_t kb0 = static_cast<uint32_t>(l16 * CH + (q4 ^ k_slot<T, CH>(l16)));
  uint32_t vb0;
  if constexpr (T == kCacheBf16) {
    const int key = 4 * q4 + (l16 >> 2);
    vb0 = static_cast<uint32_t>(key * D * 2 + ((v_slot<T, CH>(key) | ((l16 & 3) >> 1)) * 16) + (l16 & 1) * 8);
  } else {
    const int key = (l16 >> 3) * kPage + 4 * q4 + ((l16 >> 1) & 3);
    vb0 = static_cast<uint32_t>(key * D + v_slot<T, CH>(key) * 16 + (l16 & 1) * 8);
  }

  f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x4{};
  float m = -INFINITY, lsum = 0.f;
#pragma unroll 1
  for (int blk = blk0; blk < blk1; ++blk) {
    u32x4* const Kst = ring + (static_cast<unsigned>(blk - blk0) % kStages) * S::kSlots;
    u32x4* const Vst = Kst + kBlk * CH;
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kStages - 1) * S::kLoads) : "memory");   // this block is here
    f32x4 sc[2] = {f32x4{}, f32x4{}};
    if constexpr (T == kCacheBf16) {
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8 a = __builtin_bit_cast(bf16x8, Kst[(kb0 ^ (kk * 4u)) + h * (kPage * CH)]);
          sc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, qf[kk]), sc[h], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x4 a = Kst[(kb0 ^ (j * 4u)) + h * (kPage * CH)];
          sc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_bf16<T>(a.x, a.y), __builtin_bit_cast(bf16x8, qf[2 * j]), sc[h], 0, 0, 0);
          sc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_bf16<T>(a.z, a.w), __builtin_bit_cast(bf16x8, qf[2 * j + 1]), sc[h], 0, 0, 0);
        }
    }
    float pr[8], vs[8];
    if constexpr (T == kCacheBf16) {
#pragma unroll
      for (int e = 0; e < 8; ++e) pr[e] = sc[e / 4][e % 4] * p.scale_log2;
    } else {
      const f32x4* f = reinterpret_cast<const f32x4*>(Kst + 2 * kBlk * CH);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 ks = f[4 * h + q4], w = f[8 + 4 * h + q4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          pr[4 * h + r] = sc[h][r] * (ks[r] * p.scale_log2);
          vs[4 * h + r] = w[r];
        }
      }
    }
    const int pg0 = __builtin_amdgcn_readlane(src.entry, blk * 2), pg1 = __builtin_amdgcn_readlane(src.entry, blk * 2 + 1);
    if (src.keys - blk * kBlk < kBlk || pg0 < 0 || pg1 < 0) {
      // Keys past the end, and keys on a page outside the pool.
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (blk * kBlk + h * kPage + 4 * q4 + r >= src.keys || (h ? pg1 : pg0) < 0) pr[h * 4 + r] = -INFINITY;
    }
    float mx = fmaxf(fmaxf(fmaxf(pr[0], pr[1]), fmaxf(pr[2], pr[3])), fmaxf(fmaxf(pr[4], pr[5]), fmaxf(pr[6], pr[7])));
    mx = rows_max(mx);
    if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
      const float m_new = fmaxf(m, mx);
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      lsum *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] *= alpha;
    }
    const float mc = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      pr[e] = __builtin_amdgcn_exp2f(pr[e] - mc);
      lsum += pr[e];
      if constexpr (T != kCacheBf16) pr[e] *= vs[e];
    }
    bf16x8 pb[2];
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = take_bf2(pr[2 * e], pr[2 * e + 1]);
      pb[part] = __builtin_bit_cast(bf16x8, w);
    }
    const uint32_t vst = vb0 + static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)Vst));
    if constexpr (T == kCacheBf16) {
      u32x4 va[DT];
#pragma unroll
      for (int dt = 0; dt < DT; dt += 4) read_pv4<kPage * D * 2>(vst, dt, va + dt);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int part = 1; part >= 0; --part)
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va[dt]), pb[part], acc[dt], 0, 0, 0);
    } else {
      u32x2 vc[DT];
#pragma unroll
      for (int dt = 0; dt < DT; dt += 4) read_pv8(vst, dt, vc + dt);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x8 a = codes_bf16<T>(vc[dt].x, vc[dt].y);
#pragma unroll
        for (int part = 1; part >= 0; --part) acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[part], acc[dt], 0, 0, 0);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this block's LDS reads are done
    issue_block<D, T>(p, src, scales, kh, blk + kStages, blk + kStages < blk1, koff, voff, Kst);
  }

  // Merge the waves through LDS (the ring is free once all are here and nothing is in
  // flight): om[wave][head][dim].
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  float* om = reinterpret_cast<float*>(lds);
  lsum = rows_sum(lsum);
  if (l16 < nh) {
    float* dst = om + (wave * kAttendGroup + l16) * D + 4 * q4;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(dst + dt * 16) = acc[dt];
    if (q4 == 0) wave_ml[wave][l16] = f32x2{m, lsum};
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  for (int e = t; e < nh * D / 4; e += kThreads) {
    const int g = e / (D / 4), i = (e % (D / 4)) * 4;
    f32x2 ml[kWaves];
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      ml[w] = wave_ml[w][g];
      top = fmaxf(top, ml[w].x);
    }
    float l = 0.f;
    f32x4 o{};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = join_weight(ml[w].x, ml[w].y, top);
      l += f * ml[w].y;
      o += f * *reinterpret_cast<const f32x4*>(om + (w * kAttendGroup + g) * D + i);
    }
    if (len <= per) {
      write_row(p, s, h0 + g, i, o, top, l);
    } else {
      const int64_t rec = (int64_t(s) * p.Hq + h0 + g) * p.splits + split;
      *reinterpret_cast<f32x4*>(p.part_o + rec * D + i) = o;
      if (i == 0) *reinterpret_cast<f32x2*>(p.part_ml + rec * 2) = f32x2{top, l};
    }
  }
}

// Joins a row's splits: one workgroup per (query head, sequence) that has several.
// D / 4 lanes hold a record; a wave takes 256 / D records side by side and kJoinBatch of
// those in flight.  The first are read before the row's length is known (any record of
// the call may be read; those that the row does not have are left out), so a row whose
// splits fit a wave's share costs one trip to memory.  A call whose rows all fit has one
// wave per workgroup, others four; the further waves find no record of a row that fits,
// and adding nothing changes no bit, so a row's result does not depend on which it is.
constexpr int kJoinBatch = 8;
template <int D, int kThreads>
__global__ __launch_bounds__(kThreads) void join_kernel(AttendParams p, int rows) {
  constexpr int kLanes = D / 4, kSide = kThreads / kLanes, kWaveSide = 64 / kLanes;
  constexpr int kShare = kJoinBatch * kWaveSide, kRound = kThreads / 64 * kShare;
  const int h = blockIdx.x, s = blockIdx.y, t = threadIdx.x;
  const int side = t / kLanes, i = (t % kLanes) * 4;
  const int mine = t / 64 * kShare + side % kWaveSide;      // this lane's first record of a round
  const int64_t rec = (int64_t(s) * p.Hq + h) * p.splits;
  const f32x2* ml = reinterpret_cast<const f32x2*>(p.part_ml) + rec;
  const float* po = p.part_o + rec * D + i;
  f32x2 a[kJoinBatch];
  f32x4 v[kJoinBatch];
  auto read = [&](int k0) {
#pragma unroll
    for (int b = 0; b < kJoinBatch; ++b) {
      const int k = min(k0 + b * kWaveSide + mine, p.splits - 1);
      a[b] = ml[k];
      v[b] = *reinterpret_cast<const f32x4*>(po + int64_t(k) * D);
    }
  };
  read(0);
#pragma unroll
  for (int b = 0; b < kJoinBatch; ++b) asm volatile("" : "+v"(a[b]), "+v"(v[b]));
  const int len = row_length(p, s), per = attend_split_keys(len, rows);
  if (len <= per) return;
  const int n = static_cast<int>((int64_t(len) + per - 1) / per);
  float m = -INFINITY, l = 0.f;
  f32x4 o{};
  auto add = [&](float mk, float lk, f32x4 ok) {
    const float top = fmaxf(m, mk);
    const float keep = join_weight(m, l, top), w = join_weight(mk, lk, top);
    l = keep * l + w * lk;
    o = keep * o + w * ok;
    m = top;
  };
  for (int k0 = 0;;) {
#pragma unroll
    for (int b = 0; b < kJoinBatch; ++b)
      if (k0 + b * kWaveSide + mine < n) add(a[b].x, a[b].y, v[b]);
    k0 += kRound;
    if (k0 >= n) break;
    read(k0);
  }
  __shared__ f32x2 mls[kSide];
  __shared__ f32x4 os[kSide][kLanes];
  os[side][t % kLanes] = o;
  if (t % kLanes == 0) mls[side] = f32x2{m, l};
  __syncthreads();
  if (t >= kLanes) return;
#pragma unroll
  for (int k = 1; k < kSide; ++k) add(mls[k].x, mls[k].y, os[k][t]);
  write_row(p, s, h, i, o, m, l);
}

template <int D, CacheType T>
hipError_t launch(const AttendParams& p, hipStream_t s) {
  const int groups = (p.Hq / p.Hkv + kAttendGroup - 1) / kAttendGroup;
  const int rows = static_cast<int>(attend_rows(p.seqs, p.Hq, p.Hkv));
  const int items = p.splits * p.seqs;
  const int64_t grid = (int64_t(items) + 7) / 8 * 8 * p.Hkv * groups;
  attend_kernel<D, T><<<static_cast<unsigned>(grid), Shape<D, T>::kWaves * 64, 0, s>>>(p, rows, items, groups);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const dim3 joins(p.Hq, p.seqs);
  if (p.splits > kJoinBatch * 256 / D) join_kernel<D, 256><<<joins, 256, 0, s>>>(p, rows);
  else if (p.splits > 1) join_kernel<D, 64><<<joins, 64, 0, s>>>(p, rows);
  return hipGetLastError();
}

template <int D>
hipError_t launch(const AttendParams& p, CacheType type, hipStream_t s) {
  if (type == kCacheBf16) return launch<D, kCacheBf16>(p, s);
  if (type == kCacheE4m3) return launch<D, kCacheE4m3>(p, s);
  return launch<D, kCacheInt8>(p, s);
}

}  // namespace

hipError_t launch_attend(const AttendParams& p, CacheType type, hipStream_t s) {
  if (p.d == 128) return launch<128>(p, type, s);
  if (p.d == 64) return launch<64>(p, type, s);
  return hipErrorInvalidValue;
}

}  // namespace pallas
