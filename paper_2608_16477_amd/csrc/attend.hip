// Attention of one new token per sequence over a paged KV cache (bf16, E4M3 or
// INT8 rows).
//
// Calls that fill the chip live off the K/V stream, so the stream is what is divided: the 32-key
// blocks of all sequences, one behind the other, are cut into ranges of equal length
// (attend_blocks), as many as waves are resident at once (attend_ranges), and a wave
// takes a range of one KV head and up to 16 query heads that share it.  Its loads go on
// where one sequence ends and the next begins; each sequence is an online softmax in
// registers, and no wave waits for another.  What a wave has of a sequence that lies in
// its range as a whole is the result, anything else a record, which a second launch
// joins in order.  Ranges follow from the lengths alone and nothing is counted or
// accumulated across waves, so results are the same in every run.
//   us of a call, against a workgroup per KV head and split of a sequence, of a length
// that followed from the sequence's own (the first form): 64 sequences of 500 to 8000
// keys, E4M3, 64 / 8 heads of 128 (344 MB), 87 -> 69; 131,071 keys INT8 (277 MB) 65 -> 57; 60,001
// and 33,333 keys bf16, 32 / 8 heads (383 MB), 79 -> 68; 8 sequences of 1000 to 8000 keys
// bf16 (106 MB) 32 -> 27.  The first launch of these four reads what it has to and no more, at
// 5.6, 5.6, 6.4 and 5.0 TB/s; the join takes 4 to 5.  The long bf16 call is bound by the stream
// (a kernel that only reads such a buffer reaches 6.1); 8-bit rows are held back by what a
// block costs beside it as well: vector instructions take 0.36 (E4M3) and 0.54 (INT8) of the
// issue slots, bf16 0.13, and the matrix pipes are busy for 0.16, bf16 0.09.  LDS has no bank
// conflict.  Calls that do not fill the chip are a chain of loads, which the way to a range is
// longer than: they keep a workgroup per split (attend_split_kernel).
//
// Each wave moves its blocks from memory straight into a private two-stage LDS ring,
// with the rows' scales.  Scores are S^T = K Q^T with v_mfma_f32_16x16x32_bf16 (the
// query heads are the columns): lane l holds keys 4 (l / 16) + r of head l mod 16.
// O^T = V^T P^T takes those registers as its B operand as they are, with V read
// transposed from LDS.  8-bit codes are turned into bf16, which holds them exactly,
// between LDS and the MFMAs; a row's scale multiplies the score of its key (K) or its
// weight (V), in float32.  Weights stay 32-bit: they go into the MFMA as three bf16 parts
// whose sum they are.  (Two parts, 2^-17 off, us: 1 row of 500 keys bf16 7.3 (7.6), 128 of 300
// E4M3 21.8 (22.4), 64 of 500 to 8000 68.8 (69.3), 60,001 and 33,333 bf16 67.8 (68.2).)
#include "common.h"
#include "kernels.h"
#include "paged_attn.h"

namespace pallas {

namespace {

constexpr int kPage = 16;
constexpr int kBlk = 32;                 // keys per block: two pages
constexpr int kStages = 2;               // blocks in flight per wave
constexpr int kWaves = 4;                // per workgroup, each on its own
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
  static constexpr int kRing = kStages * kSlots;                 // of a wave
  // attend_ranges counts on the waves that a CU's 160 KiB of LDS hold.
  static_assert(160 * 1024 / (4 * kRing * 16) * 4 >= attend_waves(kRow), "resident waves");
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

// What a wave works with: where the blocks that it takes are, what each lane loads and
// reads of a block, and the softmax of the sequence that it is in.  (kOf: a type for each
// kernel.  Of kernels that share one, the compiler's host pass emits the stub of the first
// alone.)
template <int D, CacheType T, int kOf>
struct Wave {
  using S = Shape<D, T>;
  static constexpr int CH = S::kCh, DT = D / 16;
  const char* k;          // layer planes, at this KV head
  const char* v;
  uint32_t rs;            // bytes between tokens of a page
  int kh;
  int page, keys;         // lane 2 i + h: page of half h of block i, and the keys in it (0: none, or no page of the pool)
  uint32_t koff[S::kPerPage], voff[2 * S::kPerPage];   // byte offset in a page of what this lane loads in an instruction
  uint32_t kb0, vb0;      // where this lane reads: a K block at (row l16, chunk q4), a V block transposed
  u32x4* ring;
  u32x4 qf[D / 32];
  u32x4 qn[D / 32];       // of the sequence that comes next
  f32x4 acc[DT];          // lane: dimensions 16 dt + 4 q4 .. + 3 of head l16
  float m, lsum;          // (lsum: of this lane's keys)

  __device__ __forceinline__ void init(const AttendParams& p, int head, u32x4* at) {
    const int lane = threadIdx.x & 63, q4 = lane >> 4, l16 = lane & 15;
    kh = head;
    rs = static_cast<uint32_t>(p.Hkv) * S::kRow;
    k = static_cast<const char*>(p.k) + int64_t(kh) * S::kRow;
    v = static_cast<const char*>(p.v) + int64_t(kh) * S::kRow;
    ring = at;
#pragma unroll
    for (int n = 0; n < S::kPerPage; ++n) {
      const int r = n * S::kRowsPerLoad + lane / CH, c = lane % CH;
      koff[n] = r * rs + static_cast<uint32_t>((c ^ k_slot<T, CH>(r)) * 16);
      voff[n] = r * rs + static_cast<uint32_t>((c ^ v_slot<T, CH>(r)) * 16);
      voff[S::kPerPage + n] = r * rs + static_cast<uint32_t>((c ^ v_slot<T, CH>(kPage + r)) * 16);
    }
    kb0 = static_cast<uint32_t>(l16 * CH + (q4 ^ k_slot<T, CH>(l16)));
    if constexpr (T == kCacheBf16) {
      const int key = 4 * q4 + (l16 >> 2);
      vb0 = static_cast<uint32_t>(key * D * 2 + ((v_slot<T, CH>(key) | ((l16 & 3) >> 1)) * 16) + (l16 & 1) * 8);
    } else {
      const int key = (l16 >> 3) * kPage + 4 * q4 + ((l16 >> 1) & 3);
      vb0 = static_cast<uint32_t>(key * D + v_slot<T, CH>(key) * 16 + (l16 & 1) * 8);
    }
  }

  // Q: the MFMA's B operand, column l16 = head h0 + l16 of nh (the last one again where
  // there are fewer).  Its dimensions follow what a lane reads of K: bf16, chunk 4 kk + q4;
  // 8 bits, half kk % 2 of chunk 4 (kk / 2) + q4.
  __device__ __forceinline__ void load_q(const AttendParams& p, int s, int h0, int nh, u32x4* to) const {
    const int lane = threadIdx.x & 63, q4 = lane >> 4, l16 = lane & 15;
    const uint16_t* q = p.q + s * p.q_stride + int64_t(h0 + min(l16, nh - 1)) * D;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk)
      to[kk] = *reinterpret_cast<const u32x4*>(q + (T == kCacheBf16 ? 32 * kk + 8 * q4 : 64 * (kk / 2) + 16 * q4 + 8 * (kk % 2)));
  }
  // Waited for once, where this stands, and not inside the stream.
  __device__ __forceinline__ void await_q() {
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) asm volatile("" : "+v"(qf[kk]));
  }

  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x4{};
    m = -INFINITY;
    lsum = 0.f;
  }

  // Loads of block `i` into a stage: rows that exist; everything else reads zeros, as do
  // blocks that are not `in`.  Every step issues its loads, so that those in flight can be
  // counted.
  __device__ __forceinline__ void issue(const AttendParams& p, int i, bool in, int stage) const {
    u32x4* const st = ring + stage * S::kSlots;
    int pg[2], nv[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      pg[h] = __builtin_amdgcn_readlane(page, (i * 2 + h) & 63);
      nv[h] = in ? __builtin_amdgcn_readlane(keys, (i * 2 + h) & 63) : 0;
      const uint32_t range = nv[h] > 0 ? static_cast<uint32_t>(nv[h] - 1) * rs + S::kRow : 0;
      const int64_t base = nv[h] > 0 ? pg[h] * (int64_t(kPage) * rs) : 0;
      const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void*)(k + base), 0, range, kRsrcFlags);
      const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void*)(v + base), 0, range, kRsrcFlags);
#pragma unroll
      for (int n = 0; n < S::kPerPage; ++n)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void*)(st + (h * S::kPerPage + n) * 64), 16, koff[n], 0, 0, kAuxStream);
#pragma unroll
      for (int n = 0; n < S::kPerPage; ++n)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void*)(st + kBlk * CH + (h * S::kPerPage + n) * 64), 16,
                                                 voff[h * S::kPerPage + n], 0, 0, kAuxStream);
    }
    if constexpr (T != kCacheBf16) {
      // Lane l: the K (below 32) or V scale of key l % 32.
      const int lane = threadIdx.x & 63, key = lane % kPage;
      const bool second = lane & kPage;
      const uint32_t pgl = second ? pg[1] : pg[0];
      const uint32_t row = ((lane < 32 ? pgl : pgl + p.num_pages) * kPage + key) * p.Hkv + kh;
      const bool live = key < (second ? nv[1] : nv[0]);
      const __amdgpu_buffer_rsrc_t scales = __builtin_amdgcn_make_buffer_rsrc(
          (void*)p.scales, 0, static_cast<uint32_t>(p.num_pages) * (2 * kPage * 4) * p.Hkv, kRsrcFlags);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(scales, (lds_void*)(st + 2 * kBlk * CH), 4, live ? row * 4 : kOutside, 0, 0, 0);
    }
  }

  // The oldest of the kStages blocks whose loads were issued is here.
  __device__ __forceinline__ void await_block() const {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kStages - 1) * S::kLoads) : "memory");
  }

  // Blocks [i, stop), i below it, block n in stage n % kStages, the loads of the next kStages
  // - 1 in flight; `blocks`: all that the wave takes.  Block i is here, and block `stop` at
  // the end: what the wave stores and loads between two calls is behind the ring's loads, and
  // a wait at the head of a block would empty the ring to get past it.
  __device__ __forceinline__ void stream(const AttendParams& p, int& i, int stop, int blocks) {
    const int lane = threadIdx.x & 63, q4 = lane >> 4;
#pragma unroll 1
    do {
      const int stage = static_cast<int>(static_cast<unsigned>(i) % kStages);
      const u32x4* const Kst = ring + stage * S::kSlots;
      const u32x4* const Vst = Kst + kBlk * CH;
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
      const int nv0 = __builtin_amdgcn_readlane(keys, i * 2), nv1 = __builtin_amdgcn_readlane(keys, i * 2 + 1);
      if (nv0 < kPage || nv1 < kPage) {
        // Keys past the end, and keys on a page outside the pool.
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (4 * q4 + e >= (h ? nv1 : nv0)) pr[h * 4 + e] = -INFINITY;
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
      bf16x8 pb[3];
#pragma unroll
      for (int part = 0; part < 3; ++part) {
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
          for (int part = 2; part >= 0; --part)
            acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va[dt]), pb[part], acc[dt], 0, 0, 0);
      } else {
        u32x2 vc[DT];
#pragma unroll
        for (int dt = 0; dt < DT; dt += 4) read_pv8(vst, dt, vc + dt);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const bf16x8 a = codes_bf16<T>(vc[dt].x, vc[dt].y);
#pragma unroll
          for (int part = 2; part >= 0; --part) acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[part], acc[dt], 0, 0, 0);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this block's LDS reads are done
      issue(p, i + kStages, i + kStages < blocks, stage);
      await_block();
    } while (++i < stop);
  }
};

// Lengths of 64 sequences from `at` on, one per lane, in 32-key blocks (0 behind the last).
__device__ __forceinline__ int lane_length(const AttendParams& p, int at) {
  const int s = at + static_cast<int>(threadIdx.x & 63);
  const int len = row_length(p, min(s, p.seqs - 1));
  return s < p.seqs ? len : 0;
}
__device__ __forceinline__ int blocks_of(int len) { return static_cast<int>((static_cast<uint32_t>(len) + kBlk - 1) / kBlk); }

// Inclusive prefix sums over the wave (row shifts by 1, 2, 4, 8, then the rows' last
// lanes to the rows behind).
__device__ __forceinline__ int wave_prefix(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // row_bcast:31 into rows 2 and 3
  return v;
}

template <int D, CacheType T>
__global__ __launch_bounds__(kBoundThreads) void attend_kernel(AttendParams p, int groups, int head_shift) {
  using S = Shape<D, T>;
  constexpr int DT = D / 16;
  // One array: with several, the compiler's alias scopes make LDS reads of a
  // stage wait for the loads in flight into the other.
  __shared__ __attribute__((aligned(256))) u32x4 lds[kWaves * S::kRing];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q4 = lane >> 4, l16 = lane & 15;
  // A workgroup's waves take the same range of four heads (of two or one where the heads
  // are not a multiple), whose rows are neighbours in memory and share scale lines and table
  // entries; workgroups of one blockIdx.x, the range's other heads, go to one XCD.  (64
  // sequences E4M3, first launch: 62 us; 65 to 72 with four ranges of one head.)
  const int head = (static_cast<int>(blockIdx.y) << head_shift) + (wave & ((1 << head_shift) - 1));
  const int kh = groups == 1 ? head : head / groups, group = head - kh * groups;
  const int r0 = static_cast<int>(blockIdx.x) * (kWaves >> head_shift) + (wave >> head_shift);
  if (r0 >= p.ranges) return;
  // One sequence: the pages of this range, were it of one block (lanes 0, 1) or of two
  // (lanes 8 to 11), are read beside the length (a short call is a chain of loads).
  int ahead = 0;
  if (p.seqs == 1) ahead = p.bt[min(lane < 8 ? 2 * r0 + lane : 4 * r0 + lane - 8, p.max_pages - 1)];
  int win = 0, lens = lane_length(p, 0);        // lens: of sequences [win, win + 64)

  const int h0 = kh * p.G + group * kAttendGroup, nh = min(kAttendGroup, p.G - group * kAttendGroup);
  Wave<D, T, 0> w;
  w.init(p, kh, lds + wave * S::kRing);

  // All blocks of the call, and the ranges they make.  coarse: blocks of the first (lane +
  // 1) 64ths of the sequences.
  int before = wave_prefix(blocks_of(lens));    // blocks of the window's sequences, up to and with each
  int coarse = before;
  const int share = static_cast<int>(static_cast<uint32_t>(p.seqs + 63) / 64);
  if (share > 1) {
    int sum = 0;
#pragma unroll 8
    for (int n = 0; n < share; ++n) {
      const int q = lane * share + n, len = row_length(p, min(q, p.seqs - 1));
      sum += q < p.seqs ? blocks_of(len) : 0;
    }
    coarse = wave_prefix(sum);
  }
  const int total = __builtin_amdgcn_readlane(coarse, 63);
  const int each = attend_blocks(total, p.seqs, p.ranges);
  auto window = [&](int s) {                    // makes s one of the 64
    if (s >= win && s < win + 64) return;
    win = s & ~63;
    lens = lane_length(p, win);
    before = wave_prefix(blocks_of(lens));
  };
  auto length = [&](int s) {
    window(s);
    return __builtin_amdgcn_readlane(lens, s & 63);
  };
  int s = 0, base = 0;                          // a sequence, and the blocks before it
  // Moves them on to the sequence that block f (of the call's) is in.
  auto seek = [&](int f) {
    if (share > 1) {
      const uint64_t behind = __builtin_amdgcn_ballot_w64(coarse > f);
      const int n = behind != 0 ? __builtin_ctzll(behind) : 0;
      if (n * share > s) {
        s = n * share;
        base = __builtin_amdgcn_readlane(coarse, n - 1);
      }
    }
    while (s < p.seqs) {
      window(s);
      // blocks of the window before s
      const int skip = __builtin_amdgcn_readlane(before - blocks_of(lens), s & 63);
      const uint64_t behind = __builtin_amdgcn_ballot_w64(lane >= (s & 63) && base + before - skip > f);
      if (behind != 0) {
        const int first = __builtin_ctzll(behind);
        base += __builtin_amdgcn_readlane(before - blocks_of(lens), first) - skip;
        s = win + first;
        return;
      }
      base += __builtin_amdgcn_readlane(before, 63) - skip;
      s = win + 64;
    }
  };

  for (int r = r0; r * each < total; r += p.ranges) {
    const int f0 = r * each, f1 = min(f0 + each, total), blocks = f1 - f0;
    seek(f0);
    if (s >= p.seqs) break;                     // (lengths that changed since `total`)
    w.load_q(p, s, h0, nh, w.qf);
    // Pages of the range's blocks.
    w.page = w.keys = 0;
    const int f = f0 + lane / 2;
    int from = 0, key0 = -1;
    for (const int s0 = s, base0 = base;;) {
      const int len = length(s), nb = blocks_of(len);
      if (f >= base && f < base + nb && f < f1) {
        from = s;
        key0 = ((f - base) * 2 + lane % 2) * kPage;
        w.keys = min(max(len - key0, 0), kPage);
      }
      base += nb;
      ++s;
      // Rows without keys are jumped over (250 between two of 4000 keys bf16, 32 / 8 heads: 19
      // us, 42 one by one; 60,000 of them 510, 6270).
      if (base < f1 && s < p.seqs && length(s) == 0) seek(base);
      if (base < f1 && s < p.seqs) continue;
      s = s0;
      base = base0;
      break;
    }
    if (each == 2) ahead = __builtin_amdgcn_mov_dpp(ahead, 0x108, 0xF, 0xF, false);   // row_shl:8
    if (w.keys > 0) {
      w.page = p.seqs == 1 && each <= 2 ? ahead : p.bt[int64_t(from) * p.max_pages + key0 / kPage];
      if (w.page < 0 || w.page >= p.num_pages) {
        w.page = w.keys = 0;
        if (p.err && head == 0) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
      }
    }
#pragma unroll
    for (int i = 0; i < kStages; ++i) w.issue(p, i, i < blocks, i);
    w.await_q();
    w.await_block();
    w.begin();
    for (int i = 0;;) {
      const int cur = s, at = f0 + i - base, end = base + blocks_of(length(s));     // at: the sequence's block at i
      const int stop = min(blocks, end - f0);
      // The next sequence that has keys, and its query, are there when this one ends (us;
      // found and read after it, 1000 rows of 100 keys E4M3 57 (60), 200 of 700 bf16 34.1
      // (35.4), 8 of 1000 to 8000 26.8 (27.8); on equal long rows within 1%).
      bool more = false;
      if (stop < blocks) {
        seek(f0 + stop);
        more = s < p.seqs;
      }
      w.load_q(p, more ? s : cur, h0, nh, w.qn);
      w.stream(p, i, stop, blocks);
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) w.qf[kk] = w.qn[kk];
      w.await_q();
      const float l = rows_sum(w.lsum);
      const bool whole = at == 0 && end <= f1;
      if (l16 < nh) {
        if (whole) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) write_row(p, cur, h0 + l16, 16 * dt + 4 * q4, w.acc[dt], w.m, l);
        } else {
          // Ranges and sequences advance together, so r + s numbers the records.
          const int64_t rec = (int64_t(r) + cur) * p.Hq + h0 + l16;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(p.part_o + rec * D + 16 * dt + 4 * q4) = w.acc[dt];
          if (q4 == 0) *reinterpret_cast<f32x2*>(p.part_ml + rec * 2) = f32x2{w.m, l};
        }
      }
      if (at == 0 && head == 0 && lane == 0) {
        // The row's records: none, or from here to the range of its last block.
        reinterpret_cast<int2*>(p.parts)[cur] = int2{r, whole ? 0 : (end - 1) / each - r + 1};
      }
      if (!more) break;
      w.begin();
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load into LDS outlives its wave
}

// The same for calls of little work: a workgroup per split of `per` blocks of a sequence,
// KV head and group of query heads, whose waves take equal runs of its blocks and merge
// them through LDS.  A row of one split is written as it is (short rows: one launch).
template <int D, CacheType T, int kWaves>
__global__ __launch_bounds__(kBoundThreads) void attend_split_kernel(AttendParams p, int groups, int splits, int per) {
  using S = Shape<D, T>;
  constexpr int DT = D / 16;
  __shared__ __attribute__((aligned(256))) u32x4 lds[kWaves * S::kRing];
  const int lane = threadIdx.x & 63, q4 = lane >> 4, l16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Heads of a split on one XCD, where there are splits for all of them.
  const int heads = p.Hkv * groups, items = p.seqs * splits;
  int item, head;
  if (items < 8) {
    item = static_cast<int>(blockIdx.x) / heads;
    head = static_cast<int>(blockIdx.x) - item * heads;
  } else {
    const int y = static_cast<int>(blockIdx.x >> 3);
    item = y / heads * 8 + (blockIdx.x & 7);
    head = y % heads;
    if (item >= items) return;
  }
  const int s = item / splits, split = item - s * splits, f0 = split * per;
  const int kh = groups == 1 ? head : head / groups, group = head - kh * groups;
  const int h0 = kh * p.G + group * kAttendGroup, nh = min(kAttendGroup, p.G - group * kAttendGroup);
  // The split's pages (at most 64) beside the row's length.
  int page = p.bt[int64_t(s) * p.max_pages + min(2 * f0 + lane, p.max_pages - 1)];
  Wave<D, T, kWaves> w;
  w.load_q(p, s, h0, nh, w.qf);
  const int len = row_length(p, s);
  w.init(p, kh, lds + wave * S::kRing);
  const int blocks_all = blocks_of(len), all = min(max(blocks_all - f0, 0), per);
  if (split > 0 && all == 0) return;
  const int each = (all + kWaves - 1) / kWaves;
  const int b0 = min(wave * each, all), blocks = min(each, all - b0);
  const bool bad = page < 0 || page >= p.num_pages;
  const int key0 = (2 * f0 + lane) * kPage;
  if (p.err && wave == 0 && head == 0) {
    if (bad && key0 < len) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
    if (split == 0 && lane == 0 && len != p.lengths[s]) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_LENGTH));
  }
  // (Lane 2 i + h: of the wave's block i.)
  w.keys = __shfl(bad ? 0 : min(max(len - key0, 0), kPage), 2 * b0 + lane, 64);
  w.page = __shfl(page, 2 * b0 + lane, 64);
#pragma unroll
  for (int i = 0; i < kStages; ++i) w.issue(p, i, i < blocks, i);
  w.await_q();
  w.await_block();
  w.begin();
  int i = 0;
  if (blocks > 0) w.stream(p, i, blocks, blocks);
  // The waves' parts, each in its own ring once nothing is in flight there: [head][dim],
  // then (maximum, sum) per head.
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  const float l = rows_sum(w.lsum);
  if (l16 < nh) {
    float* dst = reinterpret_cast<float*>(w.ring) + l16 * D + 4 * q4;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(dst + dt * 16) = w.acc[dt];
    if (q4 == 0) reinterpret_cast<f32x2*>(w.ring + kAttendGroup * D / 4)[l16] = f32x2{w.m, l};
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  const bool whole = blocks_all <= per;
  if (splits > 1 && split == 0 && head == 0 && threadIdx.x == 0)      // records s * splits on (join_kernel adds s)
    reinterpret_cast<int2*>(p.parts)[s] = int2{s * splits - s, whole ? 0 : (blocks_all + per - 1) / per};
  for (int e = threadIdx.x; e < nh * D / 4; e += kWaves * 64) {
    const int g = e / (D / 4), d = (e % (D / 4)) * 4;
    f32x2 ml[kWaves];
    float top = -INFINITY, sum = 0.f;
    f32x4 o{};
#pragma unroll
    for (int n = 0; n < kWaves; ++n) {
      ml[n] = reinterpret_cast<const f32x2*>(lds + n * S::kRing + kAttendGroup * D / 4)[g];
      top = fmaxf(top, ml[n].x);
    }
#pragma unroll
    for (int n = 0; n < kWaves; ++n) {
      const float f = join_weight(ml[n].x, ml[n].y, top);
      sum += f * ml[n].y;
      o += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(lds + n * S::kRing) + g * D + d);
    }
    if (whole) {
      write_row(p, s, h0 + g, d, o, top, sum);
    } else {
      const int64_t rec = int64_t(item) * p.Hq + h0 + g;
      *reinterpret_cast<f32x4*>(p.part_o + rec * D + d) = o;
      if (d == 0) *reinterpret_cast<f32x2*>(p.part_ml + rec * 2) = f32x2{top, sum};
    }
  }
}

// Joins a row's records: one workgroup per (query head, sequence).  D / 4 lanes hold a
// record; a wave takes 256 / D records side by side and kJoinBatch of those in flight.
// The records of the only sequence of a call are read before their number is known.
// Rows without a key get their zeros here.
constexpr int kJoinBatch = 8;
template <int D, int kThreads>
__global__ __launch_bounds__(kThreads) void join_kernel(AttendParams p) {
  constexpr int kLanes = D / 4, kSide = kThreads / kLanes, kWaveSide = 64 / kLanes;
  constexpr int kShare = kJoinBatch * kWaveSide, kRound = kThreads / 64 * kShare;
  const int h = blockIdx.x, s = blockIdx.y, t = threadIdx.x;
  const int side = t / kLanes, i = (t % kLanes) * 4;
  const int mine = t / 64 * kShare + side % kWaveSide;      // this lane's first record of a round
  const int2 parts = reinterpret_cast<const int2*>(p.parts)[s];
  const int len = row_length(p, s);
  if (p.err && h == 0 && t == 0 && len != p.lengths[s]) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_LENGTH));
  const int first = p.seqs == 1 ? 0 : parts.x;
  f32x2 a[kJoinBatch];
  f32x4 v[kJoinBatch];
  auto read = [&](int k0) {
#pragma unroll
    for (int b = 0; b < kJoinBatch; ++b) {
      // (Within the records whatever is read, also where lengths change during a call.)
      const int64_t rec = min(max(first + s + k0 + b * kWaveSide + mine, 0), p.records - 1) * int64_t(p.Hq) + h;
      a[b] = reinterpret_cast<const f32x2*>(p.part_ml)[rec];
      v[b] = *reinterpret_cast<const f32x4*>(p.part_o + rec * D + i);
    }
  };
  if (p.seqs == 1 || (len > 0 && mine < parts.y)) read(0);
  if (len == 0) {
    if (t < kLanes) write_row(p, s, h, i, f32x4{}, -INFINITY, 0.f);
    return;
  }
  const int n = min(parts.y, p.records);
  if (n <= 0) return;
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
    if (k0 + mine >= n) break;
    read(k0);
  }
  // The sides, as a tree.
  __shared__ f32x2 mls[kSide];
  __shared__ f32x4 os[kSide][kLanes];
#pragma unroll
  for (int half = kSide / 2; half > 0; half /= 2) {
    if (side >= half && side < 2 * half) {
      os[side][t % kLanes] = o;
      mls[side] = f32x2{m, l};
    }
    __syncthreads();
    if (side < half) add(mls[side + half].x, mls[side + half].y, os[side + half][t % kLanes]);
  }
  if (side == 0) write_row(p, s, h, i, o, m, l);
}

// Waves per row of the join: as many as it can fill with records (at most `most`) in one go.
// Further waves have nothing to add and change no bit.
template <int D>
hipError_t launch_join(const AttendParams& p, int64_t most, hipStream_t s) {
  const dim3 joins(p.Hq, p.seqs);
  constexpr int kShare = kJoinBatch * 256 / D;
  if (most > 4 * kShare) join_kernel<D, 1024><<<joins, 1024, 0, s>>>(p);
  else if (most > kShare) join_kernel<D, 256><<<joins, 256, 0, s>>>(p);
  else join_kernel<D, 64><<<joins, 64, 0, s>>>(p);
  return hipGetLastError();
}

template <int D, CacheType T, int kWaves>
hipError_t launch_split(const AttendParams& p, int groups, int splits, int per, hipStream_t s) {
  const int64_t items = int64_t(p.seqs) * splits, all = items < 8 ? items : (items + 7) / 8 * 8;
  attend_split_kernel<D, T, kWaves><<<static_cast<unsigned>(all * p.Hkv * groups), kWaves * 64, 0, s>>>(p, groups, splits, per);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || splits == 1) return e;
  return launch_join<D>(p, splits, s);
}

// How a call is run (us on the GPU; 8 KV heads of 128).
//   Rows of up to kShortKeys keys, up to kShortGroups (sequence, head) pairs: a workgroup each
// and one launch.  Its waves' rings fill a CU's LDS, or half of it where there are several
// rows to a CU.  As ranges in parentheses: 4 rows of 60 keys bf16 4.7 (8.3), 128 of 300 E4M3
// 22.4 (25.9), bf16 31.9 (31.6), 128 of 500 bf16 50.4 (48.2), 180 of them 66.8 (70.1); beyond the
// limits, 1 of 1000 E4M3 11.7 (9.6), 256 of 300 40.3 (36.1).
//   Else splits of one or two blocks a wave, if those are at most a workgroup per CU: 1 row of
// 4000 keys bf16 10.5 (12.5), 16,000 E4M3 15.8 (18.7), 8 of 1000 INT8 10.4 (14.3).  Four blocks
// a wave gain nothing on equal rows and lose on others (27 of 30 to 2000 keys, 4 heads of
// 64, 11.7 (8.7)), as do two workgroups per CU (16,000 keys 19.3).
//   Else ranges.
//   The host knows max_length alone, so the bound that a call states chooses.  With room
// for 4096 and for 32,768 keys: 4 rows of 60 bf16 9.1, 9.0 (4.7 with 60), 1 of 500 8.4, 10.7 (7.6),
// 1 of 4000 10.5, 14.1; 8 of 1000 to 8000 and 64 E4M3 level.
constexpr int kShortKeys = 512;
constexpr int kShortGroups = 1536;
constexpr int kSplitBlocks = 2;

template <int D, CacheType T>
hipError_t launch(const AttendParams& p, hipStream_t s) {
  const int groups = (p.G + kAttendGroup - 1) / kAttendGroup, heads = p.Hkv * groups;
  constexpr int kFill = std::min(attend_waves(Shape<D, T>::kRow), 8);     // waves whose rings fill a CU's LDS
  const int64_t rows = int64_t(p.seqs) * heads;
  const int most = static_cast<int>(attend_total(1, p.max_length));       // blocks of a row
  if (p.max_length <= kShortKeys && rows <= kShortGroups)
    return rows <= 256 ? launch_split<D, T, kFill>(p, groups, 1, most, s) : launch_split<D, T, kFill / 2>(p, groups, 1, most, s);
  for (int each = 1; each <= kSplitBlocks; each *= 2) {
    // (Records, seqs * splits <= 256 / heads: fewer than attend_ranges, so there is room.)
    const int per = kFill * each, splits = (most + per - 1) / per;
    if (rows * splits <= 256) return launch_split<D, T, kFill>(p, groups, splits, per, s);
  }
  const int head_shift = heads % 4 == 0 ? 2 : heads % 2 == 0 ? 1 : 0;
  const int per = kWaves >> head_shift;         // ranges of a workgroup
  attend_kernel<D, T><<<dim3((p.ranges + per - 1) / per, heads >> head_shift), kWaves * 64, 0, s>>>(p, groups, head_shift);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  return launch_join<D>(p, p.ranges / p.seqs < kJoinBatch * 256 / D ? 0 : attend_row_records(most, p.seqs, p.ranges), s);
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
