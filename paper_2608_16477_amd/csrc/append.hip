// New tokens' K and V into a paged cache, K and the queries rotated on the way.
//
// Pair i of a Q or K head turns by pos * f_i (the plan's 64-bit fixed-point turns; whole turns
// drop out exactly), V is copied or quantised as it is.  One launch reads each row once and
// writes it where it belongs: 4 d bytes a Q head, and a K or V head's 2 d and its cached row.
//
// What is stored in 8 or 4 bits is decided at borders between codes: a K value rounded to bf16
// one way or the other, which float32 sums of two products do in one of some thousand values,
// can be a whole code away.  So the rotation is in 64 bits (v_fma_f64 has float32's rate here)
// and rounded to float32 and then to bf16: codes do not depend on how it was computed, but
// for values within position 2^-61 + 2^-48 (the plan's turns; the polynomials), times the
// pair's magnitudes, of a border.
//
// Long calls are bound by memory: 3000 tokens of 64 / 8 heads of 128 to a bf16 cache (123 MB) 22.5 us, 5.5
// TB/s; 12,000 of them 93.  1999 tokens of 20 / 4 heads to INT8 (27 MB) 9.4, with the launch and a
// chain of position, table and row before them; calls of a few tokens are that chain, 3.2 (8 tokens) to 3.7 us
// (64, E2M1).  Rotary of Q, of K and the store one after the other read and write K once more, in three
// launches: 64 tokens 7.6, 1999 12.8.  (3000 to bf16: the two rotations alone 26.4.)
#include "common.h"
#include "kernels.h"
#include "quant_rows.h"

namespace pallas {

namespace {

constexpr int kThreads = 256;   // at most
constexpr int kPage = 16;
constexpr int kBf16 = 0;        // a cache of bf16 rows, beside the pallas_quant_formats
// bf16 rows of this many bytes are stored non-temporally (3000 tokens of 72 heads: 23 us, 33 with
// plain stores); fewer stay in the caches for what reads them next.
constexpr int64_t kNtStoreBytes = int64_t(4) << 20;

// (cos, sin) of an angle of `a` 2^-64 turns, times m.  What is left of a quarter, |x| <= pi / 4,
// goes through Taylor's polynomials; the first terms left out are below 2^-53 (sine, x^17 / 17!)
// and 2^-49 (cosine, x^16 / 16!).
__device__ __forceinline__ void turn_cos_sin64(uint64_t a, double m, double& c, double& s) {
  const uint64_t quarter = (a + (uint64_t(1) << 61)) >> 62;
  const double x = static_cast<double>(static_cast<int64_t>(a - (quarter << 62))) * 0x1.921fb54442d18p-62;   // 2 pi 2^-64
  const double z = x * x;
  double sp = __builtin_fma(z, -7.6471637318198165e-13, 1.6059043836821613e-10);   // 1 / 15!, 1 / 13!, ..
  sp = __builtin_fma(z, sp, -2.5052108385441720e-08);
  sp = __builtin_fma(z, sp, 2.7557319223985893e-06);
  sp = __builtin_fma(z, sp, -1.9841269841269841e-04);
  sp = __builtin_fma(z, sp, 8.3333333333333333e-03);
  sp = __builtin_fma(z, sp, -1.6666666666666667e-01);
  sp = __builtin_fma(z * x, sp, x);
  double cp = __builtin_fma(z, -1.1470745597729725e-11, 2.0876756987868099e-09);   // 1 / 14!, 1 / 12!, ..
  cp = __builtin_fma(z, cp, -2.7557319223985891e-07);
  cp = __builtin_fma(z, cp, 2.4801587301587302e-05);
  cp = __builtin_fma(z, cp, -1.3888888888888889e-03);
  cp = __builtin_fma(z, cp, 4.1666666666666667e-02);
  cp = __builtin_fma(z, cp, -0.5);
  cp = __builtin_fma(z, cp, 1.0);
  const bool odd = quarter & 1;
  c = (odd ? sp : cp) * ((quarter + 1) & 2 ? -m : m);
  s = (odd ? cp : sp) * (quarter & 2 ? -m : m);
}

// The elements of a head that a lane takes are four pairs (in the half layout two runs of
// four) of turned elements, or eight neighbours behind them.  kFast: runs of four are
// aligned to 8 bytes, which needs rotary_dim to be a multiple of 8.
struct Place {
  int lo[4], hi[4];
};
template <bool kFast>
__device__ __forceinline__ Place place_of(const AppendParams& p, int j) {
  Place at;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int u = 4 * j + e;
    const bool half = !p.interleaved && 2 * (kFast ? 4 * j : u) < p.r;
    if constexpr (kFast) {
      at.lo[e] = half ? u : 8 * j + e;
      at.hi[e] = half ? u + p.r / 2 : 8 * j + 4 + e;
    } else {
      at.lo[e] = half ? u : 2 * u;
      at.hi[e] = half ? u + p.r / 2 : 2 * u + 1;
    }
  }
  return at;
}
template <bool kFast>
__device__ __forceinline__ void read_pairs(const uint16_t* x, const Place& at, uint32_t (&w)[4]) {
  if constexpr (kFast) {
    const u32x2 a = *reinterpret_cast<const u32x2*>(x + at.lo[0]), b = *reinterpret_cast<const u32x2*>(x + at.hi[0]);
    w[0] = a.x, w[1] = a.y, w[2] = b.x, w[3] = b.y;
  } else {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      w[e] = x[at.lo[2 * e]] | static_cast<uint32_t>(x[at.lo[2 * e + 1]]) << 16;
      w[2 + e] = x[at.hi[2 * e]] | static_cast<uint32_t>(x[at.hi[2 * e + 1]]) << 16;
    }
  }
}
template <bool kNt, class V>
__device__ __forceinline__ void put(V v, void* at) {
  if constexpr (kNt) __builtin_nontemporal_store(v, static_cast<V*>(at));
  else *static_cast<V*>(at) = v;
}
template <bool kFast, bool kNt>
__device__ __forceinline__ void write_pairs(uint16_t* y, const Place& at, const uint32_t (&w)[4]) {
  if constexpr (kFast) {
    put<kNt>(u32x2{w[0], w[1]}, y + at.lo[0]);
    put<kNt>(u32x2{w[2], w[3]}, y + at.hi[0]);
  } else {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      y[at.lo[2 * e]] = static_cast<uint16_t>(w[e]), y[at.lo[2 * e + 1]] = static_cast<uint16_t>(w[e] >> 16);
      y[at.hi[2 * e]] = static_cast<uint16_t>(w[2 + e]), y[at.hi[2 * e + 1]] = static_cast<uint16_t>(w[2 + e] >> 16);
    }
  }
}

// D / 8 lanes take a head; `slots` heads of a token go side by side (several tokens where a
// token has fewer), in the order Q, K, V.  The workgroup works out the angles of its tokens once,
// each a thread's, while the first loads are on their way.  (Three heads of a lane in flight
// together, as in rope.hip, cost the chip's waves their registers: 12,000 tokens of 80 heads 99 us, 93;
// 4000 of 48 21, 18.)
template <int D, int kFormat, bool kFast, bool kNt>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendParams p, int slots, int tokens_per, int heads_per) {
  constexpr int kLanes = D / 8, kMost = kThreads / kLanes;
  struct Turn {
    double c, s;
  };
  __shared__ __attribute__((aligned(16))) Turn turns[kMost / 2 * (D / 2)];      // (at least two heads a token)
  __shared__ __attribute__((aligned(16))) uint16_t turned[kFormat == kBf16 ? 8 : kThreads * 8];   // a head's place: its lanes' 16 bytes
  const int j = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
  const int heads = p.Hq + 2 * p.Hkv;
  const int t0 = blockIdx.x * tokens_per, mine = tokens_per > 1 ? slot / heads : 0, t = t0 + mine;
  int h = tokens_per > 1 ? slot % heads : slot + blockIdx.y * heads_per;
  int h1 = tokens_per > 1 ? heads : min(heads, static_cast<int>(blockIdx.y + 1) * heads_per);
  if (slot >= (tokens_per > 1 ? tokens_per * heads : slots) || t >= p.tokens) h1 = h;      // (nothing, but the angles)
  const int pos = p.pos[min(t, p.tokens - 1)];
  if (pos < 0) h1 = h;      // padding
  const Place at = place_of<kFast>(p, j);
  uint32_t w[4];
  auto read = [&] {
    if (h >= p.Hq + p.Hkv) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(p.v + t * p.v_stride + (h - p.Hq - p.Hkv) * D + j * 8);
      w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    } else {
      read_pairs<kFast>(h < p.Hq ? p.q + t * p.q_stride + h * D : p.k + t * p.k_stride + (h - p.Hq) * D, at, w);
    }
  };
  if (h < h1) read();
  int64_t row = -1;         // the token's first K row in its page slot, among the rows of both planes
  if (h < h1) {
    const int seq = p.seq ? p.seq[t] : t;
    int pg = -1;
    if (seq >= 0 && seq < p.seqs && pos / kPage < p.max_pages) pg = p.bt[static_cast<int64_t>(seq) * p.max_pages + pos / kPage];
    if (pg >= 0 && pg < p.num_pages) row = (static_cast<int64_t>(pg) * kPage + pos % kPage) * p.Hkv;
  }
  const int pairs = p.r / 2;
  for (int i = threadIdx.x; i < tokens_per * pairs; i += blockDim.x) {
    const int of = tokens_per > 1 ? i / pairs : 0, u = i - of * pairs;
    const int64_t at_pos = tokens_per > 1 ? p.pos[min(t0 + of, p.tokens - 1)] : pos;
    turn_cos_sin64(static_cast<uint64_t>(at_pos) * p.turns[u], p.magnitude, turns[of * (D / 2) + u].c, turns[of * (D / 2) + u].s);
  }
  __syncthreads();
  if (h >= h1) return;
  double c[4], s[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int u = 4 * j + e;
    const Turn n = turns[mine * (D / 2) + min(u, pairs - 1)];
    c[e] = n.c, s[e] = n.s;
  }
  for (;;) {
    const bool q = h < p.Hq, v = h >= p.Hq + p.Hkv;
    const int hh = q ? h : v ? h - p.Hq - p.Hkv : h - p.Hq;
    if (!q && row < 0) {      // (K and V rows are the last of a token)
      if (p.err && j == 0) atomicOr(p.err, static_cast<int32_t>(PALLAS_DEVERR_PAGE));
      return;
    }
    if (!v) {
      // w: first elements of the pairs, then second ones (fast, neighbours: pairs 0, 1 and 2, 3)
      const bool beside = kFast && (p.interleaved || 8 * j >= p.r);
      float y[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t wa = beside ? w[e] : w[e / 2] >> (16 * (e % 2)), wb = beside ? w[e] >> 16 : w[2 + e / 2] >> (16 * (e % 2));
        const double x0 = bflo(wa), x1 = bflo(wb);
        y[e] = static_cast<float>(__builtin_fma(x0, c[e], -(x1 * s[e])));
        y[4 + e] = static_cast<float>(__builtin_fma(x1, c[e], x0 * s[e]));
      }
      uint32_t n[4];
      if (beside) {
#pragma unroll
        for (int e = 0; e < 4; ++e) n[e] = pack_bf2(y[e], y[4 + e]);
      } else {
        n[0] = pack_bf2(y[0], y[1]), n[1] = pack_bf2(y[2], y[3]), n[2] = pack_bf2(y[4], y[5]), n[3] = pack_bf2(y[6], y[7]);
      }
      // (Elements behind the turned ones are copied, whatever their bits.)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (kFast) {
          w[e] = 8 * j < p.r ? n[e] : w[e];
        } else {
          const int u = 4 * j + 2 * (e % 2);      // pairs u and u + 1 in the halves of this word
          w[e] = (2 * u < p.r ? n[e] & 0xFFFFu : w[e] & 0xFFFFu) | (2 * u + 2 < p.r ? n[e] & 0xFFFF0000u : w[e] & 0xFFFF0000u);
        }
      }
    }
    const int64_t to = row + hh + (v ? static_cast<int64_t>(p.num_pages) * kPage * p.Hkv : 0);
    if (q) {
      write_pairs<kFast, kNt>(p.q_out + t * p.q_out_stride + hh * D, at, w);
    } else if constexpr (kFormat == kBf16) {
      uint16_t* y = static_cast<uint16_t*>(p.cache) + to * D;
      if (v) put<kNt>(u32x4{w[0], w[1], w[2], w[3]}, y + j * 8);
      else write_pairs<kFast, kNt>(y, at, w);
    } else {
      if (!v) {
        // Into the row's order, through LDS (a row's lanes are of one wave).
        uint16_t* y = turned + threadIdx.x / kLanes * D;
        write_pairs<kFast, false>(y, at, w);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const u32x4 x = *reinterpret_cast<const u32x4*>(y + j * 8);
        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
      const RowCodes<8> codes = quantise_row<kFormat, D, 8>(w);
      uint8_t* cache = static_cast<uint8_t*>(p.cache);
      if constexpr (kFormat == PALLAS_QUANT_E2M1) {
        constexpr int kGroup = D / 32;      // lanes of a quarter
        *reinterpret_cast<uint32_t*>(cache + to * (D / 2) + j * 4) = codes.codes[0];
        if (j % kGroup == 0) reinterpret_cast<uint8_t*>(p.scales)[to * 4 + j / kGroup] = static_cast<uint8_t>(codes.scale);
      } else {
        *reinterpret_cast<u32x2*>(cache + to * D + j * 8) = u32x2{codes.codes[0], codes.codes[1]};
        if (j == 0) p.scales[to] = __uint_as_float(codes.scale);
      }
    }
    h += slots;
    if (h >= h1) return;
    read();
  }
}

template <int D, int kFormat>
void launch(const AppendParams& p, hipStream_t s) {
  constexpr int kMost = kThreads / (D / 8);
  const int heads = p.Hq + 2 * p.Hkv;
  // Workgroups as wide as a token's heads fill evenly.
  const int tokens_per = std::max(kMost / heads, 1), passes = (heads + kMost - 1) / kMost;
  const int slots = tokens_per > 1 ? tokens_per * heads : (heads + passes - 1) / passes;
  // Few tokens: a token's heads over several workgroups.
  const int heads_per = p.tokens < 512 ? slots : heads;
  const dim3 grid((p.tokens + tokens_per - 1) / tokens_per, tokens_per > 1 ? 1 : (heads + heads_per - 1) / heads_per);
  const int threads = (D / 8 * slots + 63) / 64 * 64;
  if (p.r % 8 != 0) append_kernel<D, kFormat, false, false><<<grid, threads, 0, s>>>(p, slots, tokens_per, heads_per);
  else if (int64_t(p.tokens) * (p.Hq + p.Hkv) * D * 2 >= kNtStoreBytes) append_kernel<D, kFormat, true, true><<<grid, threads, 0, s>>>(p, slots, tokens_per, heads_per);
  else append_kernel<D, kFormat, true, false><<<grid, threads, 0, s>>>(p, slots, tokens_per, heads_per);
}

template <int D>
void launch(const AppendParams& p, hipStream_t s) {
  if (p.format == kBf16) launch<D, kBf16>(p, s);
  else for_format(p.format, [&](auto f) { launch<D, f.value>(p, s); });
}

}  // namespace

hipError_t launch_append(const AppendParams& p, hipStream_t s) {
  if (p.tokens == 0) return hipSuccess;
  if (p.d == 128) launch<128>(p, s);
  else if (p.d == 64) launch<64>(p, s);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pallas
