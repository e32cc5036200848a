// Device helpers that the two attention kernels for single tokens share
// (attention_decode.hip, attend.hip): LDS layouts of cached bf16 rows, transposed
// reads, reductions over the rows of a wave.
#pragma once

#include "common.h"

namespace pallas {

typedef __attribute__((address_space(3))) void lds_void;

// LDS rows are whole head rows of CH 16-byte chunks; chunk c of row r sits in
// slot c ^ swz(r).  K: the 16 rows an MFMA operand read covers at one chunk
// land on 16 distinct 4-bank groups.  V: the 8 keys x 2 chunks that half of a
// transposed read covers do.
template <int CH>
__device__ __forceinline__ int swz_k(int row) { return CH == 16 ? row & 15 : (row >> 1) & 7; }
template <int CH>
__device__ __forceinline__ int swz_v(int row) { return CH == 16 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); }

// Four output tiles of the PV operand from a V block at LDS byte address
// `vb`: keys 4 q4 .. + 3 of its first page (at the tile's address, vb XOR 32
// per tile) and of its second (`kSecond` bytes further).  In each 16-lane
// group, ds_read_b64_tr_b16 hands lane i element i % 4 of the 64-bit words
// read by lanes i / 4, i / 4 + 4, i / 4 + 8 and i / 4 + 12: four consecutive
// keys of one dimension.  Reads and their wait are one statement: before the
// builtin form of this read the compiler waits for every load in flight into
// LDS, which would empty the ring at each block.
template <int kSecond>
__device__ __forceinline__ void read_pv4(uint32_t vb, int dt0, u32x4* a) {
  const uint32_t x0 = vb ^ ((dt0 + 0) * 32u), x1 = vb ^ ((dt0 + 1) * 32u);
  const uint32_t x2 = vb ^ ((dt0 + 2) * 32u), x3 = vb ^ ((dt0 + 3) * 32u);
  u32x2 l0, l1, l2, l3, h0, h1, h2, h3;
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %4, %10\n\t"
      "ds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %11\n\t"
      "ds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(l0), "=&v"(h0), "=&v"(l1), "=&v"(h1), "=&v"(l2), "=&v"(h2), "=&v"(l3), "=&v"(h3)
      : "v"(x0), "v"(x1), "v"(x2), "v"(x3), "n"(kSecond)
      : "memory");
  a[0] = u32x4{l0.x, l0.y, h0.x, h0.y};
  a[1] = u32x4{l1.x, l1.y, h1.x, h1.y};
  a[2] = u32x4{l2.x, l2.y, h2.x, h2.y};
  a[3] = u32x4{l3.x, l3.y, h3.x, h3.y};
}

// Max / sum over the four 16-lane rows of a wave (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float rows_max(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float rows_sum(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// (a, b) as packed bf16, and what is left of them.
__device__ __forceinline__ uint32_t take_bf2(float& a, float& b) {
  const uint32_t w = pack_bf2(a, b);
  a -= bflo(w);
  b -= bfhi(w);
  return w;
}

}  // namespace pallas
