// C ABI of the cache operators (rotary positions, the 8- and 4-bit cache, attention of one
// new token): argument checks and launches.  Every check runs before anything is
// enqueued.
#include <algorithm>
#include <cmath>

#include "api.h"
#include "kernels.h"
#include "pallas.h"
#include "profile.h"

using pallas::fail;

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int launched(hipError_t e, const char* where) { return e == hipSuccess ? PALLAS_OK : pallas::hip_fail(e, where); }

int check_quant_pool(const pallas_quant_pool* p, int layer, const char* what) {
  if (!p) return fail(PALLAS_ERR_INVALID_ARG, "%s: null pool", what);
  if (!p->codes || !p->scales) return fail(PALLAS_ERR_INVALID_ARG, "%s: null codes or scales", what);
  if (p->num_pages <= 0 || p->page_size <= 0 || p->n_layers <= 0 || p->n_kv_heads <= 0 || p->head_dim <= 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: non-positive pool dimension", what);
  if (!aligned(p->codes, 16) || !aligned(p->scales, 16))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: codes or scales not 16-byte aligned", what);
  if (p->format != PALLAS_QUANT_E4M3 && p->format != PALLAS_QUANT_INT8 && p->format != PALLAS_QUANT_E2M1)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: format %d", what, p->format);
  if (layer < 0 || layer >= p->n_layers)
    return fail(PALLAS_ERR_OUT_OF_RANGE, "%s: layer %d of %d", what, layer, p->n_layers);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: head_dim %d (supported: 64, 128)", what, p->head_dim);
  if (p->page_size != 16)
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: page_size %d (supported: 16)", what, p->page_size);
  if (p->n_kv_heads > 4096) return fail(PALLAS_ERR_UNSUPPORTED, "%s: %d KV heads (at most 4096)", what, p->n_kv_heads);
  return PALLAS_OK;
}

// Rows of one layer's K plane.
int64_t plane_rows(const pallas_quant_pool* p) { return int64_t(p->num_pages) * p->page_size * p->n_kv_heads; }
// Bytes of a row's codes.
int code_bytes(const pallas_quant_pool* p) { return p->format == PALLAS_QUANT_E2M1 ? p->head_dim / 2 : p->head_dim; }
pallas::CacheType cache_type(const pallas_quant_pool* p) {
  return p->format == PALLAS_QUANT_E2M1 ? pallas::kCacheE2m1 : p->format == PALLAS_QUANT_INT8 ? pallas::kCacheInt8 : pallas::kCacheE4m3;
}

// The rows of a call that writes or reads tokens of a cache, of n_kv_heads and head_dim.
int check_rows(const char* what, int n_kv_heads, int head_dim, int32_t num_tokens, const int32_t* d_seq_ids,
               const int32_t* d_positions, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
               int32_t num_seqs, const int32_t* d_block_tables, int32_t max_pages, const int32_t* d_err) {
  if (num_tokens < 0 || num_seqs <= 0 || max_pages <= 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: negative num_tokens, or num_seqs or max_pages below 1", what);
  if (!d_positions || !k || !v || !d_block_tables)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: null positions, rows or tables", what);
  if (!d_seq_ids && num_tokens > num_seqs)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: %d tokens without sequence ids, of %d sequences", what, num_tokens, num_seqs);
  const int64_t row = int64_t(n_kv_heads) * head_dim;
  if (!aligned(k, 16) || !aligned(v, 16) || k_stride % 8 != 0 || v_stride % 8 != 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: rows not 16-byte aligned", what);
  if (k_stride < row || v_stride < row)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: row stride below the %lld elements of a row", what, (long long)row);
  if (!aligned(d_seq_ids, 4) || !aligned(d_positions, 4) || !aligned(d_block_tables, 4) || !aligned(d_err, 4))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: sequence ids, positions, tables or d_err not 4-byte aligned", what);
  return PALLAS_OK;
}

int check_kv_pool(const pallas_kv_pool* pool, int layer, const char* what) {
  if (int rc = pallas::check_pool(pool, what)) return rc;
  if (layer < 0 || layer >= pool->n_layers)
    return fail(PALLAS_ERR_OUT_OF_RANGE, "%s: layer %d of %d", what, layer, pool->n_layers);
  if (pool->page_size != 16)
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: page_size %d (supported: 16)", what, pool->page_size);
  return PALLAS_OK;
}

int check_plan(const pallas_rope_plan* plan) {
  if (!plan) return fail(PALLAS_ERR_INVALID_ARG, "rope: null plan");
  const int r = plan->rotary_dim;
  if (r < 2 || r > PALLAS_ROPE_MAX_DIM || r % 2 != 0 ||
      (plan->layout != PALLAS_ROPE_HALF && plan->layout != PALLAS_ROPE_INTERLEAVED) || !(plan->magnitude > 0.f))
    return fail(PALLAS_ERR_INVALID_ARG, "rope: not a plan that pallas_rope_init filled");
  return PALLAS_OK;
}

int quant_call(bool store, const pallas_quant_pool* pool, int32_t layer, int32_t num_tokens, const int32_t* d_seq_ids,
               const int32_t* d_positions, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
               int32_t num_seqs, const int32_t* d_block_tables, int32_t max_pages, int32_t* d_err, void* stream) {
  const char* what = store ? "quant store" : "quant load";
  if (int rc = check_quant_pool(pool, layer, what)) return rc;
  if (int rc = check_rows(what, pool->n_kv_heads, pool->head_dim, num_tokens, d_seq_ids, d_positions, k, k_stride, v,
                          v_stride, num_seqs, d_block_tables, max_pages, d_err))
    return rc;
  const int64_t row = int64_t(pool->n_kv_heads) * pool->head_dim;
  // A launch has fewer than 2^32 threads, 16 elements each.
  if (int64_t(num_tokens) * 2 * row >= (int64_t(1) << 35))
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: %d tokens of %lld K and V elements (below 2^35 in all)", what, num_tokens,
                (long long)(2 * row));
  pallas::QuantParams p{};
  p.codes = static_cast<uint8_t*>(pool->codes) + 2 * layer * plane_rows(pool) * code_bytes(pool);
  p.scales = pool->scales + 2 * layer * plane_rows(pool);
  p.num_pages = pool->num_pages;
  p.Hkv = pool->n_kv_heads;
  p.d = pool->head_dim;
  p.format = pool->format;
  p.seq = d_seq_ids;
  p.pos = d_positions;
  p.bt = d_block_tables;
  p.tokens = num_tokens;
  p.seqs = num_seqs;
  p.max_pages = max_pages;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.err = d_err;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (store) {
    p.k = static_cast<const uint16_t*>(k);
    p.v = static_cast<const uint16_t*>(v);
    pallas::ProfScope ps(PALLAS_K_QKV_EPI, s);
    return launched(pallas::launch_quant_store(p, s), "quant store launch");
  }
  p.k_out = static_cast<uint16_t*>(const_cast<void*>(k));
  p.v_out = static_cast<uint16_t*>(const_cast<void*>(v));
  pallas::ProfScope ps(PALLAS_K_PACK, s);
  return launched(pallas::launch_quant_load(p, s), "quant load launch");
}

// Appending to either kind of cache; the caller has checked the pool and set what p says of it.
int append_call(const char* what, const pallas_rope_plan* plan, pallas::AppendParams& p, int32_t num_tokens,
                const int32_t* d_seq_ids, const int32_t* d_positions, int32_t n_q_heads, const void* d_q,
                int64_t q_stride, void* d_q_out, int64_t q_out_stride, const void* d_k, int64_t k_stride,
                const void* d_v, int64_t v_stride, int32_t num_seqs, const int32_t* d_block_tables, int32_t max_pages,
                int32_t* d_err, void* stream) {
  if (int rc = check_plan(plan)) return rc;
  if (p.d != 64 && p.d != 128) return fail(PALLAS_ERR_UNSUPPORTED, "%s: head_dim %d (supported: 64, 128)", what, p.d);
  if (plan->rotary_dim > p.d)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: rotary_dim %d of heads of %d", what, plan->rotary_dim, p.d);
  if (int rc = check_rows(what, p.Hkv, p.d, num_tokens, d_seq_ids, d_positions, d_k, k_stride, d_v, v_stride, num_seqs,
                          d_block_tables, max_pages, d_err))
    return rc;
  if (n_q_heads < 0 || (n_q_heads > 0) != (d_q != nullptr) || (n_q_heads > 0) != (d_q_out != nullptr))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: %d query heads with %s", what, n_q_heads, d_q && d_q_out ? "rows" : "null rows");
  if (n_q_heads > 0) {
    const int64_t row = int64_t(n_q_heads) * p.d;
    if (!aligned(d_q, 16) || !aligned(d_q_out, 16) || q_stride % 8 != 0 || q_out_stride % 8 != 0)
      return fail(PALLAS_ERR_INVALID_ARG, "%s: query rows not 16-byte aligned", what);
    if (q_stride < row || q_out_stride < row)
      return fail(PALLAS_ERR_INVALID_ARG, "%s: query row stride below the %lld elements of a row", what, (long long)row);
    if (d_q == d_q_out && num_tokens > 1 && q_stride != q_out_stride)
      return fail(PALLAS_ERR_INVALID_ARG, "%s: queries in place with another stride", what);
  }
  if (num_tokens >= (1 << 24) || n_q_heads > 4096 || p.Hkv > 4096)   // (a launch has fewer than 2^32 threads)
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: %d tokens (below 2^24), %d query and %d KV heads (at most 4096)", what,
                num_tokens, n_q_heads, p.Hkv);
  p.q = static_cast<const uint16_t*>(d_q);
  p.q_out = static_cast<uint16_t*>(d_q_out);
  p.k = static_cast<const uint16_t*>(d_k);
  p.v = static_cast<const uint16_t*>(d_v);
  p.q_stride = q_stride;
  p.q_out_stride = q_out_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.Hq = n_q_heads;
  p.seq = d_seq_ids;
  p.pos = d_positions;
  p.bt = d_block_tables;
  p.tokens = num_tokens;
  p.seqs = num_seqs;
  p.max_pages = max_pages;
  p.err = d_err;
  p.r = plan->rotary_dim;
  p.interleaved = plan->layout == PALLAS_ROPE_INTERLEAVED;
  p.magnitude = plan->magnitude;
  std::copy(plan->turns, plan->turns + p.r / 2, p.turns);
  hipStream_t s = static_cast<hipStream_t>(stream);
  pallas::ProfScope ps(PALLAS_K_QKV_EPI, s);
  return launched(pallas::launch_append(p, s), "append launch");
}

// A call's workspace: two ints per sequence, then records of d + 2 floats per query head.
// `ranges`: of the call, or, where its cache is not known, the most of any.
struct AttendSpace {
  int records;
  size_t o_at, ml_at, bytes;
};
AttendSpace attend_space(int64_t seqs, int Hq, int d, int max_length, int ranges) {
  const int64_t records = pallas::attend_records(seqs, max_length, ranges);
  const size_t o_at = (seqs * 8 + 255) / 256 * 256, ml_at = o_at + size_t(records) * Hq * d * 4;
  return {int(records), o_at, ml_at, (ml_at + size_t(records) * Hq * 8 + 255) / 256 * 256};
}
int attend_ranges(pallas::CacheType t, int Hq, int Hkv, int d, bool listed) {
  if (pallas::attend_pairs(t, Hq, Hkv, listed)) return pallas::attend_ranges(pallas::kAttendPairGroups, Hkv / 2);
  return pallas::attend_ranges(pallas::attend_waves(t, d), pallas::attend_heads(Hq, Hkv));
}
int most_ranges(int Hq, int Hkv, int d) {
  int most = 0;
  for (pallas::CacheType t : {pallas::kCacheE4m3, pallas::kCacheE2m1})
    for (bool listed : {false, true}) most = std::max(most, attend_ranges(t, Hq, Hkv, d, listed));
  return most;
}

int check_attend(int32_t num_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_length,
                 const char* what) {
  if (num_seqs < 1 || n_q_heads < 1 || n_kv_heads < 1 || max_length < 1)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: num_seqs, heads and max_length must be at least 1", what);
  if (n_q_heads % n_kv_heads != 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: query heads not a multiple of KV heads", what);
  if (head_dim != 64 && head_dim != 128)
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: head_dim %d (supported: 64, 128)", what, head_dim);
  if (num_seqs > 65535 || n_q_heads > 4096)
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: %d sequences (at most 65535), %d query heads (at most 4096)", what, num_seqs,
                n_q_heads);
  if (pallas::attend_total(num_seqs, max_length) > (int64_t(1) << 30))
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: %d sequences of up to %d keys (at most 2^35 in all)", what, num_seqs, max_length);
  return PALLAS_OK;
}

// The blocks of a call's lists (attend_all: no lists, every block).
struct BlockLists {
  bool listed;
  const int32_t* d_blocks;
  int32_t max_blocks;
};
constexpr BlockLists attend_all{false, nullptr, 0};
constexpr int32_t kMaxListedLength = 1 << 30;      // 16 times a number of blocks is an int

// Checks and parameters of both cache types; the caller has checked the pool.
int attend_call(const char* what, pallas::CacheType type, pallas::AttendParams& p, int page_size, int32_t num_seqs,
                int32_t n_q_heads, const void* d_q, int64_t q_stride, const int32_t* d_lengths, int32_t max_length,
                const int32_t* d_block_tables, int32_t max_pages, BlockLists lists, float scale, void* d_out,
                int64_t out_stride, float* d_lse, void* d_workspace, size_t ws_bytes, int32_t* d_err, void* stream) {
  if (int rc = check_attend(num_seqs, n_q_heads, p.Hkv, p.d, max_length, what)) return rc;
  if (!d_q || !d_lengths || !d_block_tables || !d_out || max_pages <= 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: null query, lengths, tables or output, or max_pages <= 0", what);
  if (!aligned(d_q, 16) || !aligned(d_out, 16) || q_stride % 8 != 0 || out_stride % 8 != 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: query or output rows not 16-byte aligned", what);
  if (!aligned(d_lengths, 4) || !aligned(d_block_tables, 4) || !aligned(d_lse, 4) || !aligned(d_err, 4))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: lengths, tables, d_lse or d_err not 4-byte aligned", what);
  const int64_t row = int64_t(n_q_heads) * p.d;
  if (q_stride < row || out_stride < row)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: row stride below the %lld elements of a row", what, (long long)row);
  if (max_length > int64_t(max_pages) * page_size)
    return fail(PALLAS_ERR_OUT_OF_RANGE, "%s: max_length %d outside the table (%lld)", what, max_length,
                (long long)(int64_t(max_pages) * page_size));
  if (lists.listed && (!lists.d_blocks || !aligned(lists.d_blocks, 4) || lists.max_blocks < 1))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: blocks null or not 4-byte aligned, or max_blocks below 1", what);
  if (lists.listed && max_length > kMaxListedLength)
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: max_length %d (at most 2^30)", what, max_length);
  p.scale_log2 = static_cast<float>(double(scale) * 1.4426950408889634);
  if (!std::isfinite(p.scale_log2)) return fail(PALLAS_ERR_INVALID_ARG, "%s: scale is not finite", what);
  if (!d_workspace || !aligned(d_workspace, 256))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: workspace null or not 256-byte aligned", what);
  p.lists = lists.d_blocks;
  p.listed = lists.max_blocks;
  p.max_row = lists.listed ? std::min((max_length - 1) / page_size + 1, lists.max_blocks) * page_size : max_length;
  p.ranges = attend_ranges(type, n_q_heads, p.Hkv, p.d, lists.listed);
  const AttendSpace sp = attend_space(num_seqs, n_q_heads, p.d, p.max_row, p.ranges);
  if (ws_bytes < sp.bytes)
    return fail(PALLAS_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, sp.bytes);
  p.Hq = n_q_heads;
  p.G = n_q_heads / p.Hkv;
  p.seqs = num_seqs;
  p.max_length = max_length;
  p.max_pages = max_pages;
  p.q = static_cast<const uint16_t*>(d_q);
  p.q_stride = q_stride;
  p.lengths = d_lengths;
  p.bt = d_block_tables;
  p.out = static_cast<uint16_t*>(d_out);
  p.out_stride = out_stride;
  p.lse = d_lse;
  p.records = sp.records;
  char* ws = static_cast<char*>(d_workspace);
  p.parts = reinterpret_cast<int32_t*>(ws);
  p.part_o = reinterpret_cast<float*>(ws + sp.o_at);
  p.part_ml = reinterpret_cast<float*>(ws + sp.ml_at);
  p.err = d_err;
  hipStream_t s = static_cast<hipStream_t>(stream);
  pallas::ProfScope ps(PALLAS_K_DECODE_ATTN, s);
  return launched(pallas::launch_attend(p, type, s), "attend launch");
}

int attend_kv(const char* what, const pallas_kv_pool* pool, int32_t layer, int32_t num_seqs, int32_t n_q_heads,
              const void* d_q, int64_t q_stride, const int32_t* d_lengths, int32_t max_length,
              const int32_t* d_block_tables, int32_t max_pages, BlockLists lists, float scale, void* d_out,
              int64_t out_stride, float* d_lse, void* d_workspace, size_t ws_bytes, int32_t* d_err, void* stream) {
  if (int rc = check_kv_pool(pool, layer, what)) return rc;
  const int64_t plane = int64_t(pool->num_pages) * pool->page_size * pool->n_kv_heads * pool->head_dim;
  pallas::AttendParams p{};
  p.k = static_cast<const uint16_t*>(pool->base) + 2 * layer * plane;
  p.v = static_cast<const uint16_t*>(pool->base) + (2 * layer + 1) * plane;
  p.num_pages = pool->num_pages;
  p.Hkv = pool->n_kv_heads;
  p.d = pool->head_dim;
  return attend_call(what, pallas::kCacheBf16, p, pool->page_size, num_seqs, n_q_heads, d_q, q_stride, d_lengths,
                     max_length, d_block_tables, max_pages, lists, scale, d_out, out_stride, d_lse, d_workspace, ws_bytes,
                     d_err, stream);
}

int attend_quant(const char* what, const pallas_quant_pool* pool, int32_t layer, int32_t num_seqs, int32_t n_q_heads,
                 const void* d_q, int64_t q_stride, const int32_t* d_lengths, int32_t max_length,
                 const int32_t* d_block_tables, int32_t max_pages, BlockLists lists, float scale, void* d_out,
                 int64_t out_stride, float* d_lse, void* d_workspace, size_t ws_bytes, int32_t* d_err, void* stream) {
  if (int rc = check_quant_pool(pool, layer, what)) return rc;
  const int64_t rows = plane_rows(pool);
  if (2 * rows * 4 > int64_t(0xFFFFFF00))   // addressed with 32-bit offsets
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: a layer's scales of %lld bytes exceed 4 GiB", what, (long long)(2 * rows * 4));
  pallas::AttendParams p{};
  p.k = static_cast<const uint8_t*>(pool->codes) + 2 * layer * rows * code_bytes(pool);
  p.v = static_cast<const uint8_t*>(pool->codes) + (2 * layer + 1) * rows * code_bytes(pool);
  p.scales = pool->scales + 2 * layer * rows;
  p.num_pages = pool->num_pages;
  p.Hkv = pool->n_kv_heads;
  p.d = pool->head_dim;
  return attend_call(what, cache_type(pool), p, pool->page_size, num_seqs, n_q_heads, d_q, q_stride, d_lengths,
                     max_length, d_block_tables, max_pages, lists, scale, d_out, out_stride, d_lse, d_workspace, ws_bytes,
                     d_err, stream);
}

// ------------------------------------------------------------ blocks
int check_bounds(const pallas_bounds_pool* b, int layer, const char* what) {
  if (!b) return fail(PALLAS_ERR_INVALID_ARG, "%s: null bounds", what);
  if (!b->codes || !b->scales || !aligned(b->codes, 16) || !aligned(b->scales, 16))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: bounds' codes or scales null or not 16-byte aligned", what);
  if (b->num_pages <= 0 || b->n_layers <= 0 || b->n_kv_heads <= 0 || b->head_dim <= 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: non-positive dimension of the bounds", what);
  if (layer < 0 || layer >= b->n_layers)
    return fail(PALLAS_ERR_OUT_OF_RANGE, "%s: layer %d of %d", what, layer, b->n_layers);
  if (b->head_dim != 64 && b->head_dim != 128)
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: head_dim %d (supported: 64, 128)", what, b->head_dim);
  if (b->n_kv_heads > 4096) return fail(PALLAS_ERR_UNSUPPORTED, "%s: %d KV heads (at most 4096)", what, b->n_kv_heads);
  return PALLAS_OK;
}

int bounds_call(const char* what, pallas::CacheType type, pallas::BoundsParams& p, int n_layers,
                const pallas_bounds_pool* bounds, int32_t layer, int32_t num_seqs, const int32_t* d_start,
                const int32_t* d_lengths, int32_t max_new, const int32_t* d_block_tables, int32_t max_pages,
                int32_t* d_err, void* stream) {
  if (int rc = check_bounds(bounds, layer, what)) return rc;
  if (bounds->num_pages != p.num_pages || bounds->n_layers != n_layers || bounds->n_kv_heads != p.Hkv || bounds->head_dim != p.d)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: bounds and cache of different pages, layers, heads or head_dim", what);
  if (num_seqs < 1 || max_new < 1 || max_pages <= 0 || !d_start || !d_lengths || !d_block_tables)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: null start, lengths or tables, or num_seqs, max_new or max_pages below 1", what);
  if (!aligned(d_start, 4) || !aligned(d_lengths, 4) || !aligned(d_block_tables, 4) || !aligned(d_err, 4))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: start, lengths, tables or d_err not 4-byte aligned", what);
  if (num_seqs > 65535 || int64_t(std::min(pallas::bounds_blocks(max_new), max_pages)) * p.Hkv >= (1 << 26))
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: %d sequences (at most 65535), up to %d positions of %d heads (below 2^26 blocks and heads)",
                what, num_seqs, max_new, p.Hkv);
  const int64_t rows = int64_t(bounds->num_pages) * bounds->n_kv_heads;
  p.bounds = static_cast<int8_t*>(bounds->codes) + 2 * layer * rows * bounds->head_dim;
  p.bound_scales = bounds->scales + layer * rows;
  p.start = d_start;
  p.lengths = d_lengths;
  p.most = max_new;
  p.bt = d_block_tables;
  p.seqs = num_seqs;
  p.max_pages = max_pages;
  p.err = d_err;
  hipStream_t s = static_cast<hipStream_t>(stream);
  pallas::ProfScope ps(PALLAS_K_QKV_EPI, s);
  return launched(pallas::launch_bounds(p, type, s), "bounds launch");
}

int check_select(int32_t num_seqs, int32_t n_kv_heads, int32_t max_length, const char* what) {
  if (num_seqs < 1 || max_length < 1)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: num_seqs and max_length must be at least 1", what);
  if (num_seqs > 65535 || max_length > kMaxListedLength || int64_t(num_seqs) * max_length > (int64_t(1) << 35) ||
      int64_t(max_length) * n_kv_heads >= (int64_t(1) << 34))      // (a launch has fewer than 2^32 threads)
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: %d sequences (at most 65535) of up to %d keys (at most 2^30, 2^35 in all, 2^34 times the KV heads)",
                what, num_seqs, max_length);
  return PALLAS_OK;
}
// The scores of a call: one word per sequence, KV head and block.
int64_t select_stride(int max_length) { return (int64_t(max_length) + 63) / 64 * 4; }
size_t select_space(int64_t seqs, int Hkv, int max_length) {
  return (size_t(seqs) * Hkv * select_stride(max_length) * 4 + 255) / 256 * 256;
}

}  // namespace

extern "C" {

int pallas_rope_init(const pallas_rope_config* cfg, pallas_rope_plan* plan) {
  if (!cfg || !plan) return fail(PALLAS_ERR_INVALID_ARG, "rope: null config or plan");
  const pallas_rope_config& c = *cfg;
  const int r = c.rotary_dim;
  if (r < 2 || r > PALLAS_ROPE_MAX_DIM || r % 2 != 0)
    return fail(PALLAS_ERR_INVALID_ARG, "rope: rotary_dim %d (even, 2 to %d)", r, PALLAS_ROPE_MAX_DIM);
  if (c.layout != PALLAS_ROPE_HALF && c.layout != PALLAS_ROPE_INTERLEAVED)
    return fail(PALLAS_ERR_INVALID_ARG, "rope: layout %d", c.layout);
  if (c.scaling < PALLAS_ROPE_UNSCALED || c.scaling > PALLAS_ROPE_BANDS)
    return fail(PALLAS_ERR_INVALID_ARG, "rope: scaling %d", c.scaling);
  if (!(c.theta > 1.0) || !std::isfinite(c.theta)) return fail(PALLAS_ERR_INVALID_ARG, "rope: theta must be above 1");
  if (c.scaling != PALLAS_ROPE_UNSCALED && (!(c.factor >= 1.0) || !std::isfinite(c.factor)))
    return fail(PALLAS_ERR_INVALID_ARG, "rope: factor must be at least 1");
  if (c.scaling == PALLAS_ROPE_YARN || c.scaling == PALLAS_ROPE_BANDS) {
    if (c.trained_len < 1) return fail(PALLAS_ERR_INVALID_ARG, "rope: trained_len %d", c.trained_len);
    if (!(c.slow > 0.0) || !(c.fast > c.slow) || !std::isfinite(c.fast))
      return fail(PALLAS_ERR_INVALID_ARG, "rope: fast must be above slow, and slow above 0");
  }
  if (!(c.magnitude >= 0.0) || !std::isfinite(c.magnitude))
    return fail(PALLAS_ERR_INVALID_ARG, "rope: magnitude must be positive, or 0");
  // In 64-bit mantissas: the largest frequency, a sixth of a turn, is kept to 2^-64.
  typedef long double real;
  const real two_pi = 6.283185307179586476925286766559L, L = c.trained_len, s = c.factor;
  const real theta = c.scaling == PALLAS_ROPE_NTK && r > 2 ? c.theta * std::pow(s, real(r) / (r - 2)) : real(c.theta);
  auto pair_of = [&](real turns) { return r * std::log(L / (turns * two_pi)) / (2 * std::log(real(c.theta))); };
  real lo = 0, hi = 0;
  if (c.scaling == PALLAS_ROPE_YARN) {
    lo = std::max(std::floor(pair_of(c.fast)), real(0));
    hi = std::min(std::ceil(pair_of(c.slow)), real(r - 1));
  }
  pallas_rope_plan out{};
  out.rotary_dim = r;
  out.layout = c.layout;
  double m = c.magnitude;
  if (m == 0.0) m = c.scaling == PALLAS_ROPE_YARN ? 0.1 * std::log(c.factor) + 1.0 : 1.0;
  if (!(m >= 0x1p-126 && m <= 0x1p126))
    return fail(PALLAS_ERR_INVALID_ARG, "rope: magnitude %g (2^-126 to 2^126)", m);
  out.magnitude = static_cast<float>(m);
  for (int i = 0; i < r / 2; ++i) {
    real f = std::pow(theta, real(-2 * i) / r);
    auto mix = [&](real w, real kept) { return kept * (1 - w) + kept / s * w; };   // w: how far scaled
    auto clamp01 = [](real w) { return std::min(std::max(w, real(0)), real(1)); };
    if (c.scaling == PALLAS_ROPE_LINEAR) f /= s;
    if (c.scaling == PALLAS_ROPE_YARN) f = mix(clamp01((i - lo) / std::max(hi - lo, real(0.001L))), f);
    if (c.scaling == PALLAS_ROPE_BANDS) f = mix(1 - clamp01((L * f / two_pi - c.slow) / (real(c.fast) - c.slow)), f);
    out.turns[i] = static_cast<uint64_t>(std::ldexp(f / two_pi, 64));
  }
  *plan = out;
  return PALLAS_OK;
}

int pallas_rope_apply(const pallas_rope_plan* plan, int32_t inverse, int32_t num_tokens, int32_t n_heads,
                      int32_t head_dim, const int32_t* d_positions, const void* d_x, int64_t x_token_stride,
                      int64_t x_head_stride, void* d_y, int64_t y_token_stride, int64_t y_head_stride, void* stream) {
  if (int rc = check_plan(plan)) return rc;
  const int r = plan->rotary_dim;
  if (num_tokens < 0 || n_heads < 1 || head_dim < r)
    return fail(PALLAS_ERR_INVALID_ARG, "rope: %d tokens of %d heads of %d (rotary_dim %d)", num_tokens, n_heads, head_dim, r);
  if (!d_positions || !d_x || !d_y) return fail(PALLAS_ERR_INVALID_ARG, "rope: null positions or rows");
  if (!aligned(d_x, 2) || !aligned(d_y, 2) || !aligned(d_positions, 4))
    return fail(PALLAS_ERR_INVALID_ARG, "rope: rows not 2-byte, or positions not 4-byte aligned");
  if (x_token_stride < 0 || x_head_stride < 0 || y_token_stride < 0 || y_head_stride < 0)
    return fail(PALLAS_ERR_INVALID_ARG, "rope: negative stride");
  if (int64_t(n_heads) * head_dim > (int64_t(1) << 20) || num_tokens >= (1 << 24))
    return fail(PALLAS_ERR_UNSUPPORTED, "rope: %d tokens (below 2^24) of %d heads of %d (at most 2^20 elements)", num_tokens,
                n_heads, head_dim);
  // Heads written may not fall on each other (heads read may: a stride of 0 repeats them):
  // of the two dimensions, one steps over all of the other.
  auto apart = [&](int64_t inner, int64_t n, int64_t outer, int64_t m) {
    return (n <= 1 || inner >= head_dim) && (m <= 1 || (outer >= head_dim && (n <= 1 || (outer - head_dim) / (n - 1) >= inner)));
  };
  if (!apart(y_head_stride, n_heads, y_token_stride, num_tokens) && !apart(y_token_stride, num_tokens, y_head_stride, n_heads))
    return fail(PALLAS_ERR_INVALID_ARG, "rope: output strides at which heads of %d overlap", head_dim);
  if (d_x == d_y && ((num_tokens > 1 && x_token_stride != y_token_stride) || (n_heads > 1 && x_head_stride != y_head_stride)))
    return fail(PALLAS_ERR_INVALID_ARG, "rope: in place with other strides");
  pallas::RopeParams p;
  p.x = static_cast<const uint16_t*>(d_x);
  p.y = static_cast<uint16_t*>(d_y);
  p.x_token = x_token_stride;
  p.x_head = x_head_stride;
  p.y_token = y_token_stride;
  p.y_head = y_head_stride;
  p.pos = d_positions;
  p.tokens = num_tokens;
  p.heads = n_heads;
  p.d = head_dim;
  p.r = r;
  p.interleaved = plan->layout == PALLAS_ROPE_INTERLEAVED;
  p.negate = inverse != 0;
  p.magnitude = inverse ? 1.0f / plan->magnitude : plan->magnitude;
  std::copy(plan->turns, plan->turns + PALLAS_ROPE_MAX_DIM / 2, p.turns);
  hipStream_t s = static_cast<hipStream_t>(stream);
  pallas::ProfScope ps(PALLAS_K_QKV_EPI, s);
  return launched(pallas::launch_rope(p, s), "rope launch");
}

int pallas_quant_store(const pallas_quant_pool* pool, int32_t layer, int32_t num_tokens, const int32_t* d_seq_ids,
                       const int32_t* d_positions, const void* d_k, int64_t k_stride, const void* d_v,
                       int64_t v_stride, int32_t num_seqs, const int32_t* d_block_tables, int32_t max_pages,
                       int32_t* d_err, void* stream) {
  return quant_call(true, pool, layer, num_tokens, d_seq_ids, d_positions, d_k, k_stride, d_v, v_stride, num_seqs,
                    d_block_tables, max_pages, d_err, stream);
}

int pallas_quant_load(const pallas_quant_pool* pool, int32_t layer, int32_t num_tokens, const int32_t* d_seq_ids,
                      const int32_t* d_positions, void* d_k, int64_t k_stride, void* d_v, int64_t v_stride,
                      int32_t num_seqs, const int32_t* d_block_tables, int32_t max_pages, int32_t* d_err,
                      void* stream) {
  return quant_call(false, pool, layer, num_tokens, d_seq_ids, d_positions, d_k, k_stride, d_v, v_stride, num_seqs,
                    d_block_tables, max_pages, d_err, stream);
}

int pallas_append_kv(const pallas_rope_plan* plan, const pallas_kv_pool* pool, int32_t layer, int32_t num_tokens,
                     const int32_t* d_seq_ids, const int32_t* d_positions, int32_t n_q_heads, const void* d_q,
                     int64_t q_stride, void* d_q_out, int64_t q_out_stride, const void* d_k, int64_t k_stride,
                     const void* d_v, int64_t v_stride, int32_t num_seqs, const int32_t* d_block_tables,
                     int32_t max_pages, int32_t* d_err, void* stream) {
  if (int rc = check_kv_pool(pool, layer, "append")) return rc;
  pallas::AppendParams p{};
  const int64_t plane = int64_t(pool->num_pages) * pool->page_size * pool->n_kv_heads * pool->head_dim;
  p.cache = static_cast<uint16_t*>(pool->base) + 2 * layer * plane;
  p.num_pages = pool->num_pages;
  p.Hkv = pool->n_kv_heads;
  p.d = pool->head_dim;
  return append_call("append", plan, p, num_tokens, d_seq_ids, d_positions, n_q_heads, d_q, q_stride, d_q_out,
                     q_out_stride, d_k, k_stride, d_v, v_stride, num_seqs, d_block_tables, max_pages, d_err, stream);
}

int pallas_append_quant(const pallas_rope_plan* plan, const pallas_quant_pool* pool, int32_t layer, int32_t num_tokens,
                        const int32_t* d_seq_ids, const int32_t* d_positions, int32_t n_q_heads, const void* d_q,
                        int64_t q_stride, void* d_q_out, int64_t q_out_stride, const void* d_k, int64_t k_stride,
                        const void* d_v, int64_t v_stride, int32_t num_seqs, const int32_t* d_block_tables,
                        int32_t max_pages, int32_t* d_err, void* stream) {
  if (int rc = check_quant_pool(pool, layer, "append (quantised)")) return rc;
  pallas::AppendParams p{};
  p.cache = static_cast<uint8_t*>(pool->codes) + 2 * layer * plane_rows(pool) * code_bytes(pool);
  p.scales = pool->scales + 2 * layer * plane_rows(pool);
  p.format = pool->format;
  p.num_pages = pool->num_pages;
  p.Hkv = pool->n_kv_heads;
  p.d = pool->head_dim;
  return append_call("append (quantised)", plan, p, num_tokens, d_seq_ids, d_positions, n_q_heads, d_q, q_stride, d_q_out,
                     q_out_stride, d_k, k_stride, d_v, v_stride, num_seqs, d_block_tables, max_pages, d_err, stream);
}

int pallas_attend_kv(const pallas_kv_pool* pool, int32_t layer, int32_t num_seqs, int32_t n_q_heads, const void* d_q,
                     int64_t q_stride, const int32_t* d_lengths, int32_t max_length, const int32_t* d_block_tables,
                     int32_t max_pages, float scale, void* d_out, int64_t out_stride, float* d_lse, void* d_workspace,
                     size_t ws_bytes, int32_t* d_err, void* stream) {
  return attend_kv("attend", pool, layer, num_seqs, n_q_heads, d_q, q_stride, d_lengths, max_length, d_block_tables,
                   max_pages, attend_all, scale, d_out, out_stride, d_lse, d_workspace, ws_bytes, d_err, stream);
}

int pallas_attend_quant(const pallas_quant_pool* pool, int32_t layer, int32_t num_seqs, int32_t n_q_heads,
                        const void* d_q, int64_t q_stride, const int32_t* d_lengths, int32_t max_length,
                        const int32_t* d_block_tables, int32_t max_pages, float scale, void* d_out,
                        int64_t out_stride, float* d_lse, void* d_workspace, size_t ws_bytes, int32_t* d_err,
                        void* stream) {
  return attend_quant("attend (quantised)", pool, layer, num_seqs, n_q_heads, d_q, q_stride, d_lengths, max_length,
                      d_block_tables, max_pages, attend_all, scale, d_out, out_stride, d_lse, d_workspace, ws_bytes,
                      d_err, stream);
}

int pallas_attend_blocks_kv(const pallas_kv_pool* pool, int32_t layer, int32_t num_seqs, int32_t n_q_heads,
                            const void* d_q, int64_t q_stride, const int32_t* d_lengths, int32_t max_length,
                            const int32_t* d_block_tables, int32_t max_pages, const int32_t* d_blocks,
                            int32_t max_blocks, float scale, void* d_out, int64_t out_stride, float* d_lse,
                            void* d_workspace, size_t ws_bytes, int32_t* d_err, void* stream) {
  return attend_kv("attend (blocks)", pool, layer, num_seqs, n_q_heads, d_q, q_stride, d_lengths, max_length,
                   d_block_tables, max_pages, {true, d_blocks, max_blocks}, scale, d_out, out_stride, d_lse, d_workspace,
                   ws_bytes, d_err, stream);
}

int pallas_attend_blocks_quant(const pallas_quant_pool* pool, int32_t layer, int32_t num_seqs, int32_t n_q_heads,
                               const void* d_q, int64_t q_stride, const int32_t* d_lengths, int32_t max_length,
                               const int32_t* d_block_tables, int32_t max_pages, const int32_t* d_blocks,
                               int32_t max_blocks, float scale, void* d_out, int64_t out_stride, float* d_lse,
                               void* d_workspace, size_t ws_bytes, int32_t* d_err, void* stream) {
  return attend_quant("attend (blocks, quantised)", pool, layer, num_seqs, n_q_heads, d_q, q_stride, d_lengths,
                      max_length, d_block_tables, max_pages, {true, d_blocks, max_blocks}, scale, d_out, out_stride,
                      d_lse, d_workspace, ws_bytes, d_err, stream);
}

int pallas_bounds_kv(const pallas_kv_pool* pool, const pallas_bounds_pool* bounds, int32_t layer, int32_t num_seqs,
                     const int32_t* d_start, const int32_t* d_lengths, int32_t max_new, const int32_t* d_block_tables,
                     int32_t max_pages, int32_t* d_err, void* stream) {
  if (int rc = check_kv_pool(pool, layer, "bounds")) return rc;
  pallas::BoundsParams p{};
  const int64_t plane = int64_t(pool->num_pages) * pool->page_size * pool->n_kv_heads * pool->head_dim;
  p.k = static_cast<const uint16_t*>(pool->base) + 2 * layer * plane;
  p.num_pages = pool->num_pages;
  p.Hkv = pool->n_kv_heads;
  p.d = pool->head_dim;
  return bounds_call("bounds", pallas::kCacheBf16, p, pool->n_layers, bounds, layer, num_seqs, d_start, d_lengths, max_new,
                     d_block_tables, max_pages, d_err, stream);
}

int pallas_bounds_quant(const pallas_quant_pool* pool, const pallas_bounds_pool* bounds, int32_t layer,
                        int32_t num_seqs, const int32_t* d_start, const int32_t* d_lengths, int32_t max_new,
                        const int32_t* d_block_tables, int32_t max_pages, int32_t* d_err, void* stream) {
  if (int rc = check_quant_pool(pool, layer, "bounds (quantised)")) return rc;
  pallas::BoundsParams p{};
  p.k = static_cast<const uint8_t*>(pool->codes) + 2 * layer * plane_rows(pool) * code_bytes(pool);
  p.scales = pool->scales + 2 * layer * plane_rows(pool);
  p.num_pages = pool->num_pages;
  p.Hkv = pool->n_kv_heads;
  p.d = pool->head_dim;
  return bounds_call("bounds (quantised)", cache_type(pool), p, pool->n_layers, bounds, layer, num_seqs, d_start,
                     d_lengths, max_new, d_block_tables, max_pages, d_err, stream);
}

int pallas_select_blocks(const pallas_bounds_pool* bounds, int32_t layer, int32_t num_seqs, int32_t n_q_heads,
                         const void* d_q, int64_t q_stride, const int32_t* d_lengths, int32_t max_length,
                         const int32_t* d_block_tables, int32_t max_pages, int32_t max_blocks, int32_t first,
                         int32_t last, int32_t* d_blocks, void* d_workspace, size_t ws_bytes, int32_t* d_err,
                         void* stream) {
  const char* what = "select";
  if (int rc = check_bounds(bounds, layer, what)) return rc;
  if (int rc = check_select(num_seqs, bounds->n_kv_heads, max_length, what)) return rc;
  if (n_q_heads < 1 || n_q_heads % bounds->n_kv_heads != 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: query heads not a multiple of KV heads", what);
  if (n_q_heads > 4096) return fail(PALLAS_ERR_UNSUPPORTED, "%s: %d query heads (at most 4096)", what, n_q_heads);
  if (!d_q || !d_lengths || !d_block_tables || !d_blocks || max_pages <= 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: null query, lengths, tables or blocks, or max_pages <= 0", what);
  if (!aligned(d_q, 16) || q_stride % 8 != 0) return fail(PALLAS_ERR_INVALID_ARG, "%s: query rows not 16-byte aligned", what);
  if (q_stride < int64_t(n_q_heads) * bounds->head_dim)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: row stride below the %lld elements of a row", what,
                (long long)(int64_t(n_q_heads) * bounds->head_dim));
  if (!aligned(d_lengths, 4) || !aligned(d_block_tables, 4) || !aligned(d_blocks, 4) || !aligned(d_err, 4))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: lengths, tables, blocks or d_err not 4-byte aligned", what);
  if (max_length > int64_t(max_pages) * 16)
    return fail(PALLAS_ERR_OUT_OF_RANGE, "%s: max_length %d outside the table (%lld)", what, max_length,
                (long long)(int64_t(max_pages) * 16));
  if (max_blocks < 1 || first < 0 || last < 0 || int64_t(first) + last > max_blocks)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: %d blocks, of them the first %d and the last %d", what, max_blocks, first, last);
  if (!d_workspace || !aligned(d_workspace, 256))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: workspace null or not 256-byte aligned", what);
  const size_t need = select_space(num_seqs, bounds->n_kv_heads, max_length);
  if (ws_bytes < need) return fail(PALLAS_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need);
  const int64_t rows = int64_t(bounds->num_pages) * bounds->n_kv_heads;
  pallas::SelectParams p{};
  p.bounds = static_cast<const int8_t*>(bounds->codes) + 2 * layer * rows * bounds->head_dim;
  p.bound_scales = bounds->scales + layer * rows;
  p.num_pages = bounds->num_pages;
  p.Hkv = bounds->n_kv_heads;
  p.G = n_q_heads / p.Hkv;
  p.d = bounds->head_dim;
  p.q = static_cast<const uint16_t*>(d_q);
  p.q_stride = q_stride;
  p.lengths = d_lengths;
  p.max_length = max_length;
  p.bt = d_block_tables;
  p.seqs = num_seqs;
  p.max_pages = max_pages;
  p.budget = max_blocks;
  p.first = first;
  p.last = last;
  p.blocks = d_blocks;
  p.order = static_cast<uint32_t*>(d_workspace);
  p.stride = select_stride(max_length);
  p.err = d_err;
  hipStream_t s = static_cast<hipStream_t>(stream);
  pallas::ProfScope ps(PALLAS_K_DECODE_ATTN, s);
  return launched(pallas::launch_select(p, s), "select launch");
}

size_t pallas_select_workspace_size(int32_t num_seqs, int32_t n_kv_heads, int32_t max_length) {
  if (n_kv_heads < 1 || n_kv_heads > 4096 || check_select(num_seqs, n_kv_heads, max_length, "select workspace") != PALLAS_OK)
    return 0;
  return select_space(num_seqs, n_kv_heads, max_length);
}

size_t pallas_attend_workspace_size(int32_t num_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                    int32_t max_length) {
  if (check_attend(num_seqs, n_q_heads, n_kv_heads, head_dim, max_length, "attend workspace") != PALLAS_OK) return 0;
  return attend_space(num_seqs, n_q_heads, head_dim, max_length, most_ranges(n_q_heads, n_kv_heads, head_dim)).bytes;
}

}  // extern "C"
