// C ABI of the cache operators (rotary positions, the 8-bit cache, attention of one
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
  if (p->format != PALLAS_QUANT_E4M3 && p->format != PALLAS_QUANT_INT8)
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

int quant_call(bool store, const pallas_quant_pool* pool, int32_t layer, int32_t num_tokens, const int32_t* d_seq_ids,
               const int32_t* d_positions, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
               int32_t num_seqs, const int32_t* d_block_tables, int32_t max_pages, int32_t* d_err, void* stream) {
  const char* what = store ? "quant store" : "quant load";
  if (int rc = check_quant_pool(pool, layer, what)) return rc;
  if (num_tokens < 0 || num_seqs <= 0 || max_pages <= 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: negative num_tokens, or num_seqs or max_pages below 1", what);
  if (!d_positions || !k || !v || !d_block_tables)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: null positions, rows or tables", what);
  if (!d_seq_ids && num_tokens > num_seqs)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: %d tokens without sequence ids, of %d sequences", what, num_tokens, num_seqs);
  const int64_t row = int64_t(pool->n_kv_heads) * pool->head_dim;
  if (!aligned(k, 16) || !aligned(v, 16) || k_stride % 8 != 0 || v_stride % 8 != 0)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: rows not 16-byte aligned", what);
  if (k_stride < row || v_stride < row)
    return fail(PALLAS_ERR_INVALID_ARG, "%s: row stride below the %lld elements of a row", what, (long long)row);
  if (!aligned(d_seq_ids, 4) || !aligned(d_positions, 4) || !aligned(d_block_tables, 4) || !aligned(d_err, 4))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: sequence ids, positions, tables or d_err not 4-byte aligned", what);
  // A launch has fewer than 2^32 threads, 16 elements each.
  if (int64_t(num_tokens) * 2 * row >= (int64_t(1) << 35))
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: %d tokens of %lld K and V elements (below 2^35 in all)", what, num_tokens,
                (long long)(2 * row));
  pallas::QuantParams p{};
  p.codes = static_cast<uint8_t*>(pool->codes) + 2 * layer * plane_rows(pool) * pool->head_dim;
  p.scales = pool->scales + 2 * layer * plane_rows(pool);
  p.num_pages = pool->num_pages;
  p.Hkv = pool->n_kv_heads;
  p.d = pool->head_dim;
  p.int8 = pool->format == PALLAS_QUANT_INT8;
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

// A call's workspace: two ints per sequence, then records of d + 2 floats per query head.
// `ranges`: of the call, or the most of any cache type.
struct AttendSpace {
  int records;
  size_t o_at, ml_at, bytes;
};
AttendSpace attend_space(int64_t seqs, int Hq, int d, int max_length, int ranges) {
  const int64_t records = pallas::attend_records(seqs, max_length, ranges);
  const size_t o_at = (seqs * 8 + 255) / 256 * 256, ml_at = o_at + size_t(records) * Hq * d * 4;
  return {int(records), o_at, ml_at, (ml_at + size_t(records) * Hq * 8 + 255) / 256 * 256};
}
int most_ranges(int Hq, int Hkv, int d) { return pallas::attend_ranges(d, pallas::attend_heads(Hq, Hkv)); }

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

// Checks and parameters of both cache types; the caller has checked the pool.
int attend_call(const char* what, pallas::CacheType type, pallas::AttendParams& p, int page_size, int32_t num_seqs,
                int32_t n_q_heads, const void* d_q, int64_t q_stride, const int32_t* d_lengths, int32_t max_length,
                const int32_t* d_block_tables, int32_t max_pages, float scale, void* d_out, int64_t out_stride,
                float* d_lse, void* d_workspace, size_t ws_bytes, int32_t* d_err, void* stream) {
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
  p.scale_log2 = static_cast<float>(double(scale) * 1.4426950408889634);
  if (!std::isfinite(p.scale_log2)) return fail(PALLAS_ERR_INVALID_ARG, "%s: scale is not finite", what);
  if (!d_workspace || !aligned(d_workspace, 256))
    return fail(PALLAS_ERR_INVALID_ARG, "%s: workspace null or not 256-byte aligned", what);
  const AttendSpace sp = attend_space(num_seqs, n_q_heads, p.d, max_length, most_ranges(n_q_heads, p.Hkv, p.d));
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
  p.ranges = pallas::attend_ranges(type == pallas::kCacheBf16 ? 2 * p.d : p.d, pallas::attend_heads(n_q_heads, p.Hkv));
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
  if (!plan) return fail(PALLAS_ERR_INVALID_ARG, "rope: null plan");
  const int r = plan->rotary_dim;
  if (r < 2 || r > PALLAS_ROPE_MAX_DIM || r % 2 != 0 ||
      (plan->layout != PALLAS_ROPE_HALF && plan->layout != PALLAS_ROPE_INTERLEAVED) || !(plan->magnitude > 0.f))
    return fail(PALLAS_ERR_INVALID_ARG, "rope: not a plan that pallas_rope_init filled");
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

int pallas_attend_kv(const pallas_kv_pool* pool, int32_t layer, int32_t num_seqs, int32_t n_q_heads, const void* d_q,
                     int64_t q_stride, const int32_t* d_lengths, int32_t max_length, const int32_t* d_block_tables,
                     int32_t max_pages, float scale, void* d_out, int64_t out_stride, float* d_lse, void* d_workspace,
                     size_t ws_bytes, int32_t* d_err, void* stream) {
  const char* what = "attend";
  if (int rc = pallas::check_pool(pool, what)) return rc;
  if (layer < 0 || layer >= pool->n_layers)
    return fail(PALLAS_ERR_OUT_OF_RANGE, "%s: layer %d of %d", what, layer, pool->n_layers);
  if (pool->page_size != 16)
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: page_size %d (supported: 16)", what, pool->page_size);
  const int64_t plane = int64_t(pool->num_pages) * pool->page_size * pool->n_kv_heads * pool->head_dim;
  pallas::AttendParams p{};
  p.k = static_cast<const uint16_t*>(pool->base) + 2 * layer * plane;
  p.v = static_cast<const uint16_t*>(pool->base) + (2 * layer + 1) * plane;
  p.num_pages = pool->num_pages;
  p.Hkv = pool->n_kv_heads;
  p.d = pool->head_dim;
  return attend_call(what, pallas::kCacheBf16, p, pool->page_size, num_seqs, n_q_heads, d_q, q_stride, d_lengths,
                     max_length, d_block_tables, max_pages, scale, d_out, out_stride, d_lse, d_workspace, ws_bytes,
                     d_err, stream);
}

int pallas_attend_quant(const pallas_quant_pool* pool, int32_t layer, int32_t num_seqs, int32_t n_q_heads,
                        const void* d_q, int64_t q_stride, const int32_t* d_lengths, int32_t max_length,
                        const int32_t* d_block_tables, int32_t max_pages, float scale, void* d_out,
                        int64_t out_stride, float* d_lse, void* d_workspace, size_t ws_bytes, int32_t* d_err,
                        void* stream) {
  const char* what = "attend (8-bit)";
  if (int rc = check_quant_pool(pool, layer, what)) return rc;
  const int64_t rows = plane_rows(pool);
  if (2 * rows * 4 > int64_t(0xFFFFFF00))   // addressed with 32-bit offsets
    return fail(PALLAS_ERR_UNSUPPORTED, "%s: a layer's scales of %lld bytes exceed 4 GiB", what, (long long)(2 * rows * 4));
  pallas::AttendParams p{};
  p.k = static_cast<const uint8_t*>(pool->codes) + 2 * layer * rows * pool->head_dim;
  p.v = static_cast<const uint8_t*>(pool->codes) + (2 * layer + 1) * rows * pool->head_dim;
  p.scales = pool->scales + 2 * layer * rows;
  p.num_pages = pool->num_pages;
  p.Hkv = pool->n_kv_heads;
  p.d = pool->head_dim;
  return attend_call(what, pool->format == PALLAS_QUANT_INT8 ? pallas::kCacheInt8 : pallas::kCacheE4m3, p,
                     pool->page_size, num_seqs, n_q_heads, d_q, q_stride, d_lengths, max_length, d_block_tables,
                     max_pages, scale, d_out, out_stride, d_lse, d_workspace, ws_bytes, d_err, stream);
}

size_t pallas_attend_workspace_size(int32_t num_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                    int32_t max_length) {
  if (check_attend(num_seqs, n_q_heads, n_kv_heads, head_dim, max_length, "attend workspace") != PALLAS_OK) return 0;
  return attend_space(num_seqs, n_q_heads, head_dim, max_length, most_ranges(n_q_heads, n_kv_heads, head_dim)).bytes;
}

}  // extern "C"
