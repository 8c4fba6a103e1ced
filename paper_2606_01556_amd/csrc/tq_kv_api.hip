// C ABI of the operators between the linear layers: argument checks on the
// host, then the launches on the caller's stream.  No allocation, no state.
#include <stdint.h>

#include <cmath>

#include "tq.h"
#include "tq_kv.hpp"

namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned(const void *p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline bool dtype_ok(int t) { return t == TQ_F16 || t == TQ_BF16; }
inline bool head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }

// sizes and types of a cache, its pointers, and its kernel form
tq_status check_cache(const tq_kv_cache *c, tq::KvCache &out) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr) return TQ_ERR_NULL;
  const int p = c->page_size;
  if (!head_dim_ok(c->head_dim) || !(c->bits == 16 || c->bits == 8 || c->bits == 4) || p < 16 || p > 32768 ||
      (p & (p - 1)) != 0 || c->pages < 1 || (int64_t)c->pages * p > ((int64_t)1 << 40) || c->kv_heads < 1 ||
      c->kv_heads > 1024)
    return TQ_ERR_BUFFER;
  if (!dtype_ok(c->dtype)) return TQ_ERR_DTYPE;
  if (c->bits != 16 && (c->k_scales == nullptr || c->v_scales == nullptr)) return TQ_ERR_NULL;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_scales) || !aligned16(c->v_scales))
    return TQ_ERR_ALIGN;
  out.k = static_cast<uint8_t *>(c->k);
  out.v = static_cast<uint8_t *>(c->v);
  out.ks = static_cast<uint16_t *>(c->k_scales);
  out.vs = static_cast<uint16_t *>(c->v_scales);
  out.pages = c->pages;
  out.lps = __builtin_ctz((unsigned)p);
  out.heads = c->kv_heads;
  out.d = c->head_dim;
  out.bits = c->bits;
  return TQ_OK;
}

tq_status check_rows(const tq_head_rows *r, tq::HeadRows &out) {
  if (r == nullptr || r->data == nullptr) return TQ_ERR_NULL;
  if (!aligned16(r->data) || (r->token_stride & 7) != 0 || (r->head_stride & 7) != 0) return TQ_ERR_ALIGN;
  out.p = static_cast<const uint16_t *>(r->data);
  out.ts = r->token_stride;
  out.hs = r->head_stride;
  return TQ_OK;
}

tq_status check_norm_rope(const tq_norm_rope *p, int head_dim, tq::TokenArgs &a) {
  if (p == nullptr) return TQ_ERR_NULL;
  if (p->rotary_dim < 0 || p->rotary_dim > head_dim || p->rotary_dim % 16 != 0) return TQ_ERR_SHAPE;
  if (p->rotary_dim > 0) {
    if (p->positions == nullptr || p->table == nullptr) return TQ_ERR_NULL;
    if (p->max_positions < 1) return TQ_ERR_SHAPE;
    if (!aligned(p->positions, 4) || !aligned16(p->table)) return TQ_ERR_ALIGN;
  }
  if (!aligned16(p->q_weight) || !aligned16(p->k_weight)) return TQ_ERR_ALIGN;
  if (!(p->eps >= 0.0f) || std::isinf(p->eps)) return TQ_ERR_SHAPE;
  a.qw = static_cast<const uint16_t *>(p->q_weight);
  a.kw = static_cast<const uint16_t *>(p->k_weight);
  a.eps = p->eps;
  a.positions = p->positions;
  a.table = p->table;
  a.rot = p->rotary_dim;
  a.max_pos = p->max_positions;
  a.interleaved = p->interleaved != 0;
  return TQ_OK;
}

// The kernels number the rows of a call in 31 bits, and a launch its lanes (16 values
// each, in work-groups of 256) in 32.
inline bool rows_ok(int tokens, int64_t per_token, int d) {
  const int64_t rows = (int64_t)tokens * per_token;
  return rows < ((int64_t)1 << 31) && rows * (d / 16) <= ((int64_t)1 << 32) - 256;
}

tq_status hip_status(hipError_t e) { return e == hipSuccess ? TQ_OK : TQ_ERR_HIP; }

#define TQ_TRY(expr)                       \
  do {                                     \
    const tq_status st_ = (expr);          \
    if (st_ != TQ_OK) return st_;          \
  } while (0)

}  // namespace

extern "C" {

tq_status tq_qk_norm_rope(const tq_norm_rope *p, const tq_head_rows *q, const tq_head_rows *k, int tokens,
                          int q_heads, int kv_heads, int head_dim, tq_dtype dtype, void *q_out, void *k_out,
                          void *stream) {
  tq::TokenArgs a = {};
  if (q_out == nullptr || k_out == nullptr) return TQ_ERR_NULL;
  TQ_TRY(check_rows(q, a.q));
  TQ_TRY(check_rows(k, a.k));
  if (!head_dim_ok(head_dim) || tokens < 0 || q_heads < 1 || kv_heads < 1 || q_heads > 65535 || kv_heads > 1024 ||
      !rows_ok(tokens, (int64_t)q_heads + kv_heads, head_dim))
    return TQ_ERR_SHAPE;
  if (!dtype_ok(dtype)) return TQ_ERR_DTYPE;
  TQ_TRY(check_norm_rope(p, head_dim, a));
  if (!aligned16(q_out) || !aligned16(k_out)) return TQ_ERR_ALIGN;
  if (tokens == 0) return TQ_OK;
  a.tokens = tokens; a.hq = q_heads; a.hkv = kv_heads;
  a.rows_per_token = q_heads + kv_heads;
  a.q_out = static_cast<uint16_t *>(q_out);
  a.k_out = static_cast<uint16_t *>(k_out);
  a.c.d = head_dim;
  return hip_status(tq::launch_tokens(a, dtype == TQ_BF16, static_cast<hipStream_t>(stream)));
}

tq_status tq_kv_append(const tq_kv_cache *c, const tq_head_rows *k, const tq_head_rows *v,
                       const int64_t *slots, int tokens, tq_dtype dtype, void *stream) {
  tq::TokenArgs a = {};
  if (slots == nullptr) return TQ_ERR_NULL;
  TQ_TRY(check_cache(c, a.c));
  TQ_TRY(check_rows(k, a.k));
  TQ_TRY(check_rows(v, a.v));
  if (tokens < 0 || !rows_ok(tokens, 2 * (int64_t)c->kv_heads, c->head_dim)) return TQ_ERR_SHAPE;
  if (!dtype_ok(dtype) || (c->bits == 16 && dtype != c->dtype)) return TQ_ERR_DTYPE;
  if (!aligned(slots, 8)) return TQ_ERR_ALIGN;
  if (tokens == 0) return TQ_OK;
  a.tokens = tokens; a.hkv = c->kv_heads;
  a.rows_per_token = 2 * c->kv_heads;
  a.slots = slots;
  return hip_status(tq::launch_tokens(a, dtype == TQ_BF16, static_cast<hipStream_t>(stream)));
}

tq_status tq_qk_norm_rope_append(const tq_norm_rope *p, const tq_kv_cache *c, const tq_head_rows *q,
                                 const tq_head_rows *k, const tq_head_rows *v, const int64_t *slots,
                                 int tokens, int q_heads, tq_dtype dtype, void *q_out, void *k_out,
                                 void *stream) {
  tq::TokenArgs a = {};
  if (slots == nullptr || q_out == nullptr) return TQ_ERR_NULL;
  TQ_TRY(check_cache(c, a.c));
  TQ_TRY(check_rows(q, a.q));
  TQ_TRY(check_rows(k, a.k));
  TQ_TRY(check_rows(v, a.v));
  if (tokens < 0 || q_heads < 1 || q_heads > 65535 || !rows_ok(tokens, q_heads + 2 * (int64_t)c->kv_heads, c->head_dim))
    return TQ_ERR_SHAPE;
  if (!dtype_ok(dtype) || (c->bits == 16 && dtype != c->dtype)) return TQ_ERR_DTYPE;
  TQ_TRY(check_norm_rope(p, c->head_dim, a));
  if (!aligned(slots, 8) || !aligned16(q_out) || !aligned16(k_out)) return TQ_ERR_ALIGN;
  if (tokens == 0) return TQ_OK;
  a.tokens = tokens; a.hq = q_heads; a.hkv = c->kv_heads;
  a.rows_per_token = q_heads + 2 * c->kv_heads;
  a.q_out = static_cast<uint16_t *>(q_out);
  a.k_out = static_cast<uint16_t *>(k_out);
  a.slots = slots;
  return hip_status(tq::launch_tokens(a, dtype == TQ_BF16, static_cast<hipStream_t>(stream)));
}

tq_status tq_kv_read(const tq_kv_cache *c, const int64_t *slots, int tokens, void *k_out, void *v_out,
                     tq_dtype dtype, void *stream) {
  tq::ReadArgs a = {};
  if (slots == nullptr || k_out == nullptr || v_out == nullptr) return TQ_ERR_NULL;
  TQ_TRY(check_cache(c, a.c));
  if (tokens < 0 || !rows_ok(tokens, 2 * (int64_t)c->kv_heads, c->head_dim)) return TQ_ERR_SHAPE;
  if (!dtype_ok(dtype) || (c->bits == 16 && dtype != c->dtype)) return TQ_ERR_DTYPE;
  if (!aligned(slots, 8) || !aligned16(k_out) || !aligned16(v_out)) return TQ_ERR_ALIGN;
  if (tokens == 0) return TQ_OK;
  a.slots = slots;
  a.tokens = tokens;
  a.k_out = static_cast<uint16_t *>(k_out);
  a.v_out = static_cast<uint16_t *>(v_out);
  return hip_status(tq::launch_kv_read(a, dtype == TQ_BF16, static_cast<hipStream_t>(stream)));
}

static tq_status attention_plan(const tq_kv_cache *c, const tq::KvCache &k, int batch, int q_heads, int max_pages,
                                int window, tq::AttendPlan &p) {
  if (batch < 0 || batch > 65535 || q_heads < 1 || q_heads > 65535 || q_heads % c->kv_heads != 0 || max_pages < 1 ||
      (int64_t)max_pages * c->page_size > ((int64_t)1 << 30) || window < 0)
    return TQ_ERR_SHAPE;
  p = tq::attend_plan(k, batch, q_heads, (int64_t)max_pages * c->page_size, window);
  // (the kernel numbers the steps of all streams and heads in 31 bits)
  return p.steps < ((int64_t)1 << 31) - ((int64_t)1 << 16) ? TQ_OK : TQ_ERR_SHAPE;
}

size_t tq_paged_attention_scratch_bytes(const tq_kv_cache *c, int batch, int q_heads, int max_pages, int window) {
  tq::KvCache k;
  tq::AttendPlan p;
  if (check_cache(c, k) != TQ_OK || attention_plan(c, k, batch, q_heads, max_pages, window, p) != TQ_OK) return 0;
  return p.scratch;
}

// the scores of a call
static tq_status check_scores(const tq_scores *s) {
  if (s == nullptr) return TQ_ERR_NULL;
  if (!std::isfinite(s->scale) || !std::isfinite(s->softcap) || s->softcap < 0.0f || s->window < 0) return TQ_ERR_SHAPE;
  if (!aligned(s->slopes, 4)) return TQ_ERR_ALIGN;
  return TQ_OK;
}

static tq_status attend(const tq_kv_cache *c, const tq_head_rows *q, tq_dtype dtype, int batch, int q_heads,
                        const int32_t *page_table, int64_t table_stride, int max_pages, const int32_t *lengths,
                        const tq_scores *scores, void *out, float *lse, void *scratch, void *stream) {
  tq::AttendArgs a = {};
  if (page_table == nullptr || lengths == nullptr || out == nullptr) return TQ_ERR_NULL;
  TQ_TRY(check_cache(c, a.c));
  tq::HeadRows rows;
  TQ_TRY(check_rows(q, rows));
  TQ_TRY(check_scores(scores));
  tq::AttendPlan p;
  TQ_TRY(attention_plan(c, a.c, batch, q_heads, max_pages, scores->window, p));
  if (table_stride < 0) return TQ_ERR_SHAPE;
  if (!dtype_ok(dtype) || (c->bits == 16 && dtype != c->dtype)) return TQ_ERR_DTYPE;
  if (!aligned(page_table, 4) || !aligned(lengths, 4) || !aligned16(out) || !aligned(lse, 4) || !aligned16(scratch))
    return TQ_ERR_ALIGN;
  if (batch == 0) return TQ_OK;
  if (p.scratch != 0 && scratch == nullptr) return TQ_ERR_NULL;
  a.q = rows.p; a.q_ts = rows.ts; a.q_hs = rows.hs;
  a.batch = batch; a.hq = q_heads; a.group = q_heads / c->kv_heads;
  a.table = page_table; a.table_stride = table_stride; a.max_pages = max_pages;
  a.lengths = lengths;
  a.scale = scores->scale; a.window = scores->window; a.cap = scores->softcap; a.slopes = scores->slopes;
  a.out = static_cast<uint16_t *>(out);
  a.lse = lse;
  a.scratch = static_cast<float *>(scratch);
  a.direct = p.direct;
  a.blocks = p.blocks;
  return hip_status(tq::launch_attend(a, dtype == TQ_BF16, static_cast<hipStream_t>(stream)));
}

tq_status tq_paged_attention(const tq_kv_cache *c, const tq_head_rows *q, tq_dtype dtype, int batch,
                             int q_heads, const int32_t *page_table, int64_t table_stride, int max_pages,
                             const int32_t *lengths, float scale, int window, void *out, float *lse,
                             void *scratch, void *stream) {
  const tq_scores scores = {scale, 0.0f, nullptr, window, 1};
  return attend(c, q, dtype, batch, q_heads, page_table, table_stride, max_pages, lengths, &scores, out, lse, scratch, stream);
}

tq_status tq_paged_attention_scored(const tq_kv_cache *c, const tq_head_rows *q, tq_dtype dtype, int batch, int q_heads,
                                    const int32_t *page_table, int64_t table_stride, int max_pages, const int32_t *lengths,
                                    const tq_scores *scores, void *out, float *lse, void *scratch, void *stream) {
  return attend(c, q, dtype, batch, q_heads, page_table, table_stride, max_pages, lengths, scores, out, lse, scratch, stream);
}

static tq_status plan_prompt(const tq_kv_cache *c, const tq::KvCache &k, int tokens, int batch, int q_heads, int max_pages,
                             int window, bool shared, tq::PromptPlan &p) {
  if (tokens < 0 || batch < 0 || batch > 65535 || (batch == 0 && tokens > 0) || q_heads < 1 || q_heads > 65535 ||
      q_heads % c->kv_heads != 0 || max_pages < 1 || (int64_t)max_pages * c->page_size > ((int64_t)1 << 30) || window < 0 ||
      (int64_t)tokens * q_heads >= ((int64_t)1 << 31))
    return TQ_ERR_SHAPE;
  p = tq::prompt_plan(k, tokens, batch, q_heads, (int64_t)max_pages * c->page_size, window, shared);
  // (a launch numbers its lanes in 32 bits)
  return p.blocks < ((int64_t)1 << 24) ? TQ_OK : TQ_ERR_SHAPE;
}

size_t tq_prompt_attention_scratch_bytes(const tq_kv_cache *c, int tokens, int batch, int q_heads, int max_pages, int window) {
  tq::KvCache k;
  tq::PromptPlan p;
  if (check_cache(c, k) != TQ_OK || plan_prompt(c, k, tokens, batch, q_heads, max_pages, window, false, p) != TQ_OK) return 0;
  return p.scratch;
}

tq_status tq_prompt_attention(const tq_kv_cache *c, const tq_head_rows *q, tq_dtype dtype, int tokens, int batch, int q_heads,
                              const int32_t *starts, const int32_t *page_table, int64_t table_stride, int max_pages,
                              const int32_t *lengths, const int32_t *prefix, const int32_t *first, const tq_scores *scores,
                              void *out, float *lse, void *scratch, void *stream) {
  tq::PromptArgs a = {};
  if (starts == nullptr || page_table == nullptr || lengths == nullptr || out == nullptr) return TQ_ERR_NULL;
  TQ_TRY(check_cache(c, a.c));
  tq::HeadRows rows;
  TQ_TRY(check_rows(q, rows));
  TQ_TRY(check_scores(scores));
  tq::PromptPlan p;
  TQ_TRY(plan_prompt(c, a.c, tokens, batch, q_heads, max_pages, scores->window, false, p));
  if (table_stride < 0) return TQ_ERR_SHAPE;
  if (!dtype_ok(dtype) || (c->bits == 16 && dtype != c->dtype)) return TQ_ERR_DTYPE;
  if (!aligned(starts, 4) || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(prefix, 4) || !aligned(first, 4) ||
      !aligned16(out) || !aligned(lse, 4) || !aligned16(scratch))
    return TQ_ERR_ALIGN;
  if (tokens == 0) return TQ_OK;
  if (p.scratch != 0 && scratch == nullptr) return TQ_ERR_NULL;
  a.q = rows.p; a.q_ts = rows.ts; a.q_hs = rows.hs;
  a.tokens = tokens; a.hq = q_heads; a.group = q_heads / c->kv_heads; a.batch = batch;
  a.starts = starts;
  a.table = page_table; a.table_stride = table_stride; a.max_pages = max_pages;
  a.lengths = lengths; a.prefix = prefix; a.first = first;
  a.scale = scores->scale; a.cap = scores->softcap; a.slopes = scores->slopes; a.window = scores->window;
  a.fine = scores->exact != 0;
  a.out = static_cast<uint16_t *>(out);
  a.lse = lse;
  a.scratch = static_cast<float *>(scratch);
  a.tiles = p.tiles; a.splits = p.splits; a.blocks = p.blocks; a.room = p.room; a.longest = p.longest;
  return hip_status(tq::launch_prompt(a, dtype == TQ_BF16, static_cast<hipStream_t>(stream)));
}

// both halves of a call, and where the second one's parts begin in scratch
static tq_status plan_prefix(const tq_kv_cache *c, const tq::KvCache &k, int batch, int q_heads, int groups, int prefix_pages,
                             int max_pages, tq::PromptPlan &p, tq::AttendPlan &t, size_t &first, size_t &bytes) {
  // (the join's launch numbers its lanes in 32 bits, up to 64 of them a row)
  if (groups < 1 || groups > 65535 || batch < 0 || (int64_t)batch * q_heads > ((int64_t)1 << 25)) return TQ_ERR_SHAPE;
  TQ_TRY(attention_plan(c, k, batch, q_heads, max_pages, 0, t));
  TQ_TRY(plan_prompt(c, k, batch, groups, q_heads, prefix_pages, 0, true, p));
  first = (p.scratch + 255) & ~(size_t)255;
  bytes = batch == 0 ? 0 : first + tq::attend_parts_bytes(k, batch, q_heads, t);
  return TQ_OK;
}

size_t tq_shared_prefix_attention_scratch_bytes(const tq_kv_cache *c, int batch, int q_heads, int groups, int prefix_pages,
                                                int max_pages) {
  tq::KvCache k;
  tq::PromptPlan p;
  tq::AttendPlan t;
  size_t first, bytes;
  if (check_cache(c, k) != TQ_OK || plan_prefix(c, k, batch, q_heads, groups, prefix_pages, max_pages, p, t, first, bytes) != TQ_OK)
    return 0;
  return bytes;
}

tq_status tq_shared_prefix_attention(const tq_kv_cache *c, const tq_head_rows *q, tq_dtype dtype, int batch, int q_heads,
                                     int groups, const int32_t *members, const int32_t *prefix_table, int64_t prefix_stride,
                                     int prefix_pages, const int32_t *prefix_lengths, const int32_t *page_table,
                                     int64_t table_stride, int max_pages, const int32_t *lengths, const tq_scores *scores,
                                     void *out, float *lse, void *scratch, void *stream) {
  tq::PrefixArgs a = {};
  if (members == nullptr || prefix_table == nullptr || prefix_lengths == nullptr || page_table == nullptr ||
      lengths == nullptr || out == nullptr)
    return TQ_ERR_NULL;
  tq::KvCache k;
  TQ_TRY(check_cache(c, k));
  tq::HeadRows rows;
  TQ_TRY(check_rows(q, rows));
  TQ_TRY(check_scores(scores));
  tq::PromptPlan p;
  tq::AttendPlan t;
  size_t first, bytes;
  TQ_TRY(plan_prefix(c, k, batch, q_heads, groups, prefix_pages, max_pages, p, t, first, bytes));
  if (prefix_stride < 0 || table_stride < 0 || scores->window != 0) return TQ_ERR_SHAPE;
  if (!dtype_ok(dtype) || (c->bits == 16 && dtype != c->dtype)) return TQ_ERR_DTYPE;
  if (!aligned(members, 4) || !aligned(prefix_table, 4) || !aligned(prefix_lengths, 4) || !aligned(page_table, 4) ||
      !aligned(lengths, 4) || !aligned16(out) || !aligned(lse, 4) || !aligned16(scratch))
    return TQ_ERR_ALIGN;
  if (batch == 0) return TQ_OK;
  if (scratch == nullptr) return TQ_ERR_NULL;
  tq::PromptArgs &x = a.prefix;
  x.c = k;
  x.q = rows.p; x.q_ts = rows.ts; x.q_hs = rows.hs;
  x.tokens = batch; x.hq = q_heads; x.group = q_heads / c->kv_heads; x.batch = groups;
  x.starts = members;
  x.table = prefix_table; x.table_stride = prefix_stride; x.max_pages = prefix_pages;
  x.lengths = prefix_lengths; x.own = lengths; x.own_most = max_pages * c->page_size;
  x.scale = scores->scale; x.cap = scores->softcap; x.slopes = scores->slopes;
  x.shared = true;
  x.fine = scores->exact != 0;
  x.out = static_cast<uint16_t *>(out);
  x.lse = lse;
  x.scratch = static_cast<float *>(scratch);
  x.tiles = p.tiles; x.splits = p.splits; x.blocks = p.blocks; x.room = p.room; x.longest = p.longest;
  tq::AttendArgs &y = a.own;
  y.c = k;
  y.q = rows.p; y.q_ts = rows.ts; y.q_hs = rows.hs;
  y.batch = batch; y.hq = q_heads; y.group = x.group;
  y.table = page_table; y.table_stride = table_stride; y.max_pages = max_pages;
  y.lengths = lengths;
  y.scale = x.scale; y.cap = x.cap; y.slopes = x.slopes;
  y.parts = true;
  y.scratch = reinterpret_cast<float *>(static_cast<uint8_t *>(scratch) + first);
  y.direct = t.direct;
  y.blocks = t.blocks;
  return hip_status(tq::launch_prefix(a, dtype == TQ_BF16, static_cast<hipStream_t>(stream)));
}

tq_status tq_add_rms_norm(const tq_residual_norm *p, int tokens, int n, tq_dtype dtype, void *sum, void *normed, void *stream) {
  if (p == nullptr || p->x == nullptr || (sum == nullptr && normed == nullptr) || (normed != nullptr && p->weight == nullptr))
    return TQ_ERR_NULL;
  if (tokens < 0 || n < 8 || n > tq::kNormMost || n % 8 != 0) return TQ_ERR_SHAPE;
  if (!(p->eps >= 0.0f) || std::isinf(p->eps) || !std::isfinite(p->scale)) return TQ_ERR_SHAPE;
  if (!dtype_ok(dtype)) return TQ_ERR_DTYPE;
  if (((p->x_stride | p->residual_stride | p->gate_stride) & 7) != 0) return TQ_ERR_ALIGN;
  for (const void *at : {p->x, p->residual, p->gate, p->post_weight, p->weight, (const void *)sum, (const void *)normed})
    if (!aligned16(at)) return TQ_ERR_ALIGN;
  if (tokens == 0) return TQ_OK;
  tq::NormArgs a = {};
  a.x = static_cast<const uint16_t *>(p->x); a.x_stride = p->x_stride;
  a.residual = static_cast<const uint16_t *>(p->residual); a.r_stride = p->residual_stride;
  a.gate = static_cast<const uint16_t *>(p->gate); a.g_stride = p->gate_stride;
  a.post = static_cast<const uint16_t *>(p->post_weight);
  a.weight = static_cast<const uint16_t *>(p->weight);
  a.scale = p->scale; a.eps = p->eps;
  a.tokens = tokens; a.n = n;
  a.sum = static_cast<uint16_t *>(sum);
  a.normed = static_cast<uint16_t *>(normed);
  // (a launch numbers its lanes in 32 bits: rows of up to 1024 lanes go in runs)
  const int most = 1 << 21;
  for (int done = 0; done < tokens; done += most) {
    tq::NormArgs b = a;
    b.tokens = tokens - done < most ? tokens - done : most;
    b.x += done * a.x_stride;
    if (a.residual != nullptr) b.residual += done * a.r_stride;
    if (a.gate != nullptr) b.gate += done * a.g_stride;
    if (a.sum != nullptr) b.sum += (int64_t)done * n;
    if (a.normed != nullptr) b.normed += (int64_t)done * n;
    const tq_status st = hip_status(tq::launch_norm(b, dtype == TQ_BF16, static_cast<hipStream_t>(stream)));
    if (st != TQ_OK) return st;
    if (tokens - done <= most) break;
  }
  return TQ_OK;
}

}  // extern "C"
