// C entry points of the operators on ragged batches and 8-bit pages (see include/keyformer.h): arguments are checked here, on the host,
// before anything is enqueued.
#include "keyformer.h"

#include <algorithm>
#include <cmath>

#include "kf_args.cuh"
#include "kf_pages.cuh"

namespace {

using namespace kf::args;

constexpr int64_t STRIDE_MAX = (int64_t)1 << 38;      // elements: tensor maps hold strides below 2^40 bytes
constexpr int32_t ROWS_MAX = 1 << 28, SEQUENCES_MAX = 1 << 20;

inline bool type16(int32_t type) { return type == KF_TYPE_FP16 || type == KF_TYPE_BF16; }
inline bool stride_ok(int64_t s, int d) { return s >= d && s % 8 == 0 && s < STRIDE_MAX; }
// Bytes from the first to behind the last row of [a][b] rows of d 16-bit values.
inline uint64_t extent(int64_t a, int64_t stride_a, int64_t b, int64_t stride_b, int d) {
  return ((uint64_t)(a - 1) * stride_a + (uint64_t)(b - 1) * stride_b + d) * 2;
}
// Whether [a][b] rows of d values lie apart from one another.
inline bool apart(int64_t a, int64_t stride_a, int64_t b, int64_t stride_b, int d) {
  if (a == 1 || b == 1) return true;                  // each stride is at least d
  return stride_a >= (b - 1) * stride_b + d || stride_b >= (a - 1) * stride_a + d;
}
inline bool bias_ok(int32_t mode, const float* slopes) {
  return mode == KF_BIAS_NONE || (mode == KF_BIAS_ALIBI && slopes && !misaligned(slopes, 4));
}

bool ragged_ok(const kf_ragged_args* a) {
  if (!a || a->tokens < 1 || a->tokens > ROWS_MAX || a->sequences < 1 || a->sequences > SEQUENCES_MAX) return false;
  if (a->n_heads < 1 || a->n_heads > 65535 || a->n_kv_heads < 1 || a->n_heads % a->n_kv_heads != 0 || !head_dim_ok(a->head_dim) || !type16(a->type)) return false;
  if (((int64_t)a->tokens / 128 + a->sequences) * a->n_heads > INT32_MAX) return false;
  if (!(a->logit_scale >= 0.f) || !std::isfinite(a->logit_scale) || !bias_ok(a->bias_mode, a->d_alibi_slopes)) return false;
  if (a->debug_fail_first_wait < 0 || a->debug_fail_first_wait > 1) return false;
  for (int64_t s : {a->q_token_stride, a->q_head_stride, a->k_token_stride, a->k_head_stride, a->v_token_stride, a->v_head_stride, a->out_token_stride,
                    a->out_head_stride})
    if (!stride_ok(s, a->head_dim)) return false;
  return apart(a->tokens, a->out_token_stride, a->n_heads, a->out_head_stride, a->head_dim);
}

bool cache_ok(const kf_page_cache* c) {
  if (!c || c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535 || !head_dim_ok(c->head_dim)) return false;
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return false;
  if (c->sequences < 1 || c->sequences > SEQUENCES_MAX || c->table_width < 1) return false;
  if ((int64_t)c->table_width * c->page_tokens >= (int64_t)1 << 30) return false;
  return (int64_t)c->n_pages <= (((int64_t)1 << 31) - 1) / 2 / c->page_tokens / c->n_kv_heads;
}
inline uint64_t cache_bytes(const kf_page_cache& c) { return (uint64_t)c.n_pages * c.n_kv_heads * 2 * c.page_tokens * c.head_dim; }
inline uint64_t scale_bytes(const kf_page_cache& c) { return (uint64_t)c.n_pages * c.n_kv_heads * 8; }
inline uint64_t table_bytes(const kf_page_cache& c) { return (uint64_t)c.sequences * c.table_width * 4; }

bool rows_ok(const kf_page_cache& c, const kf_page_rows* r, const int32_t* d_begin) {
  if (!r || r->tokens < 1 || r->tokens > ROWS_MAX || !type16(r->type)) return false;
  if (!d_begin && r->tokens != c.sequences) return false;
  for (int64_t s : {r->k_token_stride, r->k_head_stride, r->v_token_stride, r->v_head_stride})
    if (!stride_ok(s, c.head_dim)) return false;
  return true;
}

kf::PageCache cache_of(const kf_page_cache& c, void* d_cache, float* d_scale) {
  return {static_cast<signed char*>(d_cache), d_scale, c.n_pages, c.page_tokens, c.n_kv_heads, c.head_dim, c.sequences, c.table_width};
}
kf::PageRows page_rows(const kf_page_rows& r, const void* d_k, const void* d_v) {
  return {const_cast<void*>(d_k), const_cast<void*>(d_v), r.k_token_stride, r.k_head_stride, r.v_token_stride, r.v_head_stride, r.tokens, r.type == KF_TYPE_BF16};
}

bool attend_ok(const kf_pages_attend_args* a) {
  if (!a || !cache_ok(&a->cache) || a->n_heads < 1 || a->n_heads > 65535 || a->n_heads % a->cache.n_kv_heads != 0 || !type16(a->type)) return false;
  if (!(a->logit_scale >= 0.f) || !std::isfinite(a->logit_scale) || !bias_ok(a->bias_mode, a->d_alibi_slopes)) return false;
  if (a->debug_fail_first_wait < 0 || a->debug_fail_first_wait > 1 || (a->debug_fail_first_wait && a->debug_fail_after < 0)) return false;
  for (int64_t s : {a->q_sequence_stride, a->q_head_stride, a->out_sequence_stride, a->out_head_stride})
    if (!stride_ok(s, a->cache.head_dim)) return false;
  if (!kf::pages_attend_fits(cache_of(a->cache, nullptr, nullptr), a->n_heads)) return false;
  return apart(a->cache.sequences, a->out_sequence_stride, a->n_heads, a->out_head_stride, a->cache.head_dim);
}
struct AttendLayout { size_t partials, total; };
AttendLayout attend_layout(const kf_pages_attend_args* a) {
  const kf_page_cache& c = a->cache;
  const size_t splits = align_up((size_t)kf::pages_attend_shares(cache_of(c, nullptr, nullptr), a->n_heads) * 32);
  return {splits, splits + align_up(kf::pages_attend_partials(cache_of(c, nullptr, nullptr), a->n_heads) * 4)};
}

bool update_ok(const kf_pages_update_args* a) {
  if (!a || !cache_ok(&a->cache) || a->cache.sequences > kf::UPDATE_MAX_SEQUENCES || a->n_layers < 1 || a->n_layers > 65535) return false;
  if ((int64_t)a->cache.sequences * a->cache.table_width > (int64_t)1 << 28) return false;
  return true;
}
struct UpdateLayout { size_t list, copies, total; };
UpdateLayout update_layout(const kf_pages_update_args* a) {
  const size_t entries = (size_t)a->cache.sequences * a->cache.table_width, pages = (size_t)a->cache.n_pages;
  UpdateLayout L{};
  L.list = align_up(entries * 4);
  L.copies = L.list + align_up((entries < pages ? entries : pages) * 4);
  L.total = L.copies + align_up((size_t)a->cache.sequences * 16);
  return L;
}

inline int status(cudaError_t e) { return e == cudaSuccess ? KF_OK : (e == cudaErrorInvalidValue ? KF_EINVAL : KF_ECUDA); }

}  // namespace

extern "C" {

int kf_prefill_attend_ragged(const kf_ragged_args* a, const void* d_q, const void* d_k, const void* d_v, const int32_t* d_begin, void* d_out, void* stream) {
  if (!ragged_ok(a) || !d_q || !d_k || !d_v || !d_begin || !d_out) return KF_EINVAL;
  for (const void* p : {d_q, d_k, d_v, static_cast<const void*>(d_out)})
    if (misaligned(p, 16)) return KF_EINVAL;
  if (misaligned(d_begin, 4)) return KF_EINVAL;
  const int d = a->head_dim;
  const bool alibi = a->bias_mode == KF_BIAS_ALIBI;
  if (conflict({rows_of(d_out, a->tokens, a->out_token_stride, a->n_heads, a->out_head_stride, d)},
               {rows_of(d_q, a->tokens, a->q_token_stride, a->n_heads, a->q_head_stride, d),
                rows_of(d_k, a->tokens, a->k_token_stride, a->n_kv_heads, a->k_head_stride, d),
                rows_of(d_v, a->tokens, a->v_token_stride, a->n_kv_heads, a->v_head_stride, d),
                {d_begin, ((uint64_t)a->sequences + 1) * 4},
                {alibi ? a->d_alibi_slopes : nullptr, (uint64_t)a->n_heads * 4}}))
    return KF_EINVAL;
  kf::RaggedArgs r{};
  r.q = d_q; r.k = d_k; r.v = d_v; r.out = d_out; r.begin = d_begin;
  r.slopes = alibi ? a->d_alibi_slopes : nullptr;
  r.q_token = a->q_token_stride; r.q_head = a->q_head_stride;
  r.k_token = a->k_token_stride; r.k_head = a->k_head_stride;
  r.v_token = a->v_token_stride; r.v_head = a->v_head_stride;
  r.out_token = a->out_token_stride; r.out_head = a->out_head_stride;
  r.tokens = a->tokens; r.sequences = a->sequences; r.H = a->n_heads; r.Hkv = a->n_kv_heads; r.head_dim = d;
  r.bf16 = a->type == KF_TYPE_BF16;
  const bool fails = a->debug_fail_first_wait != 0;
  r.fail_item = fails && a->debug_fail_after >= 0 ? a->debug_fail_after : -1;
  r.leave_item = fails && a->debug_fail_after < 0 ? -1 - a->debug_fail_after : -1;
  r.scale = a->logit_scale > 0.f ? a->logit_scale : (float)(1.0 / std::sqrt((double)d));
  return status(kf::launch_ragged(r, static_cast<cudaStream_t>(stream)));
}

int kf_pages_write(const kf_page_cache* c, const kf_page_rows* r, const void* d_k, const void* d_v, const int32_t* d_begin, const int32_t* d_length,
                   const int32_t* d_table, void* d_cache, float* d_scale, void* stream) {
  if (!cache_ok(c) || !rows_ok(*c, r, d_begin) || !d_k || !d_v || !d_length || !d_table || !d_cache || !d_scale) return KF_EINVAL;
  if (misaligned(d_k, 16) || misaligned(d_v, 16) || misaligned(d_cache, 16) || misaligned(d_scale, 8)) return KF_EINVAL;
  if (misaligned(d_begin, 4) || misaligned(d_length, 4) || misaligned(d_table, 4)) return KF_EINVAL;
  const uint64_t S = (uint64_t)c->sequences;
  if (conflict({{d_cache, cache_bytes(*c)}, {d_scale, scale_bytes(*c)}},
               {{d_k, extent(r->tokens, r->k_token_stride, c->n_kv_heads, r->k_head_stride, c->head_dim)},
                {d_v, extent(r->tokens, r->v_token_stride, c->n_kv_heads, r->v_head_stride, c->head_dim)},
                {d_begin, (S + 1) * 4}, {d_length, S * 4}, {d_table, table_bytes(*c)}}))
    return KF_EINVAL;
  return status(kf::launch_pages_write(cache_of(*c, d_cache, d_scale), page_rows(*r, d_k, d_v), d_begin, d_length, d_table, static_cast<cudaStream_t>(stream)));
}

int kf_pages_read(const kf_page_cache* c, const kf_page_rows* r, const void* d_cache, const float* d_scale, const int32_t* d_table, const int32_t* d_begin,
                  const int32_t* d_first, void* d_k, void* d_v, void* stream) {
  if (!cache_ok(c) || !rows_ok(*c, r, d_begin) || !d_k || !d_v || !d_begin || !d_table || !d_cache || !d_scale) return KF_EINVAL;
  if (misaligned(d_k, 16) || misaligned(d_v, 16) || misaligned(d_cache, 16) || misaligned(d_scale, 8)) return KF_EINVAL;
  if (misaligned(d_begin, 4) || misaligned(d_first, 4) || misaligned(d_table, 4)) return KF_EINVAL;
  if (!apart(r->tokens, r->k_token_stride, c->n_kv_heads, r->k_head_stride, c->head_dim) ||
      !apart(r->tokens, r->v_token_stride, c->n_kv_heads, r->v_head_stride, c->head_dim))
    return KF_EINVAL;
  const uint64_t S = (uint64_t)c->sequences;
  if (conflict({rows_of(d_k, r->tokens, r->k_token_stride, c->n_kv_heads, r->k_head_stride, c->head_dim),
                rows_of(d_v, r->tokens, r->v_token_stride, c->n_kv_heads, r->v_head_stride, c->head_dim)},
               {{d_cache, cache_bytes(*c)}, {d_scale, scale_bytes(*c)}, {d_begin, (S + 1) * 4}, {d_first, S * 4}, {d_table, table_bytes(*c)}}))
    return KF_EINVAL;
  return status(kf::launch_pages_read(cache_of(*c, const_cast<void*>(d_cache), const_cast<float*>(d_scale)), page_rows(*r, d_k, d_v), d_begin, d_first, d_table,
                                      static_cast<cudaStream_t>(stream)));
}

size_t kf_pages_attend_scratch_bytes(const kf_pages_attend_args* a) { return attend_ok(a) ? attend_layout(a).total : 0; }

int kf_pages_attend(const kf_pages_attend_args* a, const void* d_q, const void* d_cache, const float* d_scale, const int32_t* d_table, const int32_t* d_length,
                    void* d_out, void* d_scratch, size_t scratch_bytes, void* stream) {
  if (!attend_ok(a) || !d_q || !d_cache || !d_scale || !d_table || !d_length || !d_out || !d_scratch) return KF_EINVAL;
  if (misaligned(d_q, 16) || misaligned(d_out, 16) || misaligned(d_cache, 16) || misaligned(d_scale, 8) || misaligned(d_table, 4) || misaligned(d_length, 4) ||
      misaligned(d_scratch, 256))
    return KF_EINVAL;
  const AttendLayout L = attend_layout(a);
  if (scratch_bytes < L.total) return KF_ENOSPC;
  const kf_page_cache& c = a->cache;
  const bool alibi = a->bias_mode == KF_BIAS_ALIBI;
  if (conflict({{d_out, extent(c.sequences, a->out_sequence_stride, a->n_heads, a->out_head_stride, c.head_dim)}, {d_scratch, L.total}},
               {{d_q, extent(c.sequences, a->q_sequence_stride, a->n_heads, a->q_head_stride, c.head_dim)}, {d_cache, cache_bytes(c)}, {d_scale, scale_bytes(c)},
                {d_table, table_bytes(c)}, {d_length, (uint64_t)c.sequences * 4}, {alibi ? a->d_alibi_slopes : nullptr, (uint64_t)a->n_heads * 4}}))
    return KF_EINVAL;
  kf::PagesAttend p{};
  p.c = cache_of(c, const_cast<void*>(d_cache), const_cast<float*>(d_scale));
  p.q = d_q; p.out = d_out; p.table = d_table; p.length = d_length;
  p.slopes = alibi ? a->d_alibi_slopes : nullptr;
  p.q_sequence = a->q_sequence_stride; p.q_head = a->q_head_stride;
  p.out_sequence = a->out_sequence_stride; p.out_head = a->out_head_stride;
  p.H = a->n_heads;
  p.bf16 = a->type == KF_TYPE_BF16;
  p.fail_at = a->debug_fail_first_wait ? 16 * std::min(a->debug_fail_after, 1 << 26) : -1;   // a warp looks up 16 tiles at a time
  p.scale = a->logit_scale > 0.f ? a->logit_scale : (float)(1.0 / std::sqrt((double)c.head_dim));
  p.splits = static_cast<int4*>(d_scratch);
  p.partials = reinterpret_cast<float*>(static_cast<unsigned char*>(d_scratch) + L.partials);
  return status(kf::launch_pages_attend(p, static_cast<cudaStream_t>(stream)));
}

size_t kf_pages_update_scratch_bytes(const kf_pages_update_args* a) { return update_ok(a) ? update_layout(a).total : 0; }

int kf_pages_update(const kf_pages_update_args* a, int32_t* d_table, int32_t* d_length, int32_t* d_refs, const int32_t* d_parent, const int32_t* d_grow,
                    void* d_cache, float* d_scale, int32_t* d_missing, void* d_scratch, size_t scratch_bytes, void* stream) {
  if (!update_ok(a) || !d_table || !d_length || !d_refs || !d_cache || !d_scale || !d_missing || !d_scratch) return KF_EINVAL;
  if (misaligned(d_cache, 16) || misaligned(d_scale, 8) || misaligned(d_scratch, 256)) return KF_EINVAL;
  for (const int32_t* p : {static_cast<const int32_t*>(d_table), static_cast<const int32_t*>(d_length), static_cast<const int32_t*>(d_refs), d_parent, d_grow,
                           static_cast<const int32_t*>(d_missing)})
    if (misaligned(p, 4)) return KF_EINVAL;
  const UpdateLayout L = update_layout(a);
  if (scratch_bytes < L.total) return KF_ENOSPC;
  const kf_page_cache& c = a->cache;
  const uint64_t S = (uint64_t)c.sequences, layers = (uint64_t)a->n_layers;
  if (conflict({{d_table, table_bytes(c)}, {d_length, S * 4}, {d_refs, (uint64_t)c.n_pages * 4}, {d_cache, cache_bytes(c) * layers},
                {d_scale, scale_bytes(c) * layers}, {d_missing, 4}, {d_scratch, L.total}},
               {{d_parent, S * 4}, {d_grow, S * 4}}))
    return KF_EINVAL;
  unsigned char* scratch = static_cast<unsigned char*>(d_scratch);
  kf::PagesUpdate u{};
  u.c = cache_of(c, d_cache, d_scale);
  u.layers = a->n_layers; u.grow_all = a->grow;
  u.table = d_table; u.length = d_length; u.refs = d_refs; u.missing = d_missing;
  u.parent = d_parent; u.grow = d_grow;
  u.stays = static_cast<int32_t*>(d_scratch);
  u.free_list = reinterpret_cast<int32_t*>(scratch + L.list);
  u.copies = reinterpret_cast<int4*>(scratch + L.copies);
  return status(kf::launch_pages_update(u, static_cast<cudaStream_t>(stream)));
}

int kf_pages_compact(const kf_page_cache* c, int32_t keep_width, int32_t new_table_width, const int32_t* d_table, const int32_t* d_length, const int32_t* d_keep,
                     const int32_t* d_n_keep, const int32_t* d_new_table, void* d_cache, float* d_scale, void* stream) {
  if (!cache_ok(c) || keep_width < 1 || new_table_width < 1 || !d_table || !d_length || !d_keep || !d_n_keep || !d_new_table || !d_cache || !d_scale)
    return KF_EINVAL;
  if ((int64_t)new_table_width * c->page_tokens >= (int64_t)1 << 30 || (int64_t)keep_width > (int64_t)new_table_width * c->page_tokens) return KF_EINVAL;
  if ((int64_t)c->sequences * new_table_width > (int64_t)INT32_MAX) return KF_EINVAL;
  if (misaligned(d_cache, 16) || misaligned(d_scale, 8)) return KF_EINVAL;
  for (const int32_t* p : {d_table, d_length, d_keep, d_n_keep, d_new_table})
    if (misaligned(p, 4)) return KF_EINVAL;
  const uint64_t S = (uint64_t)c->sequences;
  if (conflict({{d_cache, cache_bytes(*c)}, {d_scale, scale_bytes(*c)}},
               {{d_table, table_bytes(*c)}, {d_length, S * 4}, {d_keep, S * c->n_kv_heads * keep_width * 4}, {d_n_keep, S * 4}, {d_new_table, S * new_table_width * 4}}))
    return KF_EINVAL;
  return status(kf::launch_pages_compact(cache_of(*c, d_cache, d_scale), keep_width, new_table_width, d_table, d_length, d_keep, d_n_keep, d_new_table,
                                         static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
