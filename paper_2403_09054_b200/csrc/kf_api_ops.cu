// C entry points of the operators that need no context (see include/keyformer.h): arguments are checked here, on the
// host, before anything is enqueued.
#include "keyformer.h"

#include <cmath>
#include <cstring>
#include <initializer_list>

#include "kf_ops.cuh"
#include "kf_packed.cuh"

namespace {

constexpr size_t ALIGN = 256;
inline size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
inline bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
// Whether [a, a + n) and [b, b + m) share a byte.
inline bool overlap(const void* a, uint64_t n, const void* b, uint64_t m) {
  const uint64_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + m && y < x + n;
}
// A tensor of a call.  `rows` > 1: that many rows of `bytes`, `stride` bytes apart; what lies between them is not the call's.
struct Range {
  const void* at;
  uint64_t bytes, rows = 1, stride = 0;
  uint64_t extent() const { return (rows - 1) * stride + bytes; }
};
// Whether one of the rows of `a` shares a byte with the extent of `b`, given that the two extents do.
bool touches(const Range& a, const Range& b) {
  if (a.rows == 1 || a.stride <= a.bytes) return true;
  const uint64_t base = reinterpret_cast<uintptr_t>(a.at), x = reinterpret_cast<uintptr_t>(b.at);
  const uint64_t begin = x > base ? x - base : 0, end = x + b.extent() - base;     // of b, from the first row on
  return begin % a.stride < a.bytes || end > (begin / a.stride + 1) * a.stride;
}
// Whether something that the call writes shares memory with another of its tensors.  Every pair of extents without a branch
// (this runs for every token and layer): two meet where both differences are negative; one that is absent ends before everything.
bool conflict(std::initializer_list<Range> writes, std::initializer_list<Range> reads) {
  constexpr int MOST = 16;
  uint64_t from[MOST], to[MOST];
  int n = 0;
  auto add = [&](const Range& r) {
    from[n] = reinterpret_cast<uintptr_t>(r.at);
    to[n] = r.at ? from[n] + r.extent() : 0;
    ++n;
  };
  for (const Range& r : writes) add(r);
  const int written = n;
  for (const Range& r : reads) add(r);
  uint64_t meet = 0;
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < n; ++j) meet |= (from[j] - to[i]) & (from[i] - to[j]);
  if (meet >> 63 == 0) return false;
  auto range = [&](int i) { return i < written ? writes.begin()[i] : reads.begin()[i - written]; };
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < n; ++j)
      if (from[j] < to[i] && from[i] < to[j] && touches(range(j), range(i))) return true;    // only what is read may have rows
  return false;
}
inline bool head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }

bool rows_ok(int64_t units, int32_t n, int32_t k, int32_t d) {
  if (units < 1 || n < 1 || k < n || !head_dim_ok(d)) return false;
  return units <= ((int64_t)1 << 37) / d / n;   // eight features a thread, 256 threads a block, fewer than 2^31 blocks (and 2^37 features)
}

bool packed_ok(const kf_packed_step* a) {
  if (!a || a->batch < 1 || a->n_heads < 1 || (int64_t)a->batch * a->n_heads > 65535) return false;
  if (a->n_kv_heads < 0 || a->n_kv_heads > a->n_heads) return false;
  const int hkv = a->n_kv_heads > 0 ? a->n_kv_heads : a->n_heads;
  if (a->n_heads % hkv != 0 || !kf::decode_group_supported(a->n_heads / hkv) || !head_dim_ok(a->head_dim)) return false;
  if (a->budget_k < 1 || a->budget_k > (1 << 26) || a->recent_w < 0 || a->recent_w > a->budget_k) return false;
  if (a->layer < 0 || a->position < 0 || !(a->tau > 0.0) || !std::isfinite(a->tau) || !(a->logit_scale >= 0.f)) return false;
  if (a->debug_fail_first_wait < 0 || a->debug_fail_first_wait > 1) return false;
  if (a->noise_mode < KF_NOISE_GUMBEL || a->noise_mode > KF_NOISE_GAUSS) return false;
  if (a->noise_mode == KF_NOISE_GAUSS && !(a->noise_sigma >= 0.f)) return false;
  if (a->bias_mode != KF_BIAS_NONE && a->bias_mode != KF_BIAS_ALIBI) return false;
  return a->bias_mode != KF_BIAS_ALIBI || a->d_alibi_slopes;
}

struct PackedLayout {
  int units, group, splits, tiles_per_split;
  size_t partials, total;   // offsets; the adjusted logits come first
};
PackedLayout packed_layout(const kf_packed_step* a) {
  PackedLayout L{};
  const int hkv = a->n_kv_heads > 0 ? a->n_kv_heads : a->n_heads;
  L.units = a->batch * hkv;
  L.group = a->n_heads / hkv;
  kf::decode_packed_plan(L.units, a->budget_k, a->head_dim, &L.splits, &L.tiles_per_split);
  const size_t units_q = (size_t)L.units * L.group;
  L.partials = align_up(units_q * ((size_t)a->budget_k + 1) * 4);
  L.total = L.partials + align_up(units_q * L.splits * (4 + (size_t)a->head_dim) * 4);
  return L;
}

bool beam_ok(const kf_beam_args* a) {
  if (!a || a->batch < 1 || a->beams < 1 || a->beams > kf::BEAM_MAX || a->vocab < 1) return false;
  if (a->take < 1 || a->take > kf::BEAM_TAKE_MAX || (int64_t)a->take > (int64_t)a->beams * a->vocab) return false;
  if (a->logits_type < KF_TYPE_FP16 || a->logits_type > KF_TYPE_FP32 || a->row_stride < a->vocab) return false;
  if (a->vocab > (1 << 26) || (int64_t)a->batch * a->beams > 65535) return false;
  return a->pad_token >= 0 && a->pad_token < a->vocab;
}

}  // namespace

extern "C" {

int32_t kf_packed_slot_bytes(int32_t head_dim) { return head_dim_ok(head_dim) ? kf::packed_slot_bytes(head_dim) : 0; }

int kf_pack_cache(int64_t units, int32_t n, int32_t budget_k, int32_t head_dim, const void* d_K, const void* d_V,
                  const int32_t* d_len, void* d_cache, void* stream) {
  if (!rows_ok(units, n, budget_k, head_dim) || !d_K || !d_V || !d_cache) return KF_EINVAL;
  if (misaligned(d_K, 16) || misaligned(d_V, 16) || misaligned(d_cache, 16) || misaligned(d_len, 4)) return KF_EINVAL;
  const uint64_t rows = (uint64_t)units * n * head_dim * 2, slots = (uint64_t)units * budget_k * kf::packed_slot_bytes(head_dim);
  if (conflict({{d_cache, slots}},
               {{d_K, rows}, {d_V, rows}, {d_len, (uint64_t)units * 4}})) return KF_EINVAL;
  return kf::launch_pack(static_cast<const __half*>(d_K), static_cast<const __half*>(d_V), d_len, static_cast<unsigned char*>(d_cache), units, n,
                         budget_k, head_dim, static_cast<cudaStream_t>(stream)) == cudaSuccess ? KF_OK : KF_ECUDA;
}

int kf_unpack_cache(int64_t units, int32_t n, int32_t budget_k, int32_t head_dim, const void* d_cache, const int32_t* d_len,
                    void* d_K, void* d_V, void* stream) {
  if (!rows_ok(units, n, budget_k, head_dim) || !d_K || !d_V || !d_cache) return KF_EINVAL;
  if (misaligned(d_K, 16) || misaligned(d_V, 16) || misaligned(d_cache, 16) || misaligned(d_len, 4)) return KF_EINVAL;
  const uint64_t rows = (uint64_t)units * n * head_dim * 2, slots = (uint64_t)units * budget_k * kf::packed_slot_bytes(head_dim);
  if (conflict({{d_K, rows}, {d_V, rows}},
               {{d_len, (uint64_t)units * 4}, {d_cache, slots}})) return KF_EINVAL;
  return kf::launch_unpack(static_cast<const unsigned char*>(d_cache), d_len, static_cast<__half*>(d_K), static_cast<__half*>(d_V), units, n,
                           budget_k, head_dim, static_cast<cudaStream_t>(stream)) == cudaSuccess ? KF_OK : KF_ECUDA;
}

size_t kf_packed_scratch_bytes(const kf_packed_step* args) { return packed_ok(args) ? packed_layout(args).total : 0; }

int kf_decode_step_packed(const kf_packed_step* a, void* d_cache, int32_t* d_pos, float* d_acc, int32_t* d_len,
                          const void* d_q, const void* d_knew, const void* d_vnew, void* d_out, float* d_score_opt,
                          int32_t* d_slot_opt, void* d_row_opt, void* d_scratch, size_t scratch_bytes, void* stream) {
  if (!packed_ok(a) || !d_cache || !d_pos || !d_acc || !d_len || !d_q || !d_knew || !d_vnew || !d_out || !d_scratch) return KF_EINVAL;
  if (misaligned(d_cache, 16) || misaligned(d_q, 16) || misaligned(d_knew, 16) || misaligned(d_vnew, 16) || misaligned(d_out, 16) ||
      misaligned(d_scratch, 256) || misaligned(d_row_opt, 2))
    return KF_EINVAL;
  if (misaligned(d_pos, 4) || misaligned(d_acc, 4) || misaligned(d_len, 4) || misaligned(d_score_opt, 4) || misaligned(d_slot_opt, 4) ||
      misaligned(a->d_alibi_slopes, 4))
    return KF_EINVAL;
  const PackedLayout L = packed_layout(a);
  if (scratch_bytes < L.total) return KF_ENOSPC;
  const uint64_t units = (uint64_t)L.units, heads = units * L.group * a->head_dim * 2, rows = units * a->head_dim * 2, slots = units * a->budget_k;
  if (conflict({{d_cache, slots * kf::packed_slot_bytes(a->head_dim)}, {d_pos, slots * 4}, {d_acc, slots * 4}, {d_len, units * 4}, {d_out, heads},
                {d_score_opt, (slots + units) * 4}, {d_slot_opt, units * 4}, {d_row_opt, rows * 2}, {d_scratch, L.total}},
               {{d_q, heads}, {d_knew, rows}, {d_vnew, rows}, {a->bias_mode == KF_BIAS_ALIBI ? a->d_alibi_slopes : nullptr, (uint64_t)a->n_heads * 4}}))
    return KF_EINVAL;
  unsigned char* scratch = static_cast<unsigned char*>(d_scratch);
  kf::PackedParams P{};
  P.cache = static_cast<unsigned char*>(d_cache);
  P.acc = d_acc; P.pos = d_pos; P.len = d_len;
  P.q = static_cast<const __half*>(d_q);
  P.knew = static_cast<const __half*>(d_knew);
  P.vnew = static_cast<const __half*>(d_vnew);
  P.out = static_cast<__half*>(d_out);
  P.score_opt = d_score_opt; P.slot_opt = d_slot_opt; P.row_opt = static_cast<__half*>(d_row_opt);
  P.y_scratch = reinterpret_cast<float*>(scratch);
  P.partials = reinterpret_cast<float*>(scratch + L.partials);
  P.slopes = a->bias_mode == KF_BIAS_ALIBI ? a->d_alibi_slopes : nullptr;
  P.k = a->budget_k; P.w = a->recent_w; P.p = a->position;
  P.splits = L.splits; P.tiles_per_split = L.tiles_per_split;
  P.H = a->n_heads; P.layer = a->layer; P.noise_mode = a->noise_mode; P.bias_mode = a->bias_mode;
  P.group = L.group;
  P.scale = a->logit_scale > 0.f ? a->logit_scale : (float)(1.0 / std::sqrt((double)a->head_dim));
  P.inv_tau = (float)(1.0 / a->tau);
  P.first_wait_limit = a->debug_fail_first_wait ? 0u : kf::DECODE_WAIT_LIMIT;
  P.noise_const = a->noise_const; P.noise_mu = a->noise_mu; P.noise_sigma = a->noise_sigma;
  P.pk = kf::philox_expand_key(a->noise_seed);
  return kf::launch_decode_packed(P, a->head_dim, L.units, static_cast<cudaStream_t>(stream)) == cudaSuccess ? KF_OK : KF_ECUDA;
}

int kf_qk_norm_rotate(const kf_qk_norm_args* a, const void* d_qkv, const void* d_q_weight, const void* d_k_weight,
                      const int32_t* d_positions, void* d_q, void* d_k, void* d_v_opt, void* stream) {
  if (!a || !d_qkv || !d_q || !d_k) return KF_EINVAL;
  if (a->batch < 1 || a->n_tokens < 1 || a->n_heads < 1 || a->n_kv_heads < 1 || a->n_heads > 65535 || a->n_kv_heads > 65535 || !head_dim_ok(a->head_dim))
    return KF_EINVAL;
  if ((int64_t)a->batch * a->n_tokens > INT32_MAX) return KF_EINVAL;
  const int64_t row = ((int64_t)a->n_heads + 2 * (int64_t)a->n_kv_heads) * a->head_dim;
  if (a->token_stride < row || a->batch_stride < 0 || a->token_stride % 8 != 0 || a->batch_stride % 8 != 0) return KF_EINVAL;
  if (a->input_type != KF_TYPE_FP16 && a->input_type != KF_TYPE_BF16) return KF_EINVAL;
  if (a->norm_mode != KF_NORM_NONE && a->norm_mode != KF_NORM_RMS) return KF_EINVAL;
  if (a->norm_mode == KF_NORM_RMS && !(a->eps >= 0.f && std::isfinite(a->eps))) return KF_EINVAL;
  if (a->norm_mode == KF_NORM_NONE && (d_q_weight || d_k_weight)) return KF_EINVAL;
  const int R = a->rotary_dims;
  if (R < 0 || R > a->head_dim || (R & (R - 1)) != 0 || (R > 0 && R < 8)) return KF_EINVAL;
  if (R > 0 && (!(a->rotary_base > 1.0f) || !std::isfinite(a->rotary_base))) return KF_EINVAL;
  if (a->rotary_style != KF_ROTARY_PAIRS && a->rotary_style != KF_ROTARY_HALVES) return KF_EINVAL;
  if (!d_positions && (int64_t)a->position0 + a->n_tokens - 1 > INT32_MAX) return KF_EINVAL;
  for (const void* p : {d_qkv, d_q_weight, d_k_weight, static_cast<const void*>(d_q), static_cast<const void*>(d_k), static_cast<const void*>(d_v_opt)})
    if (misaligned(p, 16)) return KF_EINVAL;
  if (misaligned(d_positions, 4)) return KF_EINVAL;
  const uint64_t tokens = (uint64_t)a->batch * a->n_tokens * a->head_dim * 2, out_q = tokens * a->n_heads, out_kv = tokens * a->n_kv_heads;
  const uint64_t in = ((uint64_t)(a->batch - 1) * a->batch_stride + (uint64_t)(a->n_tokens - 1) * a->token_stride + row) * 2;
  const uint64_t weight = (uint64_t)a->head_dim * 2;
  if (conflict({{d_q, out_q}, {d_k, out_kv}, {d_v_opt, out_kv}},
               {{d_qkv, in}, {d_q_weight, weight}, {d_k_weight, weight}, {d_positions, (uint64_t)a->batch * a->n_tokens * 4}}))
    return KF_EINVAL;
  kf::QkNormParams P{};
  P.qkv = d_qkv; P.q_weight = d_q_weight; P.k_weight = d_k_weight; P.positions = d_positions;
  P.q = static_cast<__half*>(d_q); P.k = static_cast<__half*>(d_k); P.v = static_cast<__half*>(d_v_opt);
  P.batch_stride = a->batch_stride; P.token_stride = a->token_stride;
  P.batch = a->batch; P.n = a->n_tokens; P.H = a->n_heads; P.Hkv = a->n_kv_heads; P.position0 = a->position0;
  P.norm = a->norm_mode == KF_NORM_RMS; P.rotary_dims = R; P.halves = a->rotary_style == KF_ROTARY_HALVES;
  P.eps = a->eps;
  P.log2_base = R > 0 ? std::log2((double)a->rotary_base) : 0.0;
  return kf::launch_qk_norm(P, a->head_dim, a->input_type == KF_TYPE_BF16, static_cast<cudaStream_t>(stream)) == cudaSuccess ? KF_OK : KF_ECUDA;
}

size_t kf_beam_scratch_bytes(const kf_beam_args* a) {
  if (!beam_ok(a)) return 0;
  int chunks = 1;
  bool wide = false;
  const int64_t rows = (int64_t)a->batch * a->beams;
  kf::beam_plan(rows, a->vocab, &chunks, &wide);
  return align_up((size_t)rows * chunks * a->take * 8) + align_up((size_t)rows * chunks * 8);
}

int kf_beam_select(const kf_beam_args* a, const void* d_logits, const float* d_scores, const uint8_t* d_finished_opt, float* d_out_scores,
                   int32_t* d_out_parent, int32_t* d_out_token, void* d_scratch, size_t scratch_bytes, void* stream) {
  if (!beam_ok(a) || !d_logits || !d_scores || !d_out_scores || !d_out_parent || !d_out_token || !d_scratch) return KF_EINVAL;
  if (misaligned(d_logits, a->logits_type == KF_TYPE_FP32 ? 4 : 2) || misaligned(d_scores, 4) || misaligned(d_out_scores, 4) ||
      misaligned(d_out_parent, 4) || misaligned(d_out_token, 4) || misaligned(d_scratch, 256))
    return KF_EINVAL;
  const size_t need = kf_beam_scratch_bytes(a);
  if (scratch_bytes < need) return KF_ENOSPC;
  const uint64_t beams = (uint64_t)a->batch * a->beams, out = (uint64_t)a->batch * a->take * 4, size = a->logits_type == KF_TYPE_FP32 ? 4 : 2;
  if (conflict({{d_out_scores, out}, {d_out_parent, out}, {d_out_token, out}, {d_scratch, need}},
               {{d_logits, a->vocab * size, beams, a->row_stride * size}, {d_scores, beams * 4}, {d_finished_opt, beams}}))
    return KF_EINVAL;
  kf::BeamParams P{};
  bool wide = false;
  const int64_t rows = (int64_t)a->batch * a->beams;
  kf::beam_plan(rows, a->vocab, &P.chunks, &wide);
  P.logits = d_logits; P.scores = d_scores; P.finished = d_finished_opt;
  P.out_scores = d_out_scores; P.out_parent = d_out_parent; P.out_token = d_out_token;
  P.lists = static_cast<uint2*>(d_scratch);
  P.stats = reinterpret_cast<float2*>(static_cast<unsigned char*>(d_scratch) + align_up((size_t)rows * P.chunks * a->take * 8));
  P.row_stride = a->row_stride;
  P.batch = a->batch; P.beams = a->beams; P.vocab = a->vocab; P.take = a->take; P.pad = a->pad_token;
  return kf::launch_beam_select(P, a->logits_type, wide, static_cast<cudaStream_t>(stream)) == cudaSuccess ? KF_OK : KF_ECUDA;
}

int kf_reorder_rows(const kf_row_buffer* buffers, int32_t n_buffers, int32_t batch, int32_t beams, const int32_t* d_parent, void* stream) {
  if (!buffers || n_buffers < 1 || n_buffers > kf::REORDER_BUFFERS || batch < 1 || batch > 65535 || beams < 1 || beams > kf::BEAM_MAX) return KF_EINVAL;
  if (!d_parent || misaligned(d_parent, 4)) return KF_EINVAL;
  kf::ReorderParams P{};
  for (int i = 0; i < n_buffers; ++i) {
    const kf_row_buffer& b = buffers[i];
    if (!b.d_base || b.row_bytes < 1 || b.row_bytes > ((int64_t)1 << 40) || b.outer < 1) return KF_EINVAL;
    if (b.outer > 1 && b.outer_stride < b.row_bytes * batch * beams) return KF_EINVAL;
    // a row that two descriptions move would be read while it is written
    auto extent = [&](const kf_row_buffer& x) { return (uint64_t)(x.outer - 1) * (x.outer > 1 ? x.outer_stride : 0) + (uint64_t)x.row_bytes * batch * beams; };
    for (int j = 0; j < i; ++j)
      if (overlap(b.d_base, extent(b), buffers[j].d_base, extent(buffers[j]))) return KF_EINVAL;
    if (overlap(b.d_base, extent(b), d_parent, (uint64_t)batch * beams * 4)) return KF_EINVAL;
    P.buf[i].base = static_cast<unsigned char*>(b.d_base);
    P.buf[i].row_bytes = b.row_bytes;
    P.buf[i].outer = b.outer;
    P.buf[i].outer_stride = b.outer_stride;
  }
  P.n_buffers = n_buffers; P.batch = batch; P.beams = beams; P.parent = d_parent;
  const cudaError_t e = kf::launch_reorder(P, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? KF_OK : (e == cudaErrorInvalidValue ? KF_EINVAL : KF_ECUDA);
}

}  // extern "C"
