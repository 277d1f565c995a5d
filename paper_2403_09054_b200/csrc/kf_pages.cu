// 8-bit pages: rows in (kf_pages_write), rows out (kf_pages_read), kept rows to new pages (kf_pages_compact), and the tables (kf_pages_update).
// The format and why scales are powers of two: kf_pages.cuh.
//
// All of them are bound by memory (or, for single tokens, by the latency of a few dependent loads): a CTA owns one page of one key/value head,
// whose K and V tiles are contiguous, so that codes move 16 bytes a thread and the scale of a tile is decided by one CTA, without
// a second pass over memory and without atomics.  Eight sequences of up to 4096 tokens (32 heads, d 128, pages of 64): written in 69 us and read back in 72,
// 6.0 and 5.8 TB/s; ALU pipe 65 % and issue slots 65 % busy while writing (codes by conversion instructions instead of one addition: 127 us).
// 16 prompts of up to 4096 tokens reduced to half: 61 us (4.6 TB/s, scattered rows of 128 bytes), and read
// back in 74.  Tables: 10 to 12 us with the copies, four to five dependent trips to
// memory.
#include "kf_pages.cuh"
#include "kf_tc.cuh"

#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

namespace kf {

namespace {

namespace cg = cooperative_groups;

constexpr int NT = 256;              // threads of a CTA of the copies, and at most of one that works on a page where pages get few rows
constexpr int HELD = 8;              // 16-byte pieces of rows a thread keeps between the maximum and the codes

// The smallest 2^e with top <= 127 * 2^e, e >= -120, by the exponent and the leading bits of top; NaN where top is not finite.
__device__ __forceinline__ float power_scale(float top) {
  const uint32_t bits = __float_as_uint(top);
  if (bits >= 0x7f800000u) return nan_f32();                    // top carries no sign
  // top = m * 2^x with 1 <= m < 2 (anything below 2^-126 is below 127 * 2^-120): e = x - 6 if m <= 127 / 64, else x - 5
  const int e = (int)(bits >> 23) - 127 - 6 + ((bits & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  return __uint_as_float((uint32_t)(max(e, -120) + 127) << 23);
}

// Four codes as binary32 integers: 2^23 + (c + 128) has the bits 0x4b000000 | (c ^ 0x80).
__device__ __forceinline__ void numbers4(uint32_t codes, float (&x)[4]) {
  const uint32_t u = codes ^ 0x80808080u;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 | i));
  add2(x[0], x[1], -8388736.f, -8388736.f);
  add2(x[2], x[3], -8388736.f, -8388736.f);
}
// rint(x * by), |x * by| <= 127, as four codes: the sum with 1.5 * 2^23 holds the integer (ties to even) in its last bits.
__device__ __forceinline__ uint32_t codes4(float x0, float x1, float x2, float x3, float by) {
  float y0, y1, y2, y3;
  fma2(y0, y1, x0, x1, by, 12582912.f);
  fma2(y2, y3, x2, x3, by, 12582912.f);
  return __byte_perm(__byte_perm(__float_as_uint(y0), __float_as_uint(y1), 0x0040), __byte_perm(__float_as_uint(y2), __float_as_uint(y3), 0x0040), 0x5410);
}
// Codes of one scale as codes of a larger one, `ratio` = the old one over the new one.
__device__ __forceinline__ uint32_t rescale4(uint32_t codes, float ratio) {
  float x[4];
  numbers4(codes, x);
  return codes4(x[0], x[1], x[2], x[3], ratio);
}

template <bool BF16>
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (BF16) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}

// The larger |x| of pairs of 16-bit values, NaN if there is one.
template <bool BF16>
__device__ __forceinline__ uint32_t top2(uint32_t a, uint32_t b) {
  b &= 0x7fff7fffu;
  if (BF16) {
    const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
  }
  const __half2 m = __hmax2_nan(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}
template <bool BF16>
__device__ __forceinline__ uint32_t top8(uint32_t top, const uint4& v) {
  return top2<BF16>(top2<BF16>(top2<BF16>(top2<BF16>(top, v.x), v.y), v.z), v.w);
}

struct WriteParams {
  PageCache c;
  const void *k, *v;
  int64_t k_token, k_head, v_token, v_head;
  const int32_t *begin, *length, *table;
  int32_t tokens, log_page, log_vec;   // log2 of the page and of the 16-byte pieces of a row of 16-bit values
};

// The rows of one page and head.  Grid: slots (see slot_sequence; the new rows of a sequence touch at most rows / page + 2 pages), heads.
template <bool BF16, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) pages_write_kernel(const __grid_constant__ WriteParams P) {
  constexpr int SIDE = NT / 2;
  __shared__ uint32_t sh_top[NT / 32];
  after_earlier_kernels();
  let_next_kernel_launch();
  const PageCache& c = P.c;
  const int side = threadIdx.x >= SIDE, tid = threadIdx.x & (SIDE - 1);
  int s = blockIdx.x, from = s, count = 1, part = 0;
  if (P.begin) {
    s = slot_sequence(P.begin, c.S, blockIdx.x, 1, P.log_page, 2);
    from = P.begin[s];
    const int to = P.begin[s + 1];
    if (from < 0 || to > P.tokens || to <= from) return;
    count = to - from;
    const int64_t local = (int64_t)blockIdx.x - slot_start(P.begin, s, 1, P.log_page, 2);
    if (local < 0 || local > count) return;
    part = (int)local;
  }
  const int old = P.length[s];                                   // tokens there already
  const int64_t capacity = (int64_t)c.W << P.log_page;
  if (old < 0 || old >= capacity) return;
  const int page_at = (old >> P.log_page) + part;                // which of the sequence's pages
  const int first_token = page_at << P.log_page;
  const int lo = max(old, first_token), hi = (int)min(min((int64_t)old + count, (int64_t)first_token + c.page), capacity);
  if (lo >= hi) return;
  const int id = P.table[(size_t)s * c.W + page_at];
  if (id < 0 || id >= c.pages) return;
  const int rows = hi - lo, r0 = lo - first_token;               // new rows, and rows that the page holds already
  const size_t tile = ((size_t)id * c.Hkv + blockIdx.y) * 2 + side;
  float* scale_at = c.scale + tile;
  const float was = r0 > 0 ? *scale_at : 0.f;
  const unsigned short* src = static_cast<const unsigned short*>(side ? P.v : P.k) + (int64_t)(from + lo - old) * (side ? P.v_token : P.k_token) +
                              (int64_t)blockIdx.y * (side ? P.v_head : P.k_head);
  const int64_t stride = side ? P.v_token : P.k_token;
  const int vecs = rows << P.log_vec;
  auto load = [&](int i) { return *reinterpret_cast<const uint4*>(src + (int64_t)(i >> P.log_vec) * stride + (i & ((1 << P.log_vec) - 1)) * 8); };
  uint4 held[HELD];
  uint32_t top = 0;
#pragma unroll
  for (int h = 0; h < HELD; ++h) {
    const int i = tid + h * SIDE;
    held[h] = i < vecs ? load(i) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int h = 0; h < HELD; ++h) top = top8<BF16>(top, held[h]);
  for (int i = tid + HELD * SIDE; i < vecs; i += SIDE) top = top8<BF16>(top, load(i));
  // the bits of |x| are in order, with NaN above infinity: the larger of the pair as a binary32 number, then the largest of the CTA
  top = max(top & 0xffffu, top >> 16);
  top = BF16 ? top << 16 : __float_as_uint(__half2float(__ushort_as_half((unsigned short)top)));
  top = __reduce_max_sync(0xffffffffu, top & 0x7fffffffu);
  if ((threadIdx.x & 31) == 0) sh_top[threadIdx.x >> 5] = top;
  __syncthreads();
  top = 0;
#pragma unroll
  for (int w = 0; w < SIDE / 32; ++w) top = max(top, sh_top[side * (SIDE / 32) + w]);
  const float fresh = power_scale(__uint_as_float(top));
  // a scale that is NaN stays one while its page fills
  const float scale = r0 == 0 ? fresh : (fresh != fresh ? fresh : (was >= fresh || was != was ? was : fresh));
  const float inverse = scale > 0.f ? 1.f / scale : 0.f;
  signed char* codes = c.codes + tile * (size_t)c.page * c.d;
  if (r0 > 0 && scale > was) {                                   // rows that are there already move to the larger scale
    const float ratio = was > 0.f ? was * inverse : 0.f;
    for (int i = tid; i < r0 * (c.d / 16); i += SIDE) {
      const uint4 v = reinterpret_cast<uint4*>(codes)[i];
      reinterpret_cast<uint4*>(codes)[i] = make_uint4(rescale4(v.x, ratio), rescale4(v.y, ratio), rescale4(v.z, ratio), rescale4(v.w, ratio));
    }
  }
  const uint32_t valid = scale == scale ? 0xffffffffu : 0u;      // what is not finite has no codes
  auto store = [&](int i, const uint4& v) {
    float x[8];
    unpack8<BF16>(v, x);
    *reinterpret_cast<uint2*>(codes + ((size_t)r0 << (P.log_vec + 3)) + (size_t)i * 8) =
        make_uint2(codes4(x[0], x[1], x[2], x[3], inverse) & valid, codes4(x[4], x[5], x[6], x[7], inverse) & valid);
  };
#pragma unroll
  for (int h = 0; h < HELD; ++h) {
    const int i = tid + h * SIDE;
    if (i < vecs) store(i, held[h]);
  }
  for (int i = tid + HELD * SIDE; i < vecs; i += SIDE) store(i, load(i));
  if (tid == 0) *scale_at = scale;
}

struct ReadParams {
  PageCache c;
  void *k, *v;
  int64_t k_token, k_head, v_token, v_head;
  const int32_t *begin, *first, *table;
  int32_t tokens, log_page, log_vec;   // log2 of the page and of the 16-byte pieces of a row of codes
  bool wide;                           // rows are aligned to 32 bytes
};

template <bool BF16, int NT>
__global__ void __launch_bounds__(NT, 2048 / NT) pages_read_kernel(const __grid_constant__ ReadParams P) {
  constexpr int SIDE = NT / 2;
  after_earlier_kernels();
  let_next_kernel_launch();
  const PageCache& c = P.c;
  const int side = threadIdx.x >= SIDE, tid = threadIdx.x & (SIDE - 1);
  const int s = slot_sequence(P.begin, c.S, blockIdx.x, 1, P.log_page, 2);
  const int from = P.begin[s], to = P.begin[s + 1];
  if (from < 0 || to > P.tokens || to <= from) return;
  const int64_t local = (int64_t)blockIdx.x - slot_start(P.begin, s, 1, P.log_page, 2);
  if (local < 0 || local > to - from) return;
  const int start = P.first ? P.first[s] : 0;                    // may be anything: tokens that do not exist read as NaN
  const int64_t page_at = ((int64_t)start >> P.log_page) + local;
  const int64_t first_token = page_at << P.log_page;
  const int64_t lo = max((int64_t)start, first_token), hi = min((int64_t)start + (to - from), first_token + c.page);
  if (lo >= hi) return;
  const int id = page_at >= 0 && page_at < c.W ? P.table[(size_t)s * c.W + page_at] : -1;
  const bool held = id >= 0 && id < c.pages;
  const size_t tile = ((size_t)(held ? id : 0) * c.Hkv + blockIdx.y) * 2 + side;
  const float scale = held ? c.scale[tile] : nan_f32();
  const uint4* codes = reinterpret_cast<const uint4*>(c.codes + (tile * c.page + (size_t)(lo - first_token)) * c.d);
  unsigned short* dst = static_cast<unsigned short*>(side ? P.v : P.k) + (from + (lo - start)) * (side ? P.v_token : P.k_token) +
                        (int64_t)blockIdx.y * (side ? P.v_head : P.k_head);
  const int64_t stride = side ? P.v_token : P.k_token;
  const int vecs = (int)(hi - lo) << P.log_vec;
#pragma unroll 2
  for (int i = tid; i < vecs; i += SIDE) {
    const uint4 w = held ? codes[i] : make_uint4(0, 0, 0, 0);
    uint32_t r[8];
    float x[16];
    numbers4(w.x, reinterpret_cast<float(&)[4]>(x[0]));
    numbers4(w.y, reinterpret_cast<float(&)[4]>(x[4]));
    numbers4(w.z, reinterpret_cast<float(&)[4]>(x[8]));
    numbers4(w.w, reinterpret_cast<float(&)[4]>(x[12]));
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const float a = x[2 * p] * scale, b = x[2 * p + 1] * scale;
      if (BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        r[p] = *reinterpret_cast<const uint32_t*>(&h);
      } else {
        const __half2 h = __floats2half2_rn(a, b);
        r[p] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    unsigned short* at = dst + (int64_t)(i >> P.log_vec) * stride + (i & ((1 << P.log_vec) - 1)) * 16;
    if (P.wide) {                                                // two stores of 16 bytes instead: 75.6 against 71.5 us
      store_sector(at, r);
    } else {
      reinterpret_cast<uint4*>(at)[0] = make_uint4(r[0], r[1], r[2], r[3]);
      reinterpret_cast<uint4*>(at)[1] = make_uint4(r[4], r[5], r[6], r[7]);
    }
  }
}

// ---- kept rows to new pages.  Grid: pages of the new table, heads, sequences (folded into x where the other limits do not hold it).
struct CompactParams {
  PageCache c;
  const int32_t *table, *length, *keep, *n_keep, *new_table;
  int32_t keep_width, new_width, log_page, log_vec;
};

template <int NT>
__global__ void __launch_bounds__(NT, 2048 / NT) pages_compact_kernel(const __grid_constant__ CompactParams P) {
  __shared__ int64_t sh_row[128];             // where a row's K codes stand, -1: nowhere
  __shared__ float sh_scale[2][128];
  __shared__ uint32_t sh_top[2][NT / 32];
  constexpr int SIDE = NT / 2;
  after_earlier_kernels();
  let_next_kernel_launch();
  const PageCache& c = P.c;
  const int s = blockIdx.x / P.new_width, j = blockIdx.x % P.new_width, h = blockIdx.y;
  const int kept = min(P.n_keep[s], P.keep_width);
  const int rows = min(kept - (j << P.log_page), c.page);
  if (rows <= 0) return;
  const int to = P.new_table[(size_t)s * P.new_width + j];
  if (to < 0 || to >= c.pages) return;
  uint32_t tk = 0, tv = 0;                    // scales carry no sign: their bits are in order, with NaN on top
  for (int r = threadIdx.x; r < rows; r += NT) {
    const int token = P.keep[((size_t)s * c.Hkv + h) * P.keep_width + (j << P.log_page) + r];
    const int slot = token >> P.log_page;
    int id = -1;
    if (token >= 0 && token < P.length[s] && slot < c.W) id = P.table[(size_t)s * c.W + slot];
    float2 scale = make_float2(nan_f32(), nan_f32());
    int64_t at = -1;
    if (id >= 0 && id < c.pages) {
      const size_t tile = ((size_t)id * c.Hkv + h) * 2;
      scale = *reinterpret_cast<const float2*>(c.scale + tile);
      at = (int64_t)(tile * c.page + (token & (c.page - 1))) * c.d;
    }
    sh_row[r] = at;
    sh_scale[0][r] = scale.x;
    sh_scale[1][r] = scale.y;
    tk = max(tk, __float_as_uint(scale.x));
    tv = max(tv, __float_as_uint(scale.y));
  }
  tk = __reduce_max_sync(0xffffffffu, tk);
  tv = __reduce_max_sync(0xffffffffu, tv);
  if ((threadIdx.x & 31) == 0) { sh_top[0][threadIdx.x >> 5] = tk; sh_top[1][threadIdx.x >> 5] = tv; }
  __syncthreads();
  const int side = threadIdx.x >= SIDE, tid = threadIdx.x & (SIDE - 1);
  uint32_t top = 0;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) top = max(top, sh_top[side][w]);
  const float scale = __uint_as_float(top);
  const float inverse = scale > 0.f ? 1.f / scale : 0.f;
  const size_t tile = ((size_t)to * c.Hkv + h) * 2 + side;
  uint4* out = reinterpret_cast<uint4*>(c.codes + tile * (size_t)c.page * c.d);
  const int log_vec = P.log_vec, vec = 1 << log_vec;            // 16-byte pieces of a row
#pragma unroll 4
  for (int i = tid; i < rows << log_vec; i += SIDE) {
    const int r = i >> log_vec;
    const int64_t at = sh_row[r];
    uint4 v = make_uint4(0, 0, 0, 0);
    if (at >= 0) v = reinterpret_cast<const uint4*>(c.codes + at + (int64_t)side * c.page * c.d)[i & (vec - 1)];
    const float ratio = sh_scale[side][r] * inverse;
    if (ratio < 1.f) v = make_uint4(rescale4(v.x, ratio), rescale4(v.y, ratio), rescale4(v.z, ratio), rescale4(v.w, ratio));
    out[i] = v;
  }
  if (tid == 0) c.scale[tile] = scale;
}

// ---- tables.  One CTA, or one cluster of eight for large tables, does the whole update: its barrier stands between counting references, looking
// for free pages and handing them out.  Every CTA works out the sequences' lengths and where each one's pages begin in the list for itself.
constexpr int CLUSTER = 8, UT = 1024, UPDATE_LIST = 8192;

constexpr int KEEPS = 1 << 30;         // tokens are fewer

struct UpdateShared {
  int source[UPDATE_MAX_SEQUENCES];   // whom a sequence goes on from (-1: it has ended)
  int length[UPDATE_MAX_SEQUENCES];   // its tokens; KEEPS: it keeps its source's page that is filled in part
  int need[UPDATE_MAX_SEQUENCES];     // pages it is to have; until that is known, the lowest sequence that goes on from this one
  int prefix[UPDATE_MAX_SEQUENCES];   // the tokens it is to have room for, then the pages handed out to the sequences before it
  int list[UPDATE_LIST];              // free pages, where one CTA hands out no more than these
  int scan[UT / 32];
  int found;
  unsigned long long beyond;
};

__device__ __forceinline__ int block_exclusive(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int sums = lane < UT / 32 ? warp_sums[lane] : 0, before = sums;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += y;
  }
  total = __shfl_sync(0xffffffffu, before, 31);
  before -= sums;
  return __shfl_sync(0xffffffffu, before, warp) + x - v;
}

struct Sequence {
  int source, full, part, keeps, stay, need, prefix;   // stay: pages kept from the source; need: pages in all
};

__global__ void __launch_bounds__(UT, 1) pages_update_kernel(const __grid_constant__ PagesUpdate U) {
  extern __shared__ __align__(16) unsigned char update_smem[];
  UpdateShared& sh = *reinterpret_cast<UpdateShared*>(update_smem);
  cg::cluster_group cluster = cg::this_cluster();
  const PageCache& c = U.c;
  const int S = c.S, W = c.W, rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks(), tid = threadIdx.x;
  const int64_t capacity = (int64_t)W * c.page;
  const int log_page = U.log_page;
  after_earlier_kernels();
  let_next_kernel_launch();

  // ---- lengths, who keeps a page that is filled in part, and the pages to hand out before each sequence
  for (int s = tid; s < S; s += UT) sh.need[s] = S;
  if (tid == 0) sh.beyond = 0;
  __syncthreads();
  for (int s = tid; s < S; s += UT) {
    int p = U.parent ? U.parent[s] : s;
    const int grow = max(U.grow ? U.grow[s] : U.grow_all, 0);
    if (p < 0 || p >= S) p = -1;
    int n = p >= 0 ? U.length[p] : 0;
    if (n < 0 || n > capacity) n = 0;
    sh.source[s] = p;
    sh.length[s] = n;
    sh.prefix[s] = grow;
    if (p >= 0) atomicMin(&sh.need[p], s);
  }
  __syncthreads();
  for (int s = tid; s < S; s += UT) {
    const int p = sh.source[s];
    if (p >= 0 && (sh.length[s] & (c.page - 1)) != 0 && sh.need[p] == s) sh.length[s] |= KEEPS;
  }
  __syncthreads();
  int wanted = 0;                                                // pages to hand out, of all sequences
  for (int base = 0; base < S; base += UT) {
    const int s = base + tid;
    int fresh = 0;
    if (s < S) {
      const int n = sh.length[s] & ~KEEPS;
      const int64_t need = ((int64_t)n + sh.prefix[s] + c.page - 1) >> log_page;
      sh.need[s] = (int)min(need, (int64_t)W);
      if (need > W) atomicAdd(&sh.beyond, (unsigned long long)(need - W));      // the table has no room for them
      fresh = sh.need[s] - (n >> log_page) - (n != sh.length[s]);
    }
    int total;
    const int before = block_exclusive(fresh, sh.scan, total);
    if (s < S) sh.prefix[s] = wanted + before;
    wanted += total;
  }
  __syncthreads();
  auto look = [&](int s) {
    Sequence q;
    const int n = sh.length[s] & ~KEEPS;
    q.source = sh.source[s];
    q.full = n >> log_page;
    q.part = n & (c.page - 1);
    q.keeps = n != sh.length[s];
    q.stay = q.full + q.keeps;
    q.need = sh.need[s];
    q.prefix = sh.prefix[s];
    return q;
  };

  // ---- references: what the table names now no longer counts, what stays does
  const uint32_t entries = (uint32_t)S * (uint32_t)W;            // at most 2^28
  const uint32_t thread = (uint32_t)(rank * UT + tid), threads = (uint32_t)ranks * UT;
  for (uint32_t i = thread; i < entries; i += threads) {
    const int s = (int)(i / (uint32_t)W), j = (int)(i - (uint32_t)s * (uint32_t)W);
    const Sequence q = look(s);
    const bool tail = j == q.full && q.part > 0;                 // the page that is filled in part
    const int old = U.table[i];
    int next = -1;
    if (j < q.stay || tail) next = q.source == s ? old : U.table[(size_t)q.source * W + j];
    if (next < 0 || next >= c.pages) next = -1;
    if (tail) U.copies[s].x = next;
    if (j >= q.stay) next = -1;
    U.stays[i] = next;
    if (next != old) {
      if (old >= 0 && old < c.pages) atomicSub(&U.refs[old], 1);
      if (next >= 0) atomicAdd(&U.refs[next], 1);
    }
  }
  cluster.sync();                                                // releases and acquires: the counts are seen by all

  // ---- free pages, lowest first: counted per CTA where there are several, then listed
  const int per = ((c.pages + ranks - 1) / ranks + 3) & ~3;      // a CTA's stretch of pages
  const int lo = (int)min((int64_t)rank * per, (int64_t)c.pages), hi = (int)min((int64_t)lo + per, (int64_t)c.pages);
  auto free_mask = [&](int p) {                                  // pages p .. p + 3
    uint32_t m = 0;
    if (p + 3 < hi && (reinterpret_cast<uintptr_t>(U.refs) & 15) == 0) {
      const int4 r = __ldcg(reinterpret_cast<const int4*>(U.refs + p));
      m = (r.x == 0) | (r.y == 0) << 1 | (r.z == 0) << 2 | (r.w == 0) << 3;
    } else {
      for (int e = 0; e < 4 && p + e < hi; ++e) m |= (uint32_t)(__ldcg(U.refs + p + e) == 0) << e;
    }
    return m;
  };
  int* free_list = ranks == 1 && wanted <= UPDATE_LIST ? sh.list : U.free_list;
  int at_rank = 0, total;                                        // free pages before the next stretch
  if (ranks > 1) {
    int mine = 0;
    if (wanted > 0)
      for (int p = lo + tid * 4; p < hi; p += UT * 4) mine += __popc(free_mask(p));
    (void)block_exclusive(mine, sh.scan, total);
    if (tid == 0) sh.found = total;
    cluster.sync();
    for (int r = 0; r < rank; ++r) at_rank += *cluster.map_shared_rank(&sh.found, r);
  }
  for (int base = lo; base < hi && at_rank < wanted; base += UT * 4) {
    const int p = base + tid * 4;
    const uint32_t m = p < hi ? free_mask(p) : 0;
    int at = block_exclusive(__popc(m), sh.scan, total) + at_rank;
    for (int e = 0; e < 4; ++e)
      if (m >> e & 1) {
        if (at < wanted) { free_list[at] = p + e; U.refs[p + e] = 1; }
        ++at;
      }
    at_rank += total;
  }
  int available = at_rank;                                       // of one CTA: all that were looked at, or as many as are wanted
  if (ranks > 1) {
    available = 0;
    for (int r = 0; r < ranks; ++r) available += *cluster.map_shared_rank(&sh.found, r);
  }
  const int given = min(wanted, available);
  cluster.sync();

  // ---- the new table
  for (uint32_t i = thread; i < entries; i += threads) {
    const int s = (int)(i / (uint32_t)W), j = (int)(i - (uint32_t)s * (uint32_t)W);
    const Sequence q = look(s);
    int next = U.stays[i];
    if (j >= q.stay && j < q.need) next = q.prefix + j - q.stay < given ? *(volatile int*)(free_list + q.prefix + j - q.stay) : -1;
    U.table[i] = next;
    if (j == 0) {
      const bool copy = q.part > 0 && !q.keeps;                  // into its first new page
      U.copies[s] = make_int4(copy ? __ldcg(&U.copies[s].x) : -1, copy && q.prefix < given ? *(volatile int*)(free_list + q.prefix) : -1, q.part, 0);
      U.length[s] = sh.length[s] & ~KEEPS;                                // every CTA has read the lengths long before
    }
  }
  if (rank == 0 && tid == 0) *U.missing = (int)min((int64_t)(wanted - given) + (int64_t)sh.beyond, (int64_t)INT32_MAX);
}

// The rows of pages that are filled in part.  Grid: sequences, layers, pieces of the heads.
__global__ void __launch_bounds__(NT) pages_copy_kernel(const __grid_constant__ PagesUpdate U) {
  after_earlier_kernels();
  let_next_kernel_launch();
  const int4 copy = __ldcg(U.copies + blockIdx.x);
  if (copy.y < 0) return;
  const PageCache& c = U.c;
  const size_t layer = (size_t)blockIdx.y * c.pages;
  const int tiles = c.Hkv * 2, from = tiles * (int)blockIdx.z / (int)gridDim.z, to = tiles * ((int)blockIdx.z + 1) / (int)gridDim.z;
  const size_t b = (layer + copy.y) * tiles;
  if (copy.x < 0) {                                               // the parent's page is missing: the copy reads as NaN
    for (int t = from + threadIdx.x; t < to; t += NT) c.scale[b + t] = nan_f32();
    return;
  }
  const size_t a = (layer + copy.x) * tiles;
  const int vec = copy.z * c.d / 16;                              // 16-byte pieces of the rows of a tile
  const size_t tile_vec = (size_t)c.page * c.d / 16;
  const uint4* src = reinterpret_cast<const uint4*>(c.codes);
  uint4* dst = reinterpret_cast<uint4*>(c.codes);
#pragma unroll 4
  for (int i = threadIdx.x; i < (to - from) * vec; i += NT) {
    const int t = i / vec, r = i - t * vec;
    dst[(b + from + t) * tile_vec + r] = src[(a + from + t) * tile_vec + r];
  }
  for (int t = from + threadIdx.x; t < to; t += NT) c.scale[b + t] = c.scale[a + t];
}

// Whether a slot has, on average, no more than one 16-byte piece of a row for each thread of a side: then 64 threads do (64 tokens of 8 heads, written and
// read back: 8.4 instead of 11.2 us).
bool few_rows(int tokens, unsigned slots, int d) { return (int64_t)tokens * (d / 8) <= (int64_t)slots * (NT / 2); }

int log2_of(int x) { int n = 0; while ((1 << n) < x) ++n; return n; }

}  // namespace

// Threads of a CTA that works on a page, half of them on K, half on V: `go` with the number (a constant of a type) that deals `pieces` per thread to a page
// of `all` on each side, within 64 and MOST.  Fewer than the page's rows keep busy leave loads for a second round, more leave threads with the chain of loads to a page
// and nothing to do: against 256 for every page, 16 prompts of 2048 tokens on 8 heads (d 128, pages of 16) are written in 39 instead of 88 us and read in
// 38 instead of 47, 8 of 2048 on 32 heads (pages of 32) in 67 instead of 98 and 72 instead of 80, 4 of 4096 on 16 heads (d 256, pages of 128) written in 91 instead of 100.
template <int MOST, int T = 64, class Go>
cudaError_t threads_for(int all, int pieces, Go go) {
  if constexpr (T < MOST)
    if (all > T / 2 * pieces) return threads_for<MOST, 2 * T>(all, pieces, go);
  return go(std::integral_constant<int, T>{});
}

// 16-byte pieces of codes for a thread: four, or two while CTAs of 256 threads for all pages run at once (one prompt of 2047 tokens, 16 heads of 256,
// reduced and read back: 10.3 instead of 11.5 us).
int pieces_of(dim3 grid) { return (int64_t)grid.x * grid.y <= 148 * 8 ? 2 : 4; }

cudaError_t launch_pages_write(const PageCache& c, const PageRows& r, const int32_t* begin, const int32_t* length, const int32_t* table, cudaStream_t stream) {
  WriteParams P{};
  P.c = c; P.k = r.k; P.v = r.v; P.k_token = r.k_token; P.k_head = r.k_head; P.v_token = r.v_token; P.v_head = r.v_head;
  P.begin = begin; P.length = length; P.table = table; P.tokens = r.tokens;
  P.log_page = log2_of(c.page); P.log_vec = log2_of(c.d / 8);
  const unsigned slots = begin ? (unsigned)((r.tokens >> P.log_page) + 2 * c.S) : (unsigned)c.S;
  const dim3 grid(slots, (unsigned)c.Hkv);
  return threads_for<1024>(few_rows(r.tokens, slots, c.d) ? 0 : c.page * c.d / 8, HELD, [&](auto n) {
    constexpr int T = decltype(n)::value;
    return r.bf16 ? launch_early(pages_write_kernel<true, T>, grid, T, 0, stream, P) : launch_early(pages_write_kernel<false, T>, grid, T, 0, stream, P);
  });
}

cudaError_t launch_pages_read(const PageCache& c, const PageRows& r, const int32_t* begin, const int32_t* first, const int32_t* table, cudaStream_t stream) {
  ReadParams P{};
  P.c = c; P.k = r.k; P.v = r.v; P.k_token = r.k_token; P.k_head = r.k_head; P.v_token = r.v_token; P.v_head = r.v_head;
  P.begin = begin; P.first = first; P.table = table; P.tokens = r.tokens;
  P.log_page = log2_of(c.page); P.log_vec = log2_of(c.d / 16);
  P.wide = (reinterpret_cast<uintptr_t>(r.k) | reinterpret_cast<uintptr_t>(r.v)) % 32 == 0 && (r.k_token | r.k_head | r.v_token | r.v_head) % 16 == 0;
  const unsigned slots = (unsigned)((r.tokens >> P.log_page) + 2 * c.S);
  const dim3 grid(slots, (unsigned)c.Hkv);
  return threads_for<256>(few_rows(r.tokens, slots, c.d) ? 0 : c.page * c.d / 16, pieces_of(grid), [&](auto n) {
    constexpr int T = decltype(n)::value;
    return r.bf16 ? launch_early(pages_read_kernel<true, T>, grid, T, 0, stream, P) : launch_early(pages_read_kernel<false, T>, grid, T, 0, stream, P);
  });
}

cudaError_t launch_pages_compact(const PageCache& c, int keep_width, int new_width, const int32_t* table, const int32_t* length, const int32_t* keep,
                                 const int32_t* n_keep, const int32_t* new_table, cudaStream_t stream) {
  CompactParams P{};
  P.c = c; P.table = table; P.length = length; P.keep = keep; P.n_keep = n_keep; P.new_table = new_table;
  P.keep_width = keep_width; P.new_width = new_width; P.log_page = log2_of(c.page); P.log_vec = log2_of(c.d / 16);
  const dim3 grid((unsigned)c.S * (unsigned)new_width, (unsigned)c.Hkv);
  return threads_for<256>(c.page * c.d / 16, pieces_of(grid), [&](auto n) {
    constexpr int T = decltype(n)::value;
    return launch_early(pages_compact_kernel<T>, grid, T, 0, stream, P);
  });
}

cudaError_t launch_pages_update(const PagesUpdate& u, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(pages_update_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(UpdateShared));
  if (e != cudaSuccess) return e;
  PagesUpdate U = u;
  U.log_page = log2_of(u.c.page);
  // entries and pages one CTA goes through in a few rounds; the barriers of a cluster cost about as much
  const bool small = (int64_t)u.c.S * u.c.W + u.c.pages / 4 <= 16 * UT;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {small ? 1u : (unsigned)CLUSTER, 1u, 1u};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(small ? 1u : (unsigned)CLUSTER);
  cfg.blockDim = dim3(UT);
  cfg.dynamicSmemBytes = sizeof(UpdateShared);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, pages_update_kernel, U);
  if (e != cudaSuccess || !u.parent) return e;                    // without parents no page has a second owner
  // most CTAs find nothing to copy: no more of them than a few per SM where there are many sequences
  const int64_t rows = (int64_t)u.c.S * u.layers;
  const int pieces = (int)std::min<int64_t>(std::min(8, u.c.Hkv * 2), std::max<int64_t>(1, 1024 / rows));
  return launch_early(pages_copy_kernel, dim3((unsigned)u.c.S, (unsigned)u.layers, (unsigned)pieces), NT, 0, stream, U);
}

}  // namespace kf
