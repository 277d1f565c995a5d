// 8-bit pages: rows in (kf_pages_write), rows out (kf_pages_read), kept rows to new pages (kf_pages_compact), and the tables (kf_pages_update).
// The format and why scales are powers of two: kf_pages.cuh.
//
// All of them are bound by memory (or, for single tokens, by the latency of a few dependent loads): a CTA owns one page of one key/value head,
// whose K and V tiles are contiguous, so that codes move 16 bytes a thread and the scale of a tile is decided by one CTA, without
// a second pass over memory and without atomics.
#include "kf_pages.cuh"

#include <cooperative_groups.h>

namespace kf {

namespace {

namespace cg = cooperative_groups;

constexpr int NT = 256;              // threads of a CTA that works on a page: half of them on K, half on V
constexpr int SIDE = NT / 2;
constexpr int HELD = 8;              // 16-byte pieces of rows a thread keeps between the maximum and the codes

// The smallest 2^e with top <= 127 * 2^e, e >= -120, by the exponent and the leading bits of top; NaN where top is not finite.
__device__ __forceinline__ float power_scale(float top) {
  const uint32_t bits = __float_as_uint(top);
  if (bits >= 0x7f800000u) return nan_f32();                    // top carries no sign
  // top = m * 2^x with 1 <= m < 2 (anything below 2^-126 is below 127 * 2^-120): e = x - 6 if m <= 127 / 64, else x - 5
  const int e = (int)(bits >> 23) - 127 - 6 + ((bits & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  return __uint_as_float((uint32_t)(max(e, -120) + 127) << 23);
}

__device__ __forceinline__ signed char code_of(float x, float inverse) {
  return (signed char)(int)fminf(fmaxf(rintf(x * inverse), -127.f), 127.f);
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

// The largest |x| of eight values, as the bits of a binary32 number (NaN above infinity above all numbers).
template <bool BF16>
__device__ __forceinline__ uint32_t top8(const uint4& v) {
  float x[8];
  unpack8<BF16>(v, x);
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(x[i]) & 0x7fffffffu);
  return t;
}

struct WriteParams {
  PageCache c;
  const void *k, *v;
  int64_t k_token, k_head, v_token, v_head;
  const int32_t *begin, *length, *table;
  int32_t tokens, log_page, log_vec;   // log2 of the page and of the 16-byte pieces of a row of 16-bit values
};

// The rows of one page and head.  Grid: slots (see slot_sequence; the new rows of a sequence touch at most rows / page + 2 pages), heads.
template <bool BF16>
__global__ void __launch_bounds__(NT) pages_write_kernel(const __grid_constant__ WriteParams P) {
  __shared__ uint32_t sh_top[NT / 32];
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
  for (int h = 0; h < HELD; ++h) top = max(top, top8<BF16>(held[h]));
  for (int i = tid + HELD * SIDE; i < vecs; i += SIDE) top = max(top, top8<BF16>(load(i)));
  top = __reduce_max_sync(0xffffffffu, top);
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
      uint4 v = reinterpret_cast<uint4*>(codes)[i];
      uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t r = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) r |= (uint32_t)(unsigned char)code_of((float)(signed char)(w[q] >> (8 * b)), ratio) << (8 * b);
        w[q] = r;
      }
      reinterpret_cast<uint4*>(codes)[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  auto store = [&](int i, const uint4& v) {
    float x[8];
    unpack8<BF16>(v, x);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e >> 2] |= (uint32_t)(unsigned char)code_of(scale == scale ? x[e] : 0.f, inverse) << (8 * (e & 3));
    *reinterpret_cast<uint2*>(codes + ((size_t)r0 << (P.log_vec + 3)) + (size_t)i * 8) = make_uint2(w[0], w[1]);
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
  int32_t tokens, log_page, log_vec;
};

template <bool BF16>
__global__ void __launch_bounds__(NT) pages_read_kernel(const __grid_constant__ ReadParams P) {
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
  const uint2* codes = reinterpret_cast<const uint2*>(c.codes + (tile * c.page + (size_t)(lo - first_token)) * c.d);
  unsigned short* dst = static_cast<unsigned short*>(side ? P.v : P.k) + (from + (lo - start)) * (side ? P.v_token : P.k_token) +
                        (int64_t)blockIdx.y * (side ? P.v_head : P.k_head);
  const int64_t stride = side ? P.v_token : P.k_token;
  const int vecs = (int)(hi - lo) << P.log_vec;
#pragma unroll 4
  for (int i = tid; i < vecs; i += SIDE) {
    const uint2 w = held ? codes[i] : make_uint2(0, 0);
    uint32_t r[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t two = (p < 2 ? w.x : w.y) >> (16 * (p & 1));
      const float a = (float)(signed char)(two & 0xff) * scale, b = (float)(signed char)(two >> 8 & 0xff) * scale;
      if (BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        r[p] = *reinterpret_cast<const uint32_t*>(&h);
      } else {
        const __half2 h = __floats2half2_rn(a, b);
        r[p] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    *reinterpret_cast<uint4*>(dst + (int64_t)(i >> P.log_vec) * stride + (i & ((1 << P.log_vec) - 1)) * 8) = make_uint4(r[0], r[1], r[2], r[3]);
  }
}

// ---- kept rows to new pages.  Grid: pages of the new table, heads, sequences (folded into x where the other limits do not hold it).
struct CompactParams {
  PageCache c;
  const int32_t *table, *length, *keep, *n_keep, *new_table;
  int32_t keep_width, new_width, log_page;
};

__global__ void __launch_bounds__(NT) pages_compact_kernel(const __grid_constant__ CompactParams P) {
  __shared__ int64_t sh_row[128];             // where a row's K codes stand, -1: nowhere
  __shared__ float sh_scale[2][128];
  __shared__ uint32_t sh_top[2][4];
  const PageCache& c = P.c;
  const int s = blockIdx.x / P.new_width, j = blockIdx.x % P.new_width, h = blockIdx.y;
  const int kept = min(P.n_keep[s], P.keep_width);
  const int rows = min(kept - (j << P.log_page), c.page);
  if (rows <= 0) return;
  const int to = P.new_table[(size_t)s * P.new_width + j];
  if (to < 0 || to >= c.pages) return;
  if (threadIdx.x < 128) {
    float2 scale = make_float2(0.f, 0.f);
    int64_t at = -1;
    if ((int)threadIdx.x < rows) {
      const int token = P.keep[((size_t)s * c.Hkv + h) * P.keep_width + (j << P.log_page) + threadIdx.x];
      const int slot = token >> P.log_page;
      int id = -1;
      if (token >= 0 && token < P.length[s] && slot < c.W) id = P.table[(size_t)s * c.W + slot];
      if (id >= 0 && id < c.pages) {
        const size_t tile = ((size_t)id * c.Hkv + h) * 2;
        scale = *reinterpret_cast<const float2*>(c.scale + tile);
        at = (int64_t)(tile * c.page + (token & (c.page - 1))) * c.d;
      } else {
        scale = make_float2(nan_f32(), nan_f32());
      }
    }
    sh_row[threadIdx.x] = at;
    sh_scale[0][threadIdx.x] = scale.x;
    sh_scale[1][threadIdx.x] = scale.y;
    // scales carry no sign: their bits are in order, with NaN on top
    const uint32_t tk = __reduce_max_sync(0xffffffffu, __float_as_uint(scale.x)), tv = __reduce_max_sync(0xffffffffu, __float_as_uint(scale.y));
    if ((threadIdx.x & 31) == 0) { sh_top[0][threadIdx.x >> 5] = tk; sh_top[1][threadIdx.x >> 5] = tv; }
  }
  __syncthreads();
  const int side = threadIdx.x >= SIDE, tid = threadIdx.x & (SIDE - 1);
  uint32_t top = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = max(top, sh_top[side][w]);
  const float scale = __uint_as_float(top);
  const float inverse = scale > 0.f ? 1.f / scale : 0.f;
  const size_t tile = ((size_t)to * c.Hkv + h) * 2 + side;
  uint4* out = reinterpret_cast<uint4*>(c.codes + tile * (size_t)c.page * c.d);
  const int vec = c.d / 16;
#pragma unroll 4
  for (int i = tid; i < rows * vec; i += SIDE) {
    const int r = i / vec;
    const int64_t at = sh_row[r];
    uint4 v = make_uint4(0, 0, 0, 0);
    if (at >= 0) v = reinterpret_cast<const uint4*>(c.codes + at + (int64_t)side * c.page * c.d)[i - r * vec];
    const float own = sh_scale[side][r];
    if (own != scale) {                                          // also where either is NaN: the codes do not matter then
      const float ratio = own * inverse;
      uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t n = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) n |= (uint32_t)(unsigned char)code_of((float)(signed char)(w[q] >> (8 * b)), ratio) << (8 * b);
        w[q] = n;
      }
      v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    out[i] = v;
  }
  if (tid == 0) c.scale[tile] = scale;
}

// ---- tables.  One cluster of eight CTAs does the whole update: its barrier stands between counting references, looking for
// free pages and handing them out.  Every CTA works out the sequences' lengths and where each one's pages begin in the list for itself.
constexpr int CLUSTER = 8, UT = 1024;

struct UpdateShared {
  int owner[UPDATE_MAX_SEQUENCES];    // lowest sequence that goes on from this one
  int prefix[UPDATE_MAX_SEQUENCES];   // pages handed out to the sequences before
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
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < UT / 32; ++w) {
    const int t = warp_sums[w];
    before += w < warp ? t : 0;
    all += t;
  }
  total = all;
  return before + x - v;
}

struct Sequence {
  int parent, length, full, part, keeps, stay, need;   // stay: pages kept from the parent; need: pages in all
  int64_t beyond;                                      // pages the table has no room for
};

__global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(UT, 1) pages_update_kernel(const __grid_constant__ PagesUpdate U) {
  extern __shared__ __align__(16) unsigned char update_smem[];
  UpdateShared& sh = *reinterpret_cast<UpdateShared*>(update_smem);
  cg::cluster_group cluster = cg::this_cluster();
  const PageCache& c = U.c;
  const int S = c.S, W = c.W, rank = (int)cluster.block_rank(), tid = threadIdx.x;
  const int64_t capacity = (int64_t)W * c.page;

  auto parent_of = [&](int s) {
    const int p = U.parent ? U.parent[s] : s;
    return p >= 0 && p < S ? p : -1;
  };
  auto look = [&](int s) {
    Sequence q{};
    q.parent = parent_of(s);
    q.length = q.parent >= 0 ? U.length[q.parent] : 0;
    if (q.length < 0 || q.length > capacity) q.length = 0;
    q.full = q.length / c.page;
    q.part = q.length - q.full * c.page;
    q.keeps = q.part > 0 && sh.owner[q.parent] == s;             // a part-filled page implies a parent
    q.stay = q.full + q.keeps;
    const int64_t tokens = (int64_t)q.length + max(U.grow ? U.grow[s] : U.grow_all, 0);
    const int64_t need = (tokens + c.page - 1) / c.page;
    q.need = (int)min(need, (int64_t)W);
    q.beyond = need - q.need;
    return q;
  };

  // ---- who keeps a page that is filled in part; pages to hand out before each sequence
  for (int s = tid; s < S; s += UT) sh.owner[s] = S;
  if (tid == 0) sh.beyond = 0;
  __syncthreads();
  for (int s = tid; s < S; s += UT) {
    const int p = parent_of(s);
    if (p >= 0) atomicMin(&sh.owner[p], s);
  }
  __syncthreads();
  int wanted = 0;                                                // pages to hand out, of all sequences
  for (int base = 0; base < S; base += UT) {
    const int s = base + tid;
    int fresh = 0;
    if (s < S) {
      const Sequence q = look(s);
      fresh = q.need - q.stay;
      if (q.beyond) atomicAdd(&sh.beyond, (unsigned long long)q.beyond);
    }
    int total;
    const int before = block_exclusive(fresh, sh.scan, total);
    if (s < S) sh.prefix[s] = wanted + before;
    wanted += total;
  }

  // ---- references: what the table names now no longer counts, what stays does
  const uint32_t entries = (uint32_t)S * (uint32_t)W;            // at most 2^28
  const uint32_t thread = (uint32_t)(rank * UT + tid), threads = CLUSTER * UT;
  for (uint32_t i = thread; i < entries; i += threads) {
    const int s = (int)(i / (uint32_t)W), j = (int)(i - (uint32_t)s * (uint32_t)W);
    const Sequence q = look(s);
    const int old = U.table[i];
    int next = -1;
    if (j < q.stay || (j == q.full && q.part > 0)) next = q.parent == s ? old : U.table[(int64_t)q.parent * W + j];
    if (next < 0 || next >= c.pages) next = -1;
    if (j == q.full && q.part > 0) U.copies[s].x = next;         // the page that is filled in part
    if (j >= q.stay) next = -1;
    U.fresh_rows[i] = next;
    if (next != old) {
      if (old >= 0 && old < c.pages) atomicSub(&U.refs[old], 1);
      if (next >= 0) atomicAdd(&U.refs[next], 1);
    }
  }
  __threadfence();
  cluster.sync();

  // ---- free pages, lowest first: counted per CTA, then listed
  const int per = ((c.pages + CLUSTER - 1) / CLUSTER + 3) & ~3;  // a CTA's stretch of pages
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
  int mine = 0;
  if (wanted > 0)
    for (int p = lo + tid * 4; p < hi; p += UT * 4) mine += __popc(free_mask(p));
  int total;
  (void)block_exclusive(mine, sh.scan, total);
  if (tid == 0) sh.found = total;
  cluster.sync();
  int rank_before = 0, available = 0;
  for (int r = 0; r < CLUSTER; ++r) {
    const int n = *cluster.map_shared_rank(&sh.found, r);
    rank_before += r < rank ? n : 0;
    available += n;
  }
  const int given = min(wanted, available);
  for (int base = lo; base < hi && rank_before < given; base += UT * 4) {
    const int p = base + tid * 4;
    const uint32_t m = p < hi ? free_mask(p) : 0;
    int at = block_exclusive(__popc(m), sh.scan, total) + rank_before;
    for (int e = 0; e < 4; ++e)
      if (m >> e & 1) {
        if (at < given) { U.free_list[at] = p + e; U.refs[p + e] = 1; }
        ++at;
      }
    rank_before += total;
  }
  __threadfence();
  cluster.sync();

  // ---- the new table
  for (uint32_t i = thread; i < entries; i += threads) {
    const int s = (int)(i / (uint32_t)W), j = (int)(i - (uint32_t)s * (uint32_t)W);
    const Sequence q = look(s);
    int next = U.fresh_rows[i];
    if (j >= q.stay && j < q.need) {
      const int at = sh.prefix[s] + j - q.stay;
      next = at < given ? __ldcg(U.free_list + at) : -1;
    }
    U.table[i] = next;
    if (j == 0) {
      const bool copy = q.part > 0 && !q.keeps;
      const int at = sh.prefix[s];                               // its first new page
      const int from = copy ? __ldcg(&U.copies[s].x) : -1;
      U.copies[s] = make_int4(from, copy && at < given ? __ldcg(U.free_list + at) : -1, q.part, 0);
    }
  }
  // lengths are read by every look(): written when all CTAs are done with them
  int mine_length[UPDATE_MAX_SEQUENCES / (CLUSTER * UT) + 1];
  int k = 0;
  for (int s = rank * UT + tid; s < S; s += CLUSTER * UT) mine_length[k++] = look(s).length;
  cluster.sync();
  k = 0;
  for (int s = rank * UT + tid; s < S; s += CLUSTER * UT) U.length[s] = mine_length[k++];
  if (rank == 0 && tid == 0) *U.missing = (int)min((int64_t)(wanted - given) + (int64_t)sh.beyond, (int64_t)INT32_MAX);
}

// The rows of pages that are filled in part.  Grid: sequences, layers, pieces of the heads.
__global__ void __launch_bounds__(NT) pages_copy_kernel(const __grid_constant__ PagesUpdate U) {
  const int4 copy = U.copies[blockIdx.x];
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

int log2_of(int x) { int n = 0; while ((1 << n) < x) ++n; return n; }

}  // namespace

cudaError_t launch_pages_write(const PageCache& c, const PageRows& r, const int32_t* begin, const int32_t* length, const int32_t* table, cudaStream_t stream) {
  WriteParams P{};
  P.c = c; P.k = r.k; P.v = r.v; P.k_token = r.k_token; P.k_head = r.k_head; P.v_token = r.v_token; P.v_head = r.v_head;
  P.begin = begin; P.length = length; P.table = table; P.tokens = r.tokens;
  P.log_page = log2_of(c.page); P.log_vec = log2_of(c.d / 8);
  const unsigned slots = begin ? (unsigned)((r.tokens >> P.log_page) + 2 * c.S) : (unsigned)c.S;
  const dim3 grid(slots, (unsigned)c.Hkv);
  if (r.bf16) pages_write_kernel<true><<<grid, NT, 0, stream>>>(P);
  else pages_write_kernel<false><<<grid, NT, 0, stream>>>(P);
  return cudaGetLastError();
}

cudaError_t launch_pages_read(const PageCache& c, const PageRows& r, const int32_t* begin, const int32_t* first, const int32_t* table, cudaStream_t stream) {
  ReadParams P{};
  P.c = c; P.k = r.k; P.v = r.v; P.k_token = r.k_token; P.k_head = r.k_head; P.v_token = r.v_token; P.v_head = r.v_head;
  P.begin = begin; P.first = first; P.table = table; P.tokens = r.tokens;
  P.log_page = log2_of(c.page); P.log_vec = log2_of(c.d / 8);
  const dim3 grid((unsigned)((r.tokens >> P.log_page) + 2 * c.S), (unsigned)c.Hkv);
  if (r.bf16) pages_read_kernel<true><<<grid, NT, 0, stream>>>(P);
  else pages_read_kernel<false><<<grid, NT, 0, stream>>>(P);
  return cudaGetLastError();
}

cudaError_t launch_pages_compact(const PageCache& c, int keep_width, int new_width, const int32_t* table, const int32_t* length, const int32_t* keep,
                                 const int32_t* n_keep, const int32_t* new_table, cudaStream_t stream) {
  CompactParams P{};
  P.c = c; P.table = table; P.length = length; P.keep = keep; P.n_keep = n_keep; P.new_table = new_table;
  P.keep_width = keep_width; P.new_width = new_width; P.log_page = log2_of(c.page);
  pages_compact_kernel<<<dim3((unsigned)c.S * (unsigned)new_width, (unsigned)c.Hkv), NT, 0, stream>>>(P);
  return cudaGetLastError();
}

cudaError_t launch_pages_update(const PagesUpdate& u, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(pages_update_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(UpdateShared));
  if (e != cudaSuccess) return e;
  pages_update_kernel<<<CLUSTER, UT, sizeof(UpdateShared), stream>>>(u);
  e = cudaGetLastError();
  if (e != cudaSuccess || !u.parent) return e;                    // without parents no page has a second owner
  const int pieces = u.c.Hkv * 2 < 8 ? u.c.Hkv * 2 : 8;
  pages_copy_kernel<<<dim3((unsigned)u.c.S, (unsigned)u.layers, (unsigned)pieces), NT, 0, stream>>>(u);
  return cudaGetLastError();
}

}  // namespace kf
