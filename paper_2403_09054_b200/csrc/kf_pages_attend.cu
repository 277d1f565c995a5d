// Attention of one query token per sequence over its 8-bit pages (kf_pages_attend): out = sum_j softmax_j(x_j) v_j in one pass.
//
// Memory bounds it: 2 d bytes per cached token and key/value head, which all query heads of the group share (up to eight per CTA; larger
// groups take more CTAs, which meet in L2).  At the copy rate an SM gets 23 bytes a cycle, so per byte there is room for little
// arithmetic, and both products run on the tensor pipe as m16n8k16 instructions: S = q K^T with the query heads as rows 0-7 and tokens as
// columns, O = P V with P's two binary16 parts (the weight rounded, and what the rounding left out) as rows 0-7 and 8-15, so that only
// the output is rounded.  Codes become binary16 integers (exact) in registers on their way from shared memory; an operand of tcgen05
// would have to be written back there first.  A product may take its terms in any order: a lane contracts the features (S) or
// tokens (O) that its own wide loads bring, and S comes out in the layout in which P goes in, so that no logit passes through shared memory.
//
// Work is split by tiles: those of all (sequence, key/value head, block of query heads) units stand one after the other, and every warp of one wave
// of CTAs gets the same number of consecutive ones, whatever the lengths are (the host does not know them: every CTA adds them up).
// Within a unit tiles go from the newest token back: with ALiBi the nearest keys have the largest logits, so that a reference hardly ever moves (32 x 32
// caches of 4096 tokens 205 -> 196 us, of d 256 460 -> 417).  A warp walks its share with a private ring of tiles that TMA fills with swizzled rows (both
// products' loads are then free of bank conflicts), across the borders of units.  A unit that lies within one share is written by its warp; others leave a partial
// result per warp, which pages_merge_kernel joins.  (Chunks of one sequence per CTA instead: 271 against 210 us for 32 x 32 caches of 4096 tokens, whose SMs
// idled for 40 %.)
//
// What bounds it: 32 x 32 caches of 4096 tokens (1.07 GB) take 187 to 198 us, 5.4 to 5.7 TB/s of 6.57; the same loads without any arithmetic take 169.  45 % of the issue
// slots are used (750 warp instructions per 32 tokens of d 128, 416 of them conversions), and the registers allow eight warps, whose products of several groups of tokens the compiler
// may then mix; twelve of 168 registers, one group of tokens after the other, take as long for many caches and more where a share is short (one sequence of 131072
// tokens on 8 caches 67 instead of 62 us, 256 of 512 69 instead of 64, units of 74 sequences of 500 24 instead of 18), but for d 64 less (126 instead of 138).  48
// sequences of up to 8192 tokens on 8 caches: 83 to 90 us, 75 without arithmetic, 61 at the copy rate.  Not taken, for 32 x 32 caches: 16 warps of 128 registers and tiles of 16
// tokens (290), the table's entries ahead of time by asynchronous copies (198), larger shares for the CTAs that an SM takes first (194 to 199), a record per unit
// instead of per share for the second kernel (193), packed binary32 arithmetic in the softmax (as many instructions, the pairs have to be moved together), sums that are
// corrected for the codes' offset at the end (they would lose the last eleven bits).
#include "kf_pages.cuh"
#include "kf_tc.cuh"

namespace kf {

namespace {

constexpr int NW = 4, NT = NW * 32;
constexpr int GB = 8;                       // query heads of a unit
constexpr int SMS = 148;
constexpr int LEAST = 2;                    // tiles of a share
constexpr int ENTRIES = 256;                // of a CTA's table of where sequences begin (one per sequence up to 256 of them)
constexpr int BATCH = 16;                   // tiles a warp looks up at a time
constexpr int MERGE_WARPS = 8;
constexpr float FIRST_REF = -3.402823466e38f;   // no finite logit lies below
constexpr float LEAST_REF = -1e30f;         // of a reference that counts from another one: 2^this is nothing, and sums with it stay finite
constexpr float ROOM = 7.0f, GAP = 8.0f;    // weights are taken times 2^7 (binary16 holds 2^-32 to 2^8 of the reference); a reference moves by 2^8

template <int D>
struct Shape {
  static constexpr int TILE = D == 256 ? 16 : 32;           // tokens
  static constexpr int BYTES = 2 * TILE * D;                // K and V
  static constexpr int STAGES = D == 64 ? 16384 / BYTES : 3;   // per warp
  static constexpr int HEAD = 8 * (D / 8 + 4) + 4;          // floats between two heads' sums in shared memory: spread over the banks
  static constexpr int RESIDENT = D == 64 ? 3 : 2;          // CTAs of an SM, by registers (168 or 255 a thread); all of them are the wave
};

// What a warp knows of a tile before it comes to it.
struct __align__(16) Ahead {
  int at0, at1, rows, in_page;      // (page, head) of its page or pages (-1: the second holds no token); tokens from its first on, may exceed TILE; row
                                    // of its first token in its page
  float k0, v0, k1, v1;             // K scale times the logit scale, log2 of the V scale, of both pages
  int seq, unit, tile, count;       // sequence, unit within it, tile within that, tiles of the unit
};

struct AttendParams {
  CUtensorMap tm;             // [pages x Hkv x 2][page] rows of d bytes; boxes of min(d, 128) bytes x min(page, TILE) rows x K and V (one of them where a
                              // tile spans two pages), swizzled
  PagesAttend a;
  int32_t group, blocks;      // query heads per key/value head, and units they make up
  int32_t units;              // per sequence: key/value heads x blocks
  int32_t rows;               // query heads of a partial result
  int32_t log_page;
  float scale;                // logit scale * log2(e)
};

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same onto nothing.
__device__ __forceinline__ void mma0(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t h2(__half2 v) { return *reinterpret_cast<const uint32_t*>(&v); }
__device__ __forceinline__ __half2 b2(uint32_t v) { return *reinterpret_cast<const __half2*>(&v); }
// A pair of codes, moved to [b, x, b', x] by a byte permutation, as binary16 integers: 1024 + (c + 128) has the bits 0x6400 | (c ^ 0x80).
__device__ __forceinline__ uint32_t code_pair(uint32_t spread) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(r) : "r"(spread), "r"(0x00ff00ffu), "r"(0x64806480u));   // (a & b) ^ c
  return h2(__hadd2(b2(r), b2(0xe480e480u)));                                                               // - 1152
}

// Sum over the CTA of one number per thread, and the sum over the threads before.
__device__ __forceinline__ int cta_scan(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    before += w < warp ? warp_sums[w] : 0;
    total += warp_sums[w];
  }
  return before + x - v;
}

// SHARES: the form described above.  Without it a CTA is a unit, whose tiles its four warps take a quarter each, and joins them itself.
template <int D, bool SHARES>
__global__ void __launch_bounds__(NT, Shape<D>::RESIDENT) pages_attend_kernel(const __grid_constant__ AttendParams P) {
  using C = Shape<D>;
  constexpr int TILE = C::TILE, ST = C::STAGES;
  constexpr int GROUPS = TILE / 8;              // groups of eight tokens, the columns of one S product
  constexpr int KW = D / 16;                    // words of K codes a lane holds per token: its quarter of the features
  constexpr int ROWB = D < 128 ? D : 128;       // bytes of a shared-memory row
  constexpr int VALUES = TILE * ROWB;           // a slot: K rows, V rows, of the first 128 features, then of the others
  constexpr int COLS = 2 * TILE * ROWB;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t bars_all[NW][ST];
  __shared__ int sh_sums[NW], sh_begin[ENTRIES + 1];
  __shared__ Ahead sh_ahead[NW][2 * BATCH];
  __shared__ float2 sh_ml[NW][GB];

  after_earlier_kernels();
  let_next_kernel_launch();
  const PagesAttend& a = P.a;
  const PageCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r8 = lane >> 2, t4 = lane & 3;
  const int capacity = c.W << P.log_page;
  auto tiles_of = [&](int s) {
    const int n = s < c.S ? a.length[s] : 0;
    return n > 0 && n <= capacity ? (n + TILE - 1) / TILE : 0;
  };

  // ---- where the sequences begin, in tiles: an entry for every `stride` sequences
  const int stride = (c.S + ENTRIES - 1) / ENTRIES;
  int all = 0;
  if (SHARES) {
    constexpr int PER = ENTRIES / NT;
    int own[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      own[i] = 0;
      const int first = (tid * PER + i) * stride;
      if (first < c.S)
        for (int k = 0; k < stride; ++k) own[i] += tiles_of(first + k);
      sum += own[i];
    }
    int at = cta_scan(sum, sh_sums, all);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      sh_begin[tid * PER + i] = at;
      at += own[i];
    }
    if (tid == NT - 1) sh_begin[ENTRIES] = all;
  }
  if (SHARES) __syncthreads();
  const int own_seq = SHARES ? 0 : blockIdx.x / P.units, own_unit = SHARES ? 0 : blockIdx.x % P.units;
  const int total = SHARES ? all * P.units : tiles_of(own_seq), warps = SHARES ? gridDim.x * NW : NW;   // the host makes sure that there are fewer than 2^31 tiles
  const int share = max((int)(((uint32_t)total + warps - 1) / (uint32_t)warps), SHARES ? LEAST : 1);
  const int me = SHARES ? blockIdx.x * NW + warp : warp;
  const int from = (int)min((int64_t)me * share, (int64_t)total);
  // ---- sequences without tiles: zeros, or NaN where the length is not valid
  for (int i = SHARES ? me : own_seq; i < c.S; i += SHARES ? warps : c.S) {
    if (!SHARES && (own_unit != 0 || warp != 0)) break;
    const int n = a.length[i];
    if (n > 0 && n <= capacity) continue;
    const uint32_t v = n == 0 ? 0u : 0x7fff7fffu;
    for (int e = lane; e < a.H * (D / 8); e += 32)
      *reinterpret_cast<uint4*>(static_cast<unsigned short*>(a.out) + (int64_t)i * a.out_sequence + (int64_t)(e / (D / 8)) * a.out_head + e % (D / 8) * 8) = make_uint4(v, v, v, v);
  }
  if (SHARES && lane == 0) a.splits[2 * me].x = -1;   // no unit begins in this share and goes on behind it, as far as is known
  if (SHARES ? from >= total : total == 0) return;
  const int mine = min(share, total - from);          // tiles of this warp

  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* ring = smem + (size_t)warp * ST * C::BYTES;
  uint64_t* bars = bars_all[warp];
  if (lane == 0) {
    for (int i = 0; i < ST; ++i) mbar_init(bars + i, 1);
    mbar_fence_init();
  }
  __syncwarp();

  // ---- the tiles of the share, looked up 16 at a time by as many lanes
  const bool two = TILE > 16 && P.log_page == 4;      // a tile spans two pages
  Ahead* ahead = sh_ahead[warp];
  auto page_of = [&](int s, int kv, int slot, int& at, float& ks, float& vs) {
    int id = a.table[(size_t)s * c.W + slot];
    const bool bad = id < 0 || id >= c.pages;
    if (bad) id = 0;
    const float2 sc = *reinterpret_cast<const float2*>(c.scale + ((size_t)id * c.Hkv + kv) * 2);
    ks = bad ? nan_f32() : sc.x * P.scale;            // a page that is missing: the output is NaN
    vs = bad ? nan_f32() : log2f(sc.y);
    at = id * c.Hkv + kv;
  };
  bool failed = false;
  auto look_up = [&](int w0) {
    if (w0 == a.fail_at) failed = true;               // the self-test: as if the next wait had run out
    if (lane < BATCH && w0 + lane < mine) {
      Ahead t;
      if (SHARES) {
        const int g = from + w0 + lane, in_all = (int)((uint32_t)g / (uint32_t)P.units);
        int lo = 0, hi = ENTRIES;                     // the last entry that does not begin behind it
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (sh_begin[mid] <= in_all) lo = mid; else hi = mid;
        }
        int at = sh_begin[lo];
        t.seq = lo * stride;
        t.count = stride == 1 ? sh_begin[lo + 1] - at : tiles_of(t.seq);
        while (at + t.count <= in_all) { at += t.count; t.count = tiles_of(++t.seq); }
        const int r = g - at * P.units;
        t.unit = (int)((uint32_t)r / (uint32_t)t.count);
        t.tile = r - t.unit * t.count;
      } else {
        t.seq = own_seq;
        t.unit = own_unit;
        t.count = total;
        t.tile = from + w0 + lane;
      }
      const int token = (t.count - 1 - t.tile) * TILE, kv = t.unit / P.blocks;
      t.rows = a.length[t.seq] - token;
      page_of(t.seq, kv, token >> P.log_page, t.at0, t.k0, t.v0);
      t.in_page = token & (c.page - 1);
      t.at1 = -1;
      t.k1 = t.v1 = 0.f;
      if (two && t.rows > 16) page_of(t.seq, kv, (token >> P.log_page) + 1, t.at1, t.k1, t.v1);
      ahead[(w0 + lane) & (2 * BATCH - 1)] = t;
    }
    __syncwarp();
  };
  auto issue = [&](int w) {                           // tile w into its slot of the ring
    if (lane == 0) {
      const int4 at = *reinterpret_cast<const int4*>(&ahead[w & (2 * BATCH - 1)]);
      uint64_t* bar = bars + w % ST;
      unsigned char* dst = ring + (w % ST) * C::BYTES;
      mbar_expect_tx(bar, two && at.y < 0 ? C::BYTES / 2 : C::BYTES);
      if (!two) {
#pragma unroll
        for (int b = 0; b < D / ROWB; ++b) tma_load_3d(dst + b * COLS, &P.tm, b * ROWB, at.w, 2 * at.x, bar);
      } else {
        tma_load_3d(dst, &P.tm, 0, 0, 2 * at.x, bar);
        tma_load_3d(dst + VALUES, &P.tm, 0, 0, 2 * at.x + 1, bar);
        if (at.y >= 0) {
          tma_load_3d(dst + 16 * ROWB, &P.tm, 0, 0, 2 * at.y, bar);
          tma_load_3d(dst + VALUES + 16 * ROWB, &P.tm, 0, 0, 2 * at.y + 1, bar);
        }
      }
    }
  };
  look_up(0);
  for (int w = 0; w < ST; ++w)
    if (w < mine) issue(w);

  int w = 0, failed_at = mine;                        // the first tile that was not waited for
  while (SHARES ? w < mine : w == 0) {                // without shares once, even by a warp without tiles
    // ---- a unit, or the part of it that lies in this share
    const int4 where = SHARES ? *reinterpret_cast<const int4*>(&ahead[w & (2 * BATCH - 1)].seq) : make_int4(own_seq, own_unit, from, total);
    const int s = where.x, y = where.y, first = where.z, tiles = where.w;
    const int begun = w, end = min(mine, w + tiles - first);
    const bool whole = SHARES && first == 0 && w + tiles <= mine;
    const int kv = y / P.blocks, block = y - kv * P.blocks;
    const int heads = min(GB, P.group - block * GB), head0 = kv * P.group + block * GB, head = head0 + min(r8, heads - 1);

    // queries as the first operand of S: row = head r8, the quarter t4 of the features, four of them per step in the order 0, 2, 1, 3
    uint32_t q0[KW], q1[KW];
    float q_power;
    {
      const unsigned short* q = static_cast<const unsigned short*>(a.q) + (int64_t)s * a.q_sequence + (int64_t)head * a.q_head + t4 * (D / 4);
#pragma unroll
      for (int i = 0; i < KW; i += 2) {
        const uint4 v = *reinterpret_cast<const uint4*>(q + 4 * i);
        q0[i] = v.x; q1[i] = v.y;
        q0[i + 1] = v.z; q1[i + 1] = v.w;
      }
      int e = 0;
      if (a.bf16) {
        // bfloat16 to binary16 after a division by a power of two that brings the head's largest feature to [1, 2): exact down to 2^-17 of it (8 bits above
        // the last place of 2^-24), below that rounded to multiples of 2^-24.  The power goes back into the logit scale.
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < KW; ++i)
          top = max(max(top, max(q0[i] & 0x7fffu, q1[i] & 0x7fffu)), max(q0[i] >> 16 & 0x7fffu, q1[i] >> 16 & 0x7fffu));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        e = min(max((int)(top >> 7), 1), 253) - 127;
        const float down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
        for (int i = 0; i < KW; ++i) {
          q0[i] = h2(__floats2half2_rn(__uint_as_float(q0[i] << 16) * down, __uint_as_float(q0[i] & 0xffff0000u) * down));
          q1[i] = h2(__floats2half2_rn(__uint_as_float(q1[i] << 16) * down, __uint_as_float(q1[i] & 0xffff0000u) * down));
        }
      }
#pragma unroll
      for (int i = 0; i < KW; ++i) {
        const uint32_t x = q0[i], z = q1[i];
        q0[i] = __byte_perm(x, z, 0x5410);
        q1[i] = __byte_perm(x, z, 0x7632);
      }
      q_power = __uint_as_float((uint32_t)(127 + e) << 23);
    }
    const float slope = a.slopes ? a.slopes[head] * LOG2E : 0.f;

    // Of head r8: the reference of the logits, and of weights times V scales as it counts from that (so that it is a small number wherever the
    // logits lie, and loses nothing beside them), both common to its four lanes; l: this lane's tokens.
    float m_x = FIRST_REF, m_o = 0.f, l = 0.f;
    float o[D / 8][4];
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0.f;

    for (; w < end; ++w) {
      const int rows = ahead[w & (2 * BATCH - 1)].rows;
      const float4 scales = *reinterpret_cast<const float4*>(&ahead[w & (2 * BATCH - 1)].k0);
      const float k0 = scales.x * q_power, v0 = scales.y;
      float k1 = k0, v1 = v0;
      if (two && rows > 16) { k1 = scales.z * q_power; v1 = scales.w; }
      const unsigned char* buf = ring + (w % ST) * C::BYTES;
      if (!failed && !__all_sync(0xffffffffu, mbar_wait_bounded(bars + w % ST, (uint32_t)(w / ST & 1)))) failed = true;
      if (failed) {                                   // nothing more is asked for; the units of the share still have to be gone through
        failed_at = min(failed_at, w);
        if ((w + ST) % BATCH == 0 && w + ST < mine) look_up(w + ST);
        continue;
      }

      // ---- logits: column = token r8 of a group, this lane's quarter of the features
      float x[GROUPS][2];
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int row = g * 8 + r8;
        uint32_t kw[KW];
        if (D == 64) {
          const uint4 v = *reinterpret_cast<const uint4*>(buf + row * 64 + ((t4 ^ (row >> 1 & 3)) << 4));
          kw[0] = v.x; kw[1] = v.y; kw[2] = v.z; kw[3] = v.w;
        } else {
          // 16-byte pieces t4 D/64 + i of the row; those of 256-byte rows lie in two boxes
#pragma unroll
          for (int i = 0; i < KW / 4; ++i) {
            const int piece = t4 * (KW / 4) + i;
            const uint4 v = *reinterpret_cast<const uint4*>(buf + (piece >> 3) * COLS + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
            kw[4 * i] = v.x; kw[4 * i + 1] = v.y; kw[4 * i + 2] = v.z; kw[4 * i + 3] = v.w;
          }
        }
        float sum[4];
#pragma unroll
        for (int i = 0; i < KW; ++i) {
          if (i == 0) mma0(sum, q0[i], 0u, q1[i], 0u, code_pair(kw[i]), code_pair(kw[i] >> 8));
          else mma(sum, q0[i], 0u, q1[i], 0u, code_pair(kw[i]), code_pair(kw[i] >> 8));
        }
        const float kf = g >= 2 ? k1 : k0;
        x[g][0] = sum[0] * kf;
        x[g][1] = sum[1] * kf;
        if (D == 64) asm volatile("" ::: "memory");   // the next group's loads stay behind: registers
      }
      // head r8, tokens 8 g + 2 t4 and + 1
      if (a.slopes) {
        const float back = (float)(2 * t4 + 1 - rows);   // from the newest token to this one
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          x[g][0] = fmaf(slope, back + (float)(8 * g), x[g][0]);
          x[g][1] = fmaf(slope, back + (float)(8 * g + 1), x[g][1]);
        }
      }
      if (rows < TILE) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          if (8 * g + 2 * t4 >= rows) x[g][0] = -INFINITY;
          if (8 * g + 2 * t4 + 1 >= rows) x[g][1] = -INFINITY;
        }
      }
      // ---- references: of the softmax, and of the weights times the V scale of their page
      float tx0 = -INFINITY, tx1 = -INFINITY;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        if (g >= 2) tx1 = max3(tx1, x[g][0], x[g][1]);
        else tx0 = max3(tx0, x[g][0], x[g][1]);
      }
      const float tx = fmaxf(tx0, tx1), to = fmaxf(tx0 - m_x + v0, tx1 - m_x + v1);
      if (__any_sync(0xffffffffu, tx > m_x + GAP || to > m_o + GAP)) {
        float nx = tx;
        nx = fmaxf(nx, __shfl_xor_sync(0xffffffffu, nx, 1));
        nx = fmaxf(nx, __shfl_xor_sync(0xffffffffu, nx, 2));
        nx = fmaxf(nx, m_x);
        const float grown = nx - m_x, before = fmaxf(m_o - grown, LEAST_REF);     // grown may be infinite the first time
        m_x = nx;
        float no = fmaxf(tx0 - m_x + v0, tx1 - m_x + v1);
        no = fmaxf(no, __shfl_xor_sync(0xffffffffu, no, 1));
        no = fmaxf(no, __shfl_xor_sync(0xffffffffu, no, 2));
        m_o = fmaxf(no, before);
        l *= fast_exp2(-grown);
        const float f = fast_exp2(before - m_o);
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][e] *= f;
      }
      uint32_t hi[GROUPS], lo[GROUPS];
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const float x0 = x[g][0] - m_x, x1 = x[g][1] - m_x, up = (g >= 2 ? v1 : v0) - m_o + ROOM;
        l += fast_exp2(x0) + fast_exp2(x1);
        float p0 = fast_exp2(x0 + up), p1 = fast_exp2(x1 + up);
        if (rows < TILE) {                            // a masked token counts as nothing, whatever its page's scale is
          p0 = 8 * g + 2 * t4 < rows ? p0 : 0.f;
          p1 = 8 * g + 2 * t4 + 1 < rows ? p1 : 0.f;
        }
        const __half2 h = __floats2half2_rn(p0, p1);
        const float2 back = __half22float2(h);
        hi[g] = h2(h);
        lo[g] = h2(__floats2half2_rn(p0 - back.x, p1 - back.y));
      }
      // ---- values: column = feature r8 D/8 + i of product i, tokens 2 t4, + 1, + 8, + 9 of sixteen
#pragma unroll
      for (int k = 0; k < TILE / 16; ++k) {
        constexpr int VW = D / 32;                    // words of V codes per token: an eighth of the features
        uint32_t vw[4][VW];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = 16 * k + 2 * t4 + (e & 1) + 8 * (e >> 1);
          if (D == 64) {
            const uint2 v = *reinterpret_cast<const uint2*>(buf + VALUES + row * 64 + (((r8 >> 1) ^ (row >> 1 & 3)) << 4) + (r8 & 1) * 8);
            vw[e][0] = v.x; vw[e][1] = v.y;
          } else {
#pragma unroll
            for (int i = 0; i < VW / 4; ++i) {
              const int piece = r8 * (VW / 4) + i;
              const uint4 v = *reinterpret_cast<const uint4*>(buf + VALUES + (piece >> 3) * COLS + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
              vw[e][4 * i] = v.x; vw[e][4 * i + 1] = v.y; vw[e][4 * i + 2] = v.z; vw[e][4 * i + 3] = v.w;
            }
          }
        }
#pragma unroll
        for (int i = 0; i < VW; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            mma(o[4 * i + j], hi[2 * k], lo[2 * k], hi[2 * k + 1], lo[2 * k + 1], code_pair(__byte_perm(vw[0][i], vw[1][i], j | (4 + j) << 8)),
                code_pair(__byte_perm(vw[2][i], vw[3][i], j | (4 + j) << 8)));
        if (D == 64) asm volatile("" ::: "memory");
      }
      __syncwarp();                                   // the slot has been read by every lane
      if (w + ST < mine) {
        if ((w + ST) % BATCH == 0) look_up(w + ST);
        issue(w + ST);
      }
    }

    // ---- what the warp has of the unit.  Weights were taken against both references and times 2^7, their sum against m_x; the lane has two runs of D/8 features.
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (failed) l = nan_f32();
    // 2^m_o in two factors, the first a power of two: V scales may be as small as 2^-120 and references 2^-128, which the fast exponential takes for zero.
    const float low = floorf(0.5f * m_o), half = fast_exp2(low), bring = fast_exp2(m_o - low - ROOM) * (whole ? 1.f / l : 1.f);
    if (whole) {
      unsigned short* out = static_cast<unsigned short*>(a.out) + (int64_t)s * a.out_sequence + (int64_t)head * a.out_head + 2 * t4 * (D / 8);
      if (r8 < heads) {
#pragma unroll
        for (int run = 0; run < 2; ++run)
#pragma unroll
          for (int i = 0; i < D / 8; i += 8) {
            uint32_t r[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float u0 = (o[i + 2 * e][run] + o[i + 2 * e][run + 2]) * half * bring,
                          u1 = (o[i + 2 * e + 1][run] + o[i + 2 * e + 1][run + 2]) * half * bring;
              if (a.bf16) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(u0, u1);
                r[e] = *reinterpret_cast<const uint32_t*>(&b);
              } else {
                r[e] = h2(__floats2half2_rn(u0, u1));
              }
            }
            *reinterpret_cast<uint4*>(out + run * (D / 8) + i) = make_uint4(r[0], r[1], r[2], r[3]);
          }
      }
      continue;
    }
    // Where the unit covers all the CTA's shares, its warps' parts become one (a long sequence has hundreds of them).
    const int cta_from = from - warp * share, begins = from + begun - first, ends = begins + tiles;
    const bool joined = !SHARES || (begins <= cta_from && ends - cta_from >= NW * share);
    if (SHARES && first == 0 && lane == 0) {
      const uint32_t cta_share = NW * (uint32_t)share;
      a.splits[2 * me + 1] = make_int4((int)(((uint32_t)begins + cta_share - 1) / cta_share), (int)((uint32_t)ends / cta_share), 0, 0);
      a.splits[2 * me] = make_int4(head0, s, (int)((uint32_t)(ends - 1) / (uint32_t)share), heads);
    }
    float* part = a.partials + ((size_t)(me * 2 + (first == 0 ? 1 : 0)) * P.rows + r8) * (D + 4);
    float* at = joined ? reinterpret_cast<float*>(ring) + r8 * C::HEAD + 2 * t4 * (D / 8 + 4) : part + 2 * t4 * (D / 8);
    const int run_step = joined ? D / 8 + 4 : D / 8;
    if (r8 < heads) {
#pragma unroll
      for (int run = 0; run < 2; ++run)
#pragma unroll
        for (int i = 0; i < D / 8; i += 4)
          *reinterpret_cast<float4*>(at + run * run_step + i) =
              make_float4((o[i][run] + o[i][run + 2]) * half * bring, (o[i + 1][run] + o[i + 1][run + 2]) * half * bring,
                          (o[i + 2][run] + o[i + 2][run + 2]) * half * bring, (o[i + 3][run] + o[i + 3][run + 2]) * half * bring);
      if (t4 == 0) {
        if (joined) sh_ml[warp][r8] = make_float2(m_x, l);
        else *reinterpret_cast<float2*>(part + D) = make_float2(m_x, l);
      }
    }
    if (joined) {                                     // all four warps, each with this one part
      __syncthreads();
      part = a.partials + (size_t)(blockIdx.x * NW * 2 + (begins == cta_from ? 1 : 0)) * P.rows * (D + 4);
      for (int i = tid; i < heads * (D / 4); i += NT) {
        const int h = i / (D / 4), f = i % (D / 4) * 4;
        float top = FIRST_REF, sum = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int v = 0; v < NW; ++v) top = fmaxf(top, sh_ml[v][h].x);
#pragma unroll
        for (int v = 0; v < NW; ++v) {
          const float fo = fast_exp2(sh_ml[v][h].x - top);
          const float4 u = *reinterpret_cast<const float4*>(smem + (size_t)v * ST * C::BYTES + 4 * (h * C::HEAD + f / (D / 8) * (D / 8 + 4) + f % (D / 8)));
          acc.x = fmaf(u.x, fo, acc.x); acc.y = fmaf(u.y, fo, acc.y); acc.z = fmaf(u.z, fo, acc.z); acc.w = fmaf(u.w, fo, acc.w);
          sum = fmaf(sh_ml[v][h].y, fo, sum);
        }
        if (SHARES) {
          *reinterpret_cast<float4*>(part + h * (D + 4) + f) = acc;
          if (f == 0) *reinterpret_cast<float2*>(part + h * (D + 4) + D) = make_float2(top, sum);
        } else {
          const float by = 1.f / sum;
          uint2 r;
          if (a.bf16) {
            const __nv_bfloat162 b0 = __floats2bfloat162_rn(acc.x * by, acc.y * by), b1 = __floats2bfloat162_rn(acc.z * by, acc.w * by);
            r = make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
          } else {
            r = make_uint2(h2(__floats2half2_rn(acc.x * by, acc.y * by)), h2(__floats2half2_rn(acc.z * by, acc.w * by)));
          }
          *reinterpret_cast<uint2*>(static_cast<unsigned short*>(a.out) + (int64_t)s * a.out_sequence + (int64_t)(head0 + h) * a.out_head + f) = r;
        }
      }
    }
    if (!SHARES) break;
  }
  if (failed && mine > 0)                             // copies in flight get a second bounded wait
    for (int i = failed_at; i < min(failed_at + ST, mine); ++i) (void)mbar_wait_bounded(bars + i % ST, (uint32_t)(i / ST & 1));
}

// Joins the partial results of the units that more than one share has a part of.  A CTA per share in which such a unit begins: its eight warps are dealt
// out to the query heads, and the partial results of a head to its warps.
template <int D>
__global__ void __launch_bounds__(MERGE_WARPS * 32) pages_merge_kernel(const __grid_constant__ AttendParams P) {
  __shared__ float sh_o[MERGE_WARPS][D], sh_m[MERGE_WARPS], sh_l[MERGE_WARPS];
  after_earlier_kernels();
  let_next_kernel_launch();
  const PagesAttend& a = P.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, w0 = blockIdx.x;
  const int4 split = __ldcg(a.splits + 2 * w0);
  if (split.x < 0) return;
  // its parts: those of the shares w0 .. w1, of the CTAs c0 .. c1 - 1 one each
  const int4 ctas = __ldcg(a.splits + 2 * w0 + 1);
  const int w1 = split.z, heads = split.w, c0 = ctas.x, inner = max(ctas.y - c0, 0), lead = inner ? NW * c0 - w0 : 0;
  const int parts = w1 - w0 + 1 - inner * (NW - 1);
  const int per = MERGE_WARPS / heads, row = min(warp / per, heads - 1), part0 = warp - row * per;     // of 8 warps those behind the last head idle
  const bool used = warp < per * heads;
  constexpr int E = D / 32;
  float m = FIRST_REF, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  if (used) {
    constexpr int AT_ONCE = 4;
    for (int p = part0; p < parts; p += per * AT_ONCE) {
      float2 ml[AT_ONCE];
      float v[AT_ONCE][E];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        const int q = p + k * per, i = w0 + q + (q <= lead ? 0 : min(q - lead, inner) * (NW - 1));
        ml[k] = make_float2(FIRST_REF, 0.f);
        if (q < parts) {
          const float* part = a.partials + (((int64_t)i * 2 + (i == w0 ? 1 : 0)) * P.rows + row) * (D + 4);
          ml[k] = __ldcg(reinterpret_cast<const float2*>(part + D));
#pragma unroll
          for (int e = 0; e < E; ++e) v[k][e] = __ldcg(part + lane + 32 * e);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) v[k][e] = 0.f;
        }
      }
      float nm = m;
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) nm = fmaxf(nm, ml[k].x);
      const float fo = fast_exp2(m - nm);
      m = nm;
      l *= fo;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= fo;
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        const float fp = fast_exp2(ml[k].x - nm);
        l = fmaf(ml[k].y, fp, l);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(v[k][e], fp, o[e]);
      }
    }
  }
  if (lane == 0) { sh_m[warp] = m; sh_l[warp] = l; }
#pragma unroll
  for (int e = 0; e < E; ++e) sh_o[warp][lane + 32 * e] = o[e];
  __syncthreads();
  for (int i = threadIdx.x; i < heads * D; i += MERGE_WARPS * 32) {
    const int h = i / D, f = i - h * D;
    float top = FIRST_REF, acc = 0.f, sum = 0.f;
    for (int w = h * per; w < (h + 1) * per; ++w) top = fmaxf(top, sh_m[w]);
    for (int w = h * per; w < (h + 1) * per; ++w) {
      const float t = fast_exp2(sh_m[w] - top);
      acc = fmaf(sh_o[w][f], t, acc);
      sum = fmaf(sh_l[w], t, sum);
    }
    unsigned short* out = static_cast<unsigned short*>(a.out) + (int64_t)split.y * a.out_sequence + (int64_t)(split.x + h) * a.out_head + f;
    if (a.bf16) *reinterpret_cast<__nv_bfloat16*>(out) = __float2bfloat16_rn(acc / sum);
    else *reinterpret_cast<__half*>(out) = __float2half_rn(acc / sum);
  }
}

int blocks_of(int group) { return (group + GB - 1) / GB; }
// Tiles that the tables have room for, times units.
int64_t most_tiles(int S, int W, int page, int Hkv, int group, int d) {
  const int tile = d == 256 ? 16 : 32;
  return (int64_t)S * (((int64_t)W * page + tile - 1) / tile) * Hkv * blocks_of(group);
}
// CTAs of a launch: a wave, or fewer where all tables together could not keep it busy.
int ctas_of(int S, int W, int page, int Hkv, int group, int d) {
  const int64_t ctas = (most_tiles(S, W, page, Hkv, group, d) + NW * LEAST - 1) / (NW * LEAST);
  const int wave = SMS * (d == 64 ? Shape<64>::RESIDENT : Shape<128>::RESIDENT);
  return (int)(ctas < wave ? ctas : wave);
}

// Whether a CTA takes a unit: few units, none of which can have more than a few tiles.  The second kernel, which joins shares, then costs more than
// their even distribution saves: 8 caches of 64 / 256 / 512 / 768 tokens (d 128, four heads each) 3.7 / 4.9 / 6.9 / 8.9 us against 7.2 / 9.1 / 9.2 / 9.3, 592 caches
// of 256 / 768 tokens 12 / 29 against 16 / 31; but 8 of 1024 tokens 10.9 against 9.3, and 2048 of 64 / 256 tokens 26 / 43 against 14 / 38.
constexpr int FEW_TILES = 24, FEW_UNITS = 4 * SMS;
bool by_unit(const PageCache& c, int units) {
  const int tile = c.d == 256 ? 16 : 32;
  return ((int64_t)c.W * c.page + tile - 1) / tile <= FEW_TILES && (int64_t)c.S * units <= FEW_UNITS;
}

template <int D>
cudaError_t launch_attend_d(const AttendParams& P, cudaStream_t stream) {
  constexpr size_t smem = 1024 + (size_t)NW * Shape<D>::STAGES * Shape<D>::BYTES;
  static_assert(Shape<D>::RESIDENT * (smem + NW * 2 * BATCH * sizeof(Ahead) + 4 * (ENTRIES + 1 + NW) + 8 * NW * (GB + 4) + 1024) <= 228 * 1024,
                "shared memory of the CTAs that are to run at once");
  const PageCache& c = P.a.c;
  const bool units = by_unit(c, P.units);
  cudaError_t e = cudaFuncSetAttribute(units ? pages_attend_kernel<D, false> : pages_attend_kernel<D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  if (units) return launch_early(pages_attend_kernel<D, false>, dim3((unsigned)((int64_t)c.S * P.units)), NT, smem, stream, P);
  static_assert(GB * Shape<D>::HEAD * 4 <= Shape<D>::STAGES * Shape<D>::BYTES, "a warp's sums fit its ring");
  const int ctas = ctas_of(c.S, c.W, c.page, c.Hkv, P.group, D);
  e = launch_early(pages_attend_kernel<D, true>, dim3((unsigned)ctas), NT, smem, stream, P);
  return e != cudaSuccess ? e : launch_early(pages_merge_kernel<D>, dim3((unsigned)(ctas * NW)), MERGE_WARPS * 32, 0, stream, P);
}

}  // namespace

bool pages_attend_fits(const PageCache& c, int H) { return most_tiles(c.S, c.W, c.page, c.Hkv, H / c.Hkv, c.d) <= (int64_t)INT32_MAX; }
int pages_attend_shares(const PageCache& c, int H) { return ctas_of(c.S, c.W, c.page, c.Hkv, H / c.Hkv, c.d) * NW; }
size_t pages_attend_partials(const PageCache& c, int H) {
  const int group = H / c.Hkv, rows = group < GB ? group : GB;
  return (size_t)pages_attend_shares(c, H) * 2 * rows * (c.d + 4);
}

cudaError_t launch_pages_attend(const PagesAttend& a, cudaStream_t stream) {
  AttendParams P{};
  P.a = a;
  P.group = a.H / a.c.Hkv;
  P.blocks = blocks_of(P.group);
  P.units = a.c.Hkv * P.blocks;
  P.rows = P.group < GB ? P.group : GB;
  while ((1 << P.log_page) < a.c.page) ++P.log_page;
  P.scale = a.scale * LOG2E;
  const int D = a.c.d, tile = D == 256 ? 16 : 32;
  const uint64_t dims[3] = {(uint64_t)D, (uint64_t)a.c.page, (uint64_t)a.c.pages * a.c.Hkv * 2}, strides[2] = {(uint64_t)D, (uint64_t)a.c.page * D};
  const uint32_t box[3] = {(uint32_t)(D < 128 ? D : 128), (uint32_t)(a.c.page < tile ? a.c.page : tile), a.c.page < tile ? 1u : 2u};
  if (!make_tensor_map(&P.tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, a.c.codes, dims, strides, box, D == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorNotSupported;
  switch (D) {
    case 64: return launch_attend_d<64>(P, stream);
    case 128: return launch_attend_d<128>(P, stream);
    case 256: return launch_attend_d<256>(P, stream);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kf
