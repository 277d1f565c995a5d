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
// Work is split by tokens: the tiles of all sequences are dealt out in chunks of about the same size to one wave of CTAs, whatever the
// lengths are (the host does not know them: every CTA adds them up and finds its chunk).  The four warps of a CTA walk every fourth tile of the
// chunk, each with a private ring of tiles that TMA fills with swizzled rows (both products' loads are then free of bank conflicts).
// A chunk that is a whole sequence writes the output; others leave partial results that pages_merge_kernel joins.
#include "kf_pages.cuh"
#include "kf_tc.cuh"

namespace kf {

namespace {

constexpr int NW = 4, NT = NW * 32;
constexpr int GB = 8;                       // query heads of a CTA
constexpr int SMS = 148, RESIDENT = 3;      // CTAs that run at once: the size of a wave
constexpr float FIRST_REF = -1e30f;         // below every logit, but finite
constexpr float ROOM = 7.0f, GAP = 8.0f;    // weights are taken times 2^7 (binary16 holds 2^-32 to 2^8 of the reference); a reference moves by 2^8

template <int D>
struct Shape {
  static constexpr int TILE = D == 256 ? 16 : 32;           // tokens
  static constexpr int BYTES = 2 * TILE * D;                // K and V
  static constexpr int STAGES = 16384 / BYTES;              // per warp
  static constexpr int HEAD = 8 * (D / 8 + 4) + 4;          // floats between two heads' sums in shared memory: spread over the banks
};

struct AttendParams {
  CUtensorMap tm;             // rows of d bytes: [pages][Hkv][2][page]; boxes of min(page, TILE) rows x min(d, 128) bytes, swizzled
  PagesAttend a;
  int32_t group, blocks;      // query heads per key/value head, CTAs they take
  int32_t target;             // chunks aimed at, per (key/value head, block of query heads)
  int32_t log_page;
  float scale;                // logit scale * log2(e)
};

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t h2(__half2 v) { return *reinterpret_cast<const uint32_t*>(&v); }
__device__ __forceinline__ __half2 b2(uint32_t v) { return *reinterpret_cast<const __half2*>(&v); }
// A pair of codes, moved to [b, x, b', x] by a byte permutation, as binary16 integers: 1024 + (c + 128) has the bits 0x6400 | (c ^ 0x80).
__device__ __forceinline__ uint32_t code_pair(uint32_t spread) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(r) : "r"(spread), "r"(0x00ff00ffu), "r"(0x64806480u));   // (a & b) ^ c
  return h2(__hadd2(b2(r), b2(0xe480e480u)));                                                               // - 1152
}
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int c0, int c1, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1) : "memory");
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
  __syncthreads();
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

template <int D>
__global__ void __launch_bounds__(NT, RESIDENT) pages_attend_kernel(const __grid_constant__ AttendParams P) {
  using C = Shape<D>;
  constexpr int TILE = C::TILE, ST = C::STAGES;
  constexpr int GROUPS = TILE / 8;              // groups of eight tokens, the columns of one S product
  constexpr int KW = D / 16;                    // words of K codes a lane holds per token: its quarter of the features
  constexpr int ROWB = D < 128 ? D : 128;       // bytes of a shared-memory row
  constexpr int HALF = TILE * D;                // bytes of a K tile
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t bars_all[NW][ST];
  __shared__ float sh_m[NW][GB], sh_l[NW][GB], sh_o[NW][GB];
  __shared__ int sh_scan[NW], sh_at[4];

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const PagesAttend& a = P.a;
  const PageCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r8 = lane >> 2, t4 = lane & 3;
  const int capacity = c.W << P.log_page;
  auto tiles_of = [&](int s) {
    const int n = s < c.S ? a.length[s] : 0;
    return n > 0 && n <= capacity ? (n + TILE - 1) / TILE : 0;
  };

  // ---- this CTA's chunk: size from the tiles of all sequences, sequence from the chunks before
  int all = 0;
  {
    int mine = 0;
    for (int s = tid; s < c.S; s += NT) mine += tiles_of(s);
    (void)cta_scan(mine, sh_scan, all);
  }
  const int size = max((all + P.target - 1) / P.target, 2 * NW) + NW - 1 & ~(NW - 1);   // tiles of a chunk
  if (tid == 0) sh_at[0] = -1;
  int chunks_before = 0;
  for (int base = 0; base < c.S && chunks_before <= (int)blockIdx.x; base += NT) {
    const int s = base + tid, n = (tiles_of(s) + size - 1) / size;
    int total;
    const int first = chunks_before + cta_scan(n, sh_scan, total);
    if ((int)blockIdx.x >= first && (int)blockIdx.x < first + n) {
      sh_at[0] = s; sh_at[1] = (int)blockIdx.x - first; sh_at[2] = n; sh_at[3] = first;
    }
    chunks_before += total;
  }
  __syncthreads();
  const int s = sh_at[0];
  if (s < 0) return;
  const int chunk = sh_at[1], chunks = sh_at[2];
  const int kv = blockIdx.y / P.blocks, block = blockIdx.y % P.blocks;
  if (chunk == 0 && blockIdx.y == 0 && tid == 0) a.plan[s] = make_int2(sh_at[3], chunks);
  const int length = a.length[s];
  const int tile0 = chunk * size, tile_end = min(tile0 + size, (length + TILE - 1) / TILE);
  const int heads = min(GB, P.group - block * GB), head0 = kv * P.group + block * GB;

  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* ring = smem + (size_t)warp * ST * C::BYTES;
  uint64_t* bars = bars_all[warp];
  if (lane == 0) {
    for (int i = 0; i < ST; ++i) mbar_init(bars + i, 1);
    mbar_fence_init();
  }
  __syncwarp();

  // ---- pages of the warp's tiles, 32 tiles at a time, a lane one of them: tile w is tile0 + warp + w NW of the sequence
  const int mine = tile_end > tile0 + warp ? (tile_end - tile0 - warp + NW - 1) / NW : 0;
  const bool two = TILE > 16 && P.log_page == 4;      // a tile spans two pages
  int id0 = 0, id1 = 0;
  float ks0 = 0.f, ks1 = 0.f, vs0 = 0.f, vs1 = 0.f;   // K scale times the logit scale; log2 of the V scale
  auto page_of = [&](int slot, bool used, int& id, float& ks, float& vs) {
    id = used ? a.table[(size_t)s * c.W + slot] : 0;
    const bool bad = id < 0 || id >= c.pages;
    if (bad) id = 0;
    float2 sc = make_float2(0.f, 1.f);
    if (used) sc = *reinterpret_cast<const float2*>(c.scale + ((size_t)id * c.Hkv + kv) * 2);
    ks = sc.x * P.scale;
    vs = log2f(sc.y);
    if (bad) { ks = nan_f32(); vs = ks; }             // a page that is missing: the output is NaN
  };
  auto look_up = [&](int w0) {
    const int tile = tile0 + warp + (w0 + lane) * NW, token = tile * TILE;
    const bool used = w0 + lane < mine;
    page_of(token >> P.log_page, used, id0, ks0, vs0);
    if (two) page_of((token >> P.log_page) + 1, used && token + 16 < length, id1, ks1, vs1);
  };
  auto issue = [&](int w) {                           // tile w into its slot of the ring
    const int p0 = __shfl_sync(0xffffffffu, id0, w & 31), p1 = __shfl_sync(0xffffffffu, id1, w & 31);
    if (lane == 0) {
      const int token = (tile0 + warp + w * NW) * TILE;
      uint64_t* bar = bars + w % ST;
      unsigned char* dst = ring + (size_t)(w % ST) * C::BYTES;
      const int row = ((p0 * c.Hkv + kv) * 2 << P.log_page) + (token & (c.page - 1));
      mbar_expect_tx(bar, two && token + 16 >= length ? C::BYTES / 2 : C::BYTES);
#pragma unroll
      for (int b = 0; b < D / ROWB; ++b) {
        tma_load_2d(dst + b * TILE * ROWB, &P.tm, b * ROWB, row, bar);
        tma_load_2d(dst + HALF + b * TILE * ROWB, &P.tm, b * ROWB, row + c.page, bar);
      }
      if (two && token + 16 < length) {
        const int row1 = (p1 * c.Hkv + kv) * 2 << P.log_page;
        tma_load_2d(dst + 16 * ROWB, &P.tm, 0, row1, bar);
        tma_load_2d(dst + HALF + 16 * ROWB, &P.tm, 0, row1 + c.page, bar);
      }
    }
  };
  look_up(0);
  for (int w = 0; w < ST; ++w)
    if (w < mine) issue(w);

  // ---- queries as the first operand of S: row = head r8, the quarter t4 of the features, four of them per step
  uint32_t q0[KW], q1[KW];
  {
    const unsigned short* q = static_cast<const unsigned short*>(a.q) + (int64_t)s * a.q_sequence + (int64_t)(head0 + min(r8, heads - 1)) * a.q_head + t4 * (D / 4);
    float top = 0.f;
    uint2 raw[KW];
#pragma unroll
    for (int i = 0; i < KW; i += 2) {
      const uint4 v = *reinterpret_cast<const uint4*>(q + 4 * i);
      raw[i] = make_uint2(v.x, v.y);
      raw[i + 1] = make_uint2(v.z, v.w);
    }
    if (a.bf16) {
      // bfloat16 to binary16: exact after a division by a power of two that brings the head's largest feature to [1, 2), down to
      // 2^-24 of it.  The power goes back into the logit scale.
#pragma unroll
      for (int i = 0; i < KW; ++i) {
        const float f[4] = {__uint_as_float(raw[i].x << 16), __uint_as_float(raw[i].x & 0xffff0000u), __uint_as_float(raw[i].y << 16), __uint_as_float(raw[i].y & 0xffff0000u)};
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(f[e]));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    }
    const int e = a.bf16 ? min(max((int)(__float_as_uint(top) >> 23), 1), 253) - 127 : 0;
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
    for (int i = 0; i < KW; ++i) {
      if (a.bf16) {
        q0[i] = h2(__floats2half2_rn(__uint_as_float(raw[i].x << 16) * down, __uint_as_float(raw[i].x & 0xffff0000u) * down));
        q1[i] = h2(__floats2half2_rn(__uint_as_float(raw[i].y << 16) * down, __uint_as_float(raw[i].y & 0xffff0000u) * down));
      } else {
        q0[i] = raw[i].x;
        q1[i] = raw[i].y;
      }
    }
    top = __uint_as_float((uint32_t)(127 + e) << 23);
    sh_o[warp][r8] = top;                             // for later: the head's power of two (the same from four lanes)
  }
  __syncwarp();
  const float q_power = sh_o[warp][r8];
  const float slope = a.slopes ? a.slopes[head0 + min(r8, heads - 1)] * LOG2E : 0.f;

  float m_x = FIRST_REF, m_o = FIRST_REF, l = 0.f;    // of head r8, references common to its four lanes; l: this lane's tokens
  float o[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[i][e] = 0.f;

  // Scales of the tile that is worked on: `mine` may pass 32, then the next 32 pages are looked up before the first of them is fetched.
  float cur_k0 = ks0, cur_v0 = vs0, cur_k1 = ks1, cur_v1 = vs1;
  bool failed = a.fail_first_wait && mine > 0;
  int w = 0;
  for (; w < mine && !failed; ++w) {
    if ((w & 31) == 0 && w > 0) { cur_k0 = ks0; cur_v0 = vs0; cur_k1 = ks1; cur_v1 = vs1; }
    const float k0 = __shfl_sync(0xffffffffu, cur_k0, w & 31) * q_power, v0 = __shfl_sync(0xffffffffu, cur_v0, w & 31);
    float k1 = k0, v1 = v0;
    if (two) { k1 = __shfl_sync(0xffffffffu, cur_k1, w & 31) * q_power; v1 = __shfl_sync(0xffffffffu, cur_v1, w & 31); }
    const int token = (tile0 + warp + w * NW) * TILE;
    const int rows = length - token;                  // may exceed TILE
    const unsigned char* buf = ring + (size_t)(w % ST) * C::BYTES;
    const bool ok = mbar_wait_bounded(bars + w % ST, (uint32_t)(w / ST & 1));
    if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }

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
          const uint4 v = *reinterpret_cast<const uint4*>(buf + (piece >> 3) * (TILE * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
          kw[4 * i] = v.x; kw[4 * i + 1] = v.y; kw[4 * i + 2] = v.z; kw[4 * i + 3] = v.w;
        }
      }
      float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KW; i += 2) {
        mma(s0, q0[i], 0u, q1[i], 0u, code_pair(__byte_perm(kw[i], 0, 0x4140)), code_pair(__byte_perm(kw[i], 0, 0x4342)));
        mma(s1, q0[i + 1], 0u, q1[i + 1], 0u, code_pair(__byte_perm(kw[i + 1], 0, 0x4140)), code_pair(__byte_perm(kw[i + 1], 0, 0x4342)));
      }
      const float kf = g >= 2 ? k1 : k0;
      x[g][0] = (s0[0] + s1[0]) * kf;
      x[g][1] = (s0[1] + s1[1]) * kf;
    }
    // head r8, tokens 8 g + 2 t4 and + 1
    if (a.slopes) {
      const float back = (float)(token + 2 * t4 - (length - 1));
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
    const float tx = fmaxf(tx0, tx1), to = fmaxf(tx0 + v0, tx1 + v1);
    if (__any_sync(0xffffffffu, tx > m_x + GAP || to > m_o + GAP)) {
      float nx = tx, no = to;
      nx = fmaxf(nx, __shfl_xor_sync(0xffffffffu, nx, 1));
      no = fmaxf(no, __shfl_xor_sync(0xffffffffu, no, 1));
      nx = fmaxf(nx, __shfl_xor_sync(0xffffffffu, nx, 2));
      no = fmaxf(no, __shfl_xor_sync(0xffffffffu, no, 2));
      if (nx > m_x) { l *= fast_exp2(m_x - nx); m_x = nx; }
      const float f = no > m_o ? fast_exp2(m_o - no) : 1.f;
      if (no > m_o) m_o = no;
#pragma unroll
      for (int i = 0; i < D / 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] *= f;
    }
    uint32_t hi[GROUPS], lo[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      l += fast_exp2(x[g][0] - m_x) + fast_exp2(x[g][1] - m_x);
      const float up = (g >= 2 ? v1 : v0) - m_o + ROOM;
      float p0 = fast_exp2(x[g][0] + up), p1 = fast_exp2(x[g][1] + up);
      if (rows < TILE) {                              // a masked token counts as nothing, whatever its page's scale is
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
      constexpr int VW = D / 32;                      // words of V codes per token: an eighth of the features
      uint32_t vw[4][VW];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 16 * k + 2 * t4 + (e & 1) + 8 * (e >> 1);
        if (D == 64) {
          const uint2 v = *reinterpret_cast<const uint2*>(buf + HALF + row * 64 + (((r8 >> 1) ^ (row >> 1 & 3)) << 4) + (r8 & 1) * 8);
          vw[e][0] = v.x; vw[e][1] = v.y;
        } else {
#pragma unroll
          for (int i = 0; i < VW / 4; ++i) {
            const int piece = r8 * (VW / 4) + i;
            const uint4 v = *reinterpret_cast<const uint4*>(buf + HALF + (piece >> 3) * (TILE * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
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
    }
    __syncwarp();                                     // the slot has been read by every lane
    if (w + ST < mine) {
      if (((w + ST) & 31) == 0) look_up(w + ST);
      issue(w + ST);
    }
  }
  if (failed)
    for (int i = w; i < min(w + ST, mine); ++i) (void)mbar_wait_bounded(bars + i % ST, (uint32_t)(i / ST & 1));   // copies in flight

  // ---- join the lanes, then the warps; the sums lie in the ring, which is done with
  l += __shfl_xor_sync(0xffffffffu, l, 1);
  l += __shfl_xor_sync(0xffffffffu, l, 2);
  static_assert(GB * C::HEAD * 4 <= ST * C::BYTES, "a warp's sums fit its ring");
  __syncwarp();
  float* sums = reinterpret_cast<float*>(ring);
#pragma unroll
  for (int i = 0; i < D / 8; i += 4) {
    float* at = sums + r8 * C::HEAD + 2 * t4 * (D / 8 + 4) + i;
    *reinterpret_cast<float4*>(at) = make_float4(o[i][0] + o[i][2], o[i + 1][0] + o[i + 1][2], o[i + 2][0] + o[i + 2][2], o[i + 3][0] + o[i + 3][2]);
    *reinterpret_cast<float4*>(at + D / 8 + 4) = make_float4(o[i][1] + o[i][3], o[i + 1][1] + o[i + 1][3], o[i + 2][1] + o[i + 2][3], o[i + 3][1] + o[i + 3][3]);
  }
  if (t4 == 0) {
    sh_m[warp][r8] = m_x;
    sh_o[warp][r8] = m_o;
    sh_l[warp][r8] = failed ? nan_f32() : l;
  }
  __syncthreads();
  float* partial = a.partials + ((size_t)blockIdx.x * gridDim.y + blockIdx.y) * GB * (D + 2);
  for (int i = tid; i < heads * (D / 4); i += NT) {
    const int h = i / (D / 4), f = (i - h * (D / 4)) * 4;
    float mx = FIRST_REF, mo = FIRST_REF, lx = 0.f;
#pragma unroll
    for (int v = 0; v < NW; ++v) { mx = fmaxf(mx, sh_m[v][h]); mo = fmaxf(mo, sh_o[v][h]); }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const float fo = fast_exp2(sh_o[v][h] - mo);
      const float4 t = *reinterpret_cast<const float4*>(smem + (size_t)v * ST * C::BYTES + 4 * (h * C::HEAD + f / (D / 8) * (D / 8 + 4) + f % (D / 8)));
      acc.x = fmaf(t.x, fo, acc.x); acc.y = fmaf(t.y, fo, acc.y); acc.z = fmaf(t.z, fo, acc.z); acc.w = fmaf(t.w, fo, acc.w);
      lx = fmaf(sh_l[v][h], fast_exp2(sh_m[v][h] - mx), lx);
    }
    // weights were taken against mo and times 2^7, their sum against mx
    const float bring = fast_exp2(mo - mx - ROOM) * (chunks == 1 ? 1.f / lx : 1.f);
    acc.x *= bring; acc.y *= bring; acc.z *= bring; acc.w *= bring;
    if (chunks == 1) {
      unsigned short* out = static_cast<unsigned short*>(a.out) + (int64_t)s * a.out_sequence + (int64_t)(head0 + h) * a.out_head + f;
      uint2 r;
      if (a.bf16) {
        const __nv_bfloat162 b0 = __floats2bfloat162_rn(acc.x, acc.y), b1 = __floats2bfloat162_rn(acc.z, acc.w);
        r = make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
      } else {
        r = make_uint2(h2(__floats2half2_rn(acc.x, acc.y)), h2(__floats2half2_rn(acc.z, acc.w)));
      }
      *reinterpret_cast<uint2*>(out) = r;
    } else {
      *reinterpret_cast<float4*>(partial + h * D + f) = acc;
      if (f == 0) { partial[GB * D + 2 * h] = mx; partial[GB * D + 2 * h + 1] = lx; }
    }
  }
}

// Joins the chunks of a sequence, and says what a sequence without chunks gets.  Grid: sequences, query heads; four warps take the chunks in turn.
template <int D>
__global__ void __launch_bounds__(NT) pages_merge_kernel(const __grid_constant__ AttendParams P) {
  __shared__ float sh_o[NW][D], sh_m[NW], sh_l[NW];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const PagesAttend& a = P.a;
  const int s = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int length = a.length[s];
  const bool has = length > 0 && length <= a.c.W << P.log_page;
  const int2 plan = has ? a.plan[s] : make_int2(0, 0);
  if (has && plan.y == 1) return;
  const int kv = h / P.group, y = kv * P.blocks + (h - kv * P.group) / GB, row = (h - kv * P.group) % GB;
  constexpr int E = D / 32;
  float m = FIRST_REF, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int i = warp; i < plan.y; i += NW) {
    const float* part = a.partials + ((size_t)(plan.x + i) * (a.c.Hkv * P.blocks) + y) * GB * (D + 2);
    const float pm = part[GB * D + 2 * row], pl = part[GB * D + 2 * row + 1];
    const float nm = fmaxf(m, pm), fo = fast_exp2(m - nm), fp = fast_exp2(pm - nm);
    m = nm;
    l = fmaf(l, fo, pl * fp);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], fo, part[row * D + lane + 32 * e] * fp);
  }
  if (lane == 0) { sh_m[warp] = m; sh_l[warp] = l; }
#pragma unroll
  for (int e = 0; e < E; ++e) sh_o[warp][lane + 32 * e] = o[e];
  __syncthreads();
  const float top = fmaxf(fmaxf(sh_m[0], sh_m[1]), fmaxf(sh_m[2], sh_m[3]));
  for (int f = threadIdx.x; f < D; f += NT) {
    float acc = 0.f, sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float t = fast_exp2(sh_m[w] - top);
      acc = fmaf(sh_o[w][f], t, acc);
      sum = fmaf(sh_l[w], t, sum);
    }
    const float r = has ? acc / sum : (length == 0 ? 0.f : nan_f32());
    unsigned short* out = static_cast<unsigned short*>(a.out) + (int64_t)s * a.out_sequence + (int64_t)h * a.out_head + f;
    if (a.bf16) *reinterpret_cast<__nv_bfloat16*>(out) = __float2bfloat16_rn(r);
    else *reinterpret_cast<__half*>(out) = __float2half_rn(r);
  }
}

int blocks_of(int group) { return (group + GB - 1) / GB; }
int target_of(int Hkv, int blocks) {
  const int t = SMS * RESIDENT / (Hkv * blocks);
  return t > 1 ? t : 1;
}

template <int D>
cudaError_t launch_attend_d(const AttendParams& P, cudaStream_t stream) {
  constexpr size_t smem = 1024 + (size_t)NW * Shape<D>::STAGES * Shape<D>::BYTES;
  static_assert(RESIDENT * (smem + 2048) <= 227 * 1024, "shared memory of the CTAs that are to run at once");
  cudaError_t e = cudaFuncSetAttribute(pages_attend_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  const PageCache& c = P.a.c;
  pages_attend_kernel<D><<<dim3((unsigned)(P.target + c.S), (unsigned)(c.Hkv * P.blocks)), NT, smem, stream>>>(P);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)c.S, (unsigned)P.a.H);
  cfg.blockDim = dim3(NT);
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, pages_merge_kernel<D>, P);
}

}  // namespace

int pages_attend_chunks(int S, int Hkv, int H) { return target_of(Hkv, blocks_of(H / Hkv)) + S; }
size_t pages_attend_partials(int S, int Hkv, int H, int d) {
  return (size_t)pages_attend_chunks(S, Hkv, H) * Hkv * blocks_of(H / Hkv) * GB * (d + 2);
}

cudaError_t launch_pages_attend(const PagesAttend& a, cudaStream_t stream) {
  AttendParams P{};
  P.a = a;
  P.group = a.H / a.c.Hkv;
  P.blocks = blocks_of(P.group);
  P.target = target_of(a.c.Hkv, P.blocks);
  while ((1 << P.log_page) < a.c.page) ++P.log_page;
  P.scale = a.scale * LOG2E;
  const int D = a.c.d, tile = D == 256 ? 16 : 32;
  const uint64_t dims[2] = {(uint64_t)D, (uint64_t)a.c.pages * a.c.Hkv * 2 * a.c.page}, strides[1] = {(uint64_t)D};
  const uint32_t box[2] = {(uint32_t)(D < 128 ? D : 128), (uint32_t)(a.c.page < tile ? a.c.page : tile)};
  if (!make_tensor_map(&P.tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, a.c.codes, dims, strides, box, D == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorNotSupported;
  switch (D) {
    case 64: return launch_attend_d<64>(P, stream);
    case 128: return launch_attend_d<128>(P, stream);
    case 256: return launch_attend_d<256>(P, stream);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kf
