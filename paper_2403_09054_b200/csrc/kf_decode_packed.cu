// One generation step over a 4-bit cache (slot format: kf_packed.cuh); the arithmetic of Algorithm 1 is that of
// kf_decode.cu, only the rows are read from 4 bits.  Two launches: packed_stream_kernel reads every slot once and
// leaves one partial per split, packed_close_kernel (the closing stage of kf_close.cuh with a 4-bit row store) merges,
// scores, evicts and writes the new token's slot.
//
// Per slot 1.25 d bytes come from HBM, a quarter of the binary16 form less the group parameters, so the arithmetic that the
// binary16 kernel hides behind its loads would bound this one: 2 d multiply-adds per slot and head and as many
// conversions.  Both products therefore run on the tensor pipe as m16n8k16 instructions whose 4-bit operand is
// converted in registers (it never passes through shared memory, which is why mma.sync and not tcgen05, whose
// operands have to lie there): S = K q^T with slots as rows, O^T = V^T p^T with features as rows, the query heads of a
// cache (1, 2, 4 or 8) in the eight columns.  A contraction may take its terms in any order, so every lane contracts
// the features (for S) or the slots (for O) that its own 16-byte loads brought, and the other operand is laid out to match.
//
// Every warp walks its CTA's range by itself, 64 slots at a time: two tiles of 32 slots, each in a private shared-memory
// buffer that one bulk copy fills (a tile is contiguous), so that no register holds a row that is still on its way.  A
// lane owns two slots in the per-logit work, whose chains (generator, logarithms, exponentials) then overlap, and the
// bookkeeping of the running softmaxes is paid once for 64 slots.  A buffer is refilled as soon as its values have been used.
//
// What bounds it: latency, with nothing saturated.  1024 caches of 2048 slots (d 128, one head each; 361 MB): 86 us a call, of which 77 are
// the streaming kernel (4.7 TB/s) and 9 the closing one; the bytes alone would take 56, and its 846 warp instructions per 32 slots (480 of
// them conversions) about 49 if every issue slot were used.  By counters (half that size): issue slots 63 %, ALU 46 %, FMA pipes 47 %, DRAM
// 45 %, tensor pipe 20 %; a scheduler has 3.7 warps, and of the 5.9 cycles between two instructions of a warp 1.1 are the fixed latency
// of the one before, 1.0 other warps' turns, 0.7 memory, 0.7 a busy pipe, 0.5 dispatch.  32 caches of 4096: 13 us, one round per warp, a chain
// of dependent latencies.  256 caches of up to 1999 slots, four heads each: 36 us half full, 48 full (issue slots 58 %, DRAM 24 %), each further
// head adding its noise (90 instructions per 32 slots) and softmaxes.  Measured and not taken: tiles staged in registers (106), the
// closing stage inside the streaming CTA with one CTA per cache (101), the heads as a loop (37.4, and 42 instead of 40 at d 256).
#include "kf_close.cuh"
#include "kf_packed.cuh"

#include <algorithm>
#include <atomic>

namespace kf {

namespace {

constexpr int TILE = 32;   // slots per buffer
constexpr int SPAN = 64;   // slots per warp and round: two buffers, two slots per lane in the per-logit work
constexpr int NW = 4;      // warps per CTA

// ---- noise.  ln x for normal x > 0: x = 2^e (1 + f), f in [sqrt(1/2) - 1, sqrt(2) - 1], t = f / (2 + f),
// ln(1 + f) = 2 atanh(t) = 2 t (1 + t^2/3 + t^4/5 + ...) with 2 t = f - t f; the terms up to t^9 leave 1e-9.  Relative
// error below 3e-7 right up to x = 1, where the largest Gumbel variates come from.
__device__ __forceinline__ float ln_atanh(float x) {
  const int bits = __float_as_int(x);
  const int e = (bits - 0x3f3504f3) >> 23;                    // 0x3f3504f3: sqrt(1/2)
  const float f = __int_as_float(bits - (e << 23)) - 1.0f;
  const float t = __fdividef(f, 2.0f + f), z = t * t;
  const float r = 2.0f * z * fmaf(z, fmaf(z, fmaf(z, 1.0f / 9.0f, 1.0f / 7.0f), 0.2f), 1.0f / 3.0f);
  return fmaf((float)e, LN2, f - t * (f - r));
}
__device__ __forceinline__ float packed_gumbel(const PackedParams& P, uint32_t b, uint32_t lh, uint32_t i, uint32_t j) {
  // the outer logarithm may be the fast one.  Over all 2^23 uniforms the variate is off by at most 1.8e-6 (the largest, 16.6; the spacing of
  // binary32 there is 1.9e-6) and by 2.4e-7 where it lies within 1 of zero.
  return -LN2 * __log2f(-ln_atanh(uniform_from_word(noise_word(P.pk, b, lh, i, j))));
}

// ---- the new token's row, quantised by the closing CTA.  Warps hold 32 consecutive features at a time: one group.
template <int D, int NT, int CPT>
struct CloseRow<PackedParams, D, NT, CPT> {
  __half kn[CPT], vn[CPT];
  __half2 kg[CPT], vg[CPT];     // the groups of the thread's columns
  uint32_t code[CPT];           // K code | V code << 4
  static constexpr bool MARKS_FAILURES = true;
  static __device__ __forceinline__ void nothing_to_evict(const PackedParams& P, int u) {
    if (P.slot_opt && threadIdx.x == 0) P.slot_opt[u] = ERR_BOUNDS;
  }

  static __device__ __forceinline__ float noise(const PackedParams& P, uint32_t b, uint32_t lh, uint32_t i, uint32_t j) {
    return P.noise_mode == 0 ? packed_gumbel(P, b, lh, i, j) : noise_for(P, b, lh, i, j);
  }
  static __device__ __forceinline__ __half2 group_of(__half x) {
    __half low = x, high = x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      low = __hmin_nan(low, __shfl_xor_sync(0xffffffffu, low, o));
      high = __hmax_nan(high, __shfl_xor_sync(0xffffffffu, high, o));
    }
    return packed_group(__half2float(low), __half2float(high));
  }
  static __device__ __forceinline__ __half value(uint32_t code, __half2 g) {
    return __hfma(__float2half_rn((float)code), __low2half(g), __high2half(g));
  }
  __device__ __forceinline__ void prepare(const PackedParams& P, int u) {
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      kg[i] = group_of(kn[i]);
      vg[i] = group_of(vn[i]);
      const uint32_t kc = packed_code(__half2float(kn[i]), __high2float(kg[i]), packed_inverse(__low2half(kg[i])));
      const uint32_t vc = packed_code(__half2float(vn[i]), __high2float(vg[i]), packed_inverse(__low2half(vg[i])));
      code[i] = kc | vc << 4;
      const int c = threadIdx.x + i * NT;
      if (P.row_opt && c < D) {
        P.row_opt[(size_t)u * 2 * D + c] = value(kc, kg[i]);
        P.row_opt[(size_t)u * 2 * D + D + c] = value(vc, vg[i]);
      }
    }
  }
  __device__ __forceinline__ void store(const PackedParams& P, int u, int slot) const {
    if (P.slot_opt && threadIdx.x == 0) P.slot_opt[u] = slot;
    if (slot < 0) return;
    unsigned char* at = P.cache + ((size_t)u * P.k + slot) * packed_slot_bytes(D);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int c = threadIdx.x + i * NT;
      const uint32_t next = __shfl_down_sync(0xffffffffu, code[i], 1);   // the odd feature's codes
      if (c < D && (c & 1) == 0) {
        at[c / 2] = (unsigned char)((code[i] & 15u) | (next & 15u) << 4);
        at[D / 2 + c / 2] = (unsigned char)(code[i] >> 4 | (next & 0xf0u));
      }
      if (c < D && (c & 31) == 0) {
        *reinterpret_cast<uint32_t*>(at + D + c / 8) = h2_bits(kg[i]);
        *reinterpret_cast<uint32_t*>(at + D + D / 8 + c / 8) = h2_bits(vg[i]);
      }
    }
  }
};

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float redux_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

template <int N>
__device__ __forceinline__ void shared_words(uint32_t (&w)[N], const unsigned char* p) {
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x; w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p + 4 * i);
      w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
    }
  }
}

// CTAs an SM holds: the register limit that goes with them.  At d 128 and one head: 4 (117 registers) 86 us, 3 90, 5 (96 registers,
// spilling) 102.  d 256 needs 80 KB of buffers a CTA (187 to 245 registers), eight heads 159 to 168 registers.  Four heads at d 128 meet the
// limit of 128 and spill two or three registers.
template <int D, int G>
constexpr int resident_ctas() { return D == 256 ? 2 : (G == 8 ? 3 : 4); }

// GUMBEL: the method's own adjustment, alone in its kernel (up to sixteen places draw noise, and the instructions of all the
// alternatives together would not stay in the instruction cache).
template <int D, int G, bool GUMBEL>
__global__ void __launch_bounds__(NW * 32, resident_ctas<D, G>()) packed_stream_kernel(const __grid_constant__ PackedParams P) {
  constexpr int PSTRIDE = 4 + D;
  constexpr int NT = NW * 32;
  constexpr int SB = packed_slot_bytes(D);
  constexpr int TILE_BYTES = TILE * SB;
  extern __shared__ __align__(128) unsigned char dyn_smem[];
  // An output weight goes into the second product as two binary16 numbers, itself rounded and what the rounding left out,
  // so that only the output is rounded.  With up to four heads the two are columns of one instruction (col and col + G),
  // with eight they follow one another into the same accumulators.
  constexpr int COLS = G <= 4 ? 2 * G : G;
  __shared__ float sh_m[NW][G], sh_l[NW][COLS], sh_my[NW][G], sh_ly[NW][G], sh_f[NW][G];
  __shared__ float sh_x[NW][G][SPAN];                       // logits of the warp's slots
  __shared__ __align__(8) __half sh_p[NW][2 * G][SPAN];     // output weights of the heads, then the remainders
  __shared__ uint64_t bars_all[NW][2];
  __shared__ float sh_slope[G];
  __shared__ uint4 sh_q[D / 32][32];                        // queries, as every lane of a warp wants them

  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int s = blockIdx.x, u = blockIdx.z * gridDim.y + blockIdx.y;   // grid: splits, key/value heads, batch rows
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r8 = lane >> 2, t4 = lane & 3;
  const int len = P.len[u];
  if (len < 0 || len > P.k) return;   // a damaged entry count: nothing of this unit is touched
  const int row_begin = s * P.tiles_per_split * TILE;
  const int row_end = min(len, row_begin + P.tiles_per_split * TILE);
  const unsigned char* cache_u = P.cache + (size_t)u * P.k * SB;
  const int32_t* pos_u = P.pos + (size_t)u * P.k;
  const uint32_t b = blockIdx.z, h0 = blockIdx.y * G, lh0 = (uint32_t)P.layer * P.H + h0;

  // ---- the warp's two buffers
  const int first = row_begin + warp * SPAN;                 // first slot of the warp's first round
  const int rounds = row_end > first ? (row_end - first + NW * SPAN - 1) / (NW * SPAN) : 0;
  unsigned char* ring = dyn_smem + (size_t)warp * 2 * TILE_BYTES;
  uint64_t* bars = bars_all[warp];
  auto issue = [&](int it, int sub) {                        // fetches tile `sub` of round `it`, if it has a slot
    const int tb = first + it * NW * SPAN + sub * TILE;
    if (lane == 0 && tb < row_end) {
      const uint32_t bytes = (uint32_t)min(TILE, row_end - tb) * SB;
      mbar_expect_tx(bars + sub, bytes);
      bulk_load(ring + sub * TILE_BYTES, cache_u + (size_t)tb * SB, bytes, bars + sub);
    }
  };
  if (lane == 0) {
    mbar_init(bars, 1);
    mbar_init(bars + 1, 1);
    mbar_fence_init();
  }
  // queries as the second operand of S: column = head r8, the features this lane's K words bring, pairs (i, i + 4)
  for (int w = warp; w < D / 32; w += NW) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r8 < G) v = *reinterpret_cast<const uint4*>(P.q + ((size_t)u * G + r8) * D + t4 * (D / 4) + 8 * w);
    sh_q[w][lane] = make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
  }
  if (tid < G) sh_slope[tid] = P.slopes ? P.slopes[h0 + tid] : 0.f;
  __syncthreads();
  issue(0, 0);
  issue(0, 1);
  int pos_next[2];
#pragma unroll
  for (int sub = 0; sub < 2; ++sub) pos_next[sub] = first + sub * TILE + lane < row_end ? pos_u[first + sub * TILE + lane] : 0;

  float m_x[G], m_y[G], l_y[G];            // m_*: common to the warp; l_y: this lane's slots
#pragma unroll
  for (int g = 0; g < G; ++g) { m_x[g] = -INFINITY; m_y[g] = -INFINITY; l_y[g] = 0.f; }
  float l_x[4] = {0.f, 0.f, 0.f, 0.f};     // sums of the output weights, as the product of a row of ones: the columns of o
  float o[D / 16][4];                      // out^T: features as rows, columns 2 t4 and 2 t4 + 1
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) o[i][c] = 0.f;

  // Where the lane finds its share of a tile.  K: rows k_row + 8 i, features [t4 D/4, + D/4).  V: slots 16 h + t4 + 4 i,
  // features [r8 D/8, + D/8).  Both orders keep the lanes of a shared-memory phase on distinct banks (the slots of two
  // neighbouring lane groups lie 2 apart for K, 1 apart for V; a slot is 8 banks, mod 32, at d = 128).
  const int k_row = (r8 & 4) | (r8 & 1) << 1 | (r8 >> 1 & 1);
  const int k_codes = k_row * SB + t4 * (D / 8);
  const int k_group = k_row * SB + D + (D == 64 ? (t4 >> 1) * 4 : t4 * (D / 32));
  const int v_codes = t4 * SB + D / 2 + r8 * (D / 16);
  const int v_group = t4 * SB + D + D / 8 + (r8 * (D / 8) / PACK_GROUP) * 4;
  const int p_at = (lane & 16) + (lane & 3) * 4 + (lane >> 2 & 3);   // where the weight of slot `lane` is read as an operand
  float* y_out = P.y_scratch + (size_t)u * G * (P.k + 1) + first + lane;

  // With several heads their noise and softmaxes fill the instruction cache: the two tiles share their instructions (37.6 -> 35.9 us
  // for 256 caches with four heads; with one head unrolled tiles overlap better, 85 against 88 us for 1024 caches).
  constexpr int TILES_UNROLLED = G == 1 ? 2 : 1;
  bool failed = P.first_wait_limit == 0 && rounds > 0;       // the self-test: as if the first wait had run out
  const int last = failed ? 0 : rounds;
  int it = 0;
  for (; it < last; ++it, y_out += NW * SPAN) {
    const int rows = row_end - (first + it * NW * SPAN);             // may exceed SPAN
    int pj[2];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      pj[sub] = pos_next[sub];
      pos_next[sub] = rows - NW * SPAN > sub * TILE + lane ? pos_u[first + (it + 1) * NW * SPAN + sub * TILE + lane] : 0;
    }
    // the noise needs positions only: its long dependent chains fill the gaps of the conversions below
    float zeta[2][G];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int g = 0; g < G; ++g) zeta[sub][g] = GUMBEL ? packed_gumbel(P, b, lh0 + g, (uint32_t)P.p, (uint32_t)pj[sub])
                              : noise_for(P, b, lh0 + g, (uint32_t)P.p, (uint32_t)pj[sub]);

    // ---- logits (slots behind the last entry give numbers that nobody reads)
#pragma unroll(TILES_UNROLLED)
    for (int sub = 0; sub < 2; ++sub) {
      if (sub * TILE >= rows) break;
      const bool ok = mbar_wait_bounded(bars + sub, (uint32_t)(it & 1));
      if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
      const unsigned char* buf = ring + sub * TILE_BYTES;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float c[4] = {0.f, 0.f, 0.f, 0.f}, c2[4] = {0.f, 0.f, 0.f, 0.f};   // two chains: half the latency, and half the roundings
        constexpr int NG = D == 256 ? 2 : 1;      // groups a lane's features span
        uint32_t kw[2][D / 32], kg[2][NG];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          shared_words(kw[i], buf + k_codes + (16 * h + 8 * i) * SB);
          shared_words(kg[i], buf + k_group + (16 * h + 8 * i) * SB);
        }
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
          __half2 a[2][4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const __half2 g = bits_h2(kg[i][NG == 2 ? w / 4 : 0]);
            nibble_pairs(kw[i][w], a[i]);
#pragma unroll
            for (int e = 0; e < 4; ++e) a[i][e] = __hfma2(a[i][e], __low2half2(g), __high2half2(g));
          }
          const uint4 qf = sh_q[w][lane];
          mma_16816(c, h2_bits(a[0][0]), h2_bits(a[1][0]), h2_bits(a[0][1]), h2_bits(a[1][1]), qf.x, qf.y);
          mma_16816(c2, h2_bits(a[0][2]), h2_bits(a[1][2]), h2_bits(a[0][3]), h2_bits(a[1][3]), qf.z, qf.w);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] += c2[i];
        const int at = sub * TILE + 16 * h + k_row;
        if (2 * t4 < G) { sh_x[warp][2 * t4][at] = c[0]; sh_x[warp][2 * t4][at + 8] = c[2]; }
        if (2 * t4 + 1 < G) { sh_x[warp][2 * t4 + 1][at] = c[1]; sh_x[warp][2 * t4 + 1][at + 8] = c[3]; }
      }
    }
    if (failed) break;
    __syncwarp();

    // ---- per logit (a lane owns slots `lane` and `lane` + 32): bias, noise, the two running softmaxes.  The output weights are taken
    //      against a reference that moves only when a round exceeds it by 2^8, so that the accumulators are hardly ever
    //      rescaled, and times 2^7: binary16 holds them up to 2^15, and down to 2^-32 of the reference (a warp may walk 2^18 slots, whose
    //      small weights count together).  The sums are binary32.
    float scale_o[G];
    bool moved = false;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      // every lane computes, so that the warp stays together; what has no entry becomes -inf at the end
      float x[2], y[2];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const bool valid = sub * TILE + lane < rows;
        x[sub] = fmaf(-sh_slope[g], (float)(P.p - pj[sub]), sh_x[warp][g][sub * TILE + lane] * P.scale);
        y[sub] = (x[sub] + zeta[sub][g]) * P.inv_tau;
        if (valid) y_out[(size_t)g * (P.k + 1) + sub * TILE] = y[sub];
        x[sub] = valid ? x[sub] : -INFINITY;
        y[sub] = valid ? y[sub] : -INFINITY;
      }
      const float tx = redux_max(fmaxf(x[0], x[1])), my_new = fmaxf(m_y[g], redux_max(fmaxf(y[0], y[1])));
      scale_o[g] = 1.f;
      if (!(tx <= m_x[g] + 5.5f)) {   // 2^8 = e^5.55; also the first round (and a NaN, which stays one)
        scale_o[g] = fast_exp2((m_x[g] - tx) * LOG2E);
        m_x[g] = tx;
        moved = true;
      }
      float ey = 0.f;
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const bool valid = sub * TILE + lane < rows;
        ey += valid ? fast_exp2((y[sub] - my_new) * LOG2E) : 0.f;
        const float px = valid ? fast_exp2(fmaf(x[sub] - m_x[g], LOG2E, 7.f)) : 0.f;
        const __half hi = __float2half_rn(px);
        sh_p[warp][g][sub * TILE + p_at] = hi;
        sh_p[warp][G + g][sub * TILE + p_at] = __float2half_rn(px - __half2float(hi));
      }
      l_y[g] = fmaf(l_y[g], fast_exp2((m_y[g] - my_new) * LOG2E), ey);
      m_y[g] = my_new;
    }
    if (moved) {
      float f0 = 1.f, f1 = 1.f;   // of this lane's two columns
#pragma unroll
      for (int g = 0; g < G; ++g) {
        if (2 * t4 < COLS && g == 2 * t4 % G) f0 = scale_o[g];
        if (2 * t4 + 1 < COLS && g == (2 * t4 + 1) % G) f1 = scale_o[g];
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) { o[i][0] *= f0; o[i][1] *= f1; o[i][2] *= f0; o[i][3] *= f1; }
      l_x[0] *= f0;
      l_x[1] *= f1;
    }
    __syncwarp();

    // ---- values; a slot behind the last entry counts as zeros, whatever the buffer holds
#pragma unroll(TILES_UNROLLED)
    for (int sub = 0; sub < 2; ++sub) {
      if (sub * TILE >= rows) break;
      const unsigned char* buf = ring + sub * TILE_BYTES;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        constexpr int W = D / 64;
        uint2 pb = make_uint2(0, 0), rest = pb;   // weights of slots 16 h + t4 + 4 {0 .. 3} for column r8
        if (r8 < COLS) pb = *reinterpret_cast<const uint2*>(&sh_p[warp][r8][sub * TILE + 16 * h + 4 * t4]);
        if (G == 8) rest = *reinterpret_cast<const uint2*>(&sh_p[warp][G + r8 % G][sub * TILE + 16 * h + 4 * t4]);
        mma_16816(l_x, 0x3c003c00u, 0u, 0x3c003c00u, 0u, pb.x, pb.y);
        if (G == 8) mma_16816(l_x, 0x3c003c00u, 0u, 0x3c003c00u, 0u, rest.x, rest.y);
        uint32_t vw[4][W], vg[4][1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          shared_words(vw[i], buf + v_codes + (16 * h + 4 * i) * SB);
          shared_words(vg[i], buf + v_group + (16 * h + 4 * i) * SB);
        }
        if (rows < SPAN) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (sub * TILE + 16 * h + 4 * i + t4 >= rows) vg[i][0] = 0u;      // scale and minimum 0
        }
#pragma unroll
        for (int w = 0; w < W; ++w) {
          __half2 lo[2][4], hi[2][4];   // features 8 w + (0 .. 3) and + (4 .. 7); a pair is two of the lane's slots
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const __half2 sc = bits_h2(__byte_perm(vg[2 * e][0], vg[2 * e + 1][0], 0x5410)), mn = bits_h2(__byte_perm(vg[2 * e][0], vg[2 * e + 1][0], 0x7632));
            nibble_pairs(__byte_perm(vw[2 * e][w], vw[2 * e + 1][w], 0x5410), lo[e]);
            nibble_pairs(__byte_perm(vw[2 * e][w], vw[2 * e + 1][w], 0x7632), hi[e]);
#pragma unroll
            for (int j = 0; j < 4; ++j) { lo[e][j] = __hfma2(lo[e][j], sc, mn); hi[e][j] = __hfma2(hi[e][j], sc, mn); }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            mma_16816(o[4 * w + j], h2_bits(lo[0][j]), h2_bits(hi[0][j]), h2_bits(lo[1][j]), h2_bits(hi[1][j]), pb.x, pb.y);
            if (G == 8) mma_16816(o[4 * w + j], h2_bits(lo[0][j]), h2_bits(hi[0][j]), h2_bits(lo[1][j]), h2_bits(hi[1][j]), rest.x, rest.y);
          }
        }
      }
      __syncwarp();   // the buffer has been read by every lane
      if (it + 1 < last) issue(it + 1, sub);
    }
  }
  if (failed) {
    // a copy did not land in time: the unit is marked below; the copies still in flight get a second bounded wait
    for (int sub = 0; sub < 2; ++sub)
      if (first + it * NW * SPAN + sub * TILE < row_end) (void)mbar_wait_bounded(bars + sub, (uint32_t)(it & 1));
  }

  // ---- merge the lanes, then the warps of this CTA; the sums lie in the buffers, which are done with
  static_assert(COLS * D * 4 <= 2 * TILE_BYTES, "a warp's sums fit its buffers");
  float* sums = reinterpret_cast<float*>(ring);              // [COLS][D]
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const int f = r8 * (D / 8) + (i >> 2) * 8 + (i & 3);
    if (2 * t4 < COLS) { sums[2 * t4 * D + f] = o[i][0]; sums[2 * t4 * D + f + 4] = o[i][2]; }
    if (2 * t4 + 1 < COLS) { sums[(2 * t4 + 1) * D + f] = o[i][1]; sums[(2 * t4 + 1) * D + f + 4] = o[i][3]; }
  }
  if (r8 == 0) {
    if (2 * t4 < COLS) sh_l[warp][2 * t4] = l_x[0];
    if (2 * t4 + 1 < COLS) sh_l[warp][2 * t4 + 1] = l_x[1];
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
    l_y[g] = warp_sum(l_y[g]);
    if (lane == 0) { sh_m[warp][g] = m_x[g]; sh_my[warp][g] = m_y[g]; sh_ly[warp][g] = l_y[g]; }
  }
  const bool lost = __syncthreads_or(failed);
  float* part = P.partials + ((size_t)u * P.splits + s) * G * PSTRIDE;      // [head][4 + D]
  if (tid < G) {                                                            // one thread per head joins the statistics
    const int g = tid;
    float M = -INFINITY, MY = -INFINITY, L = 0.f, LY = 0.f;
#pragma unroll
    for (int wi = 0; wi < NW; ++wi) { M = fmaxf(M, sh_m[wi][g]); MY = fmaxf(MY, sh_my[wi][g]); }
#pragma unroll
    for (int wi = 0; wi < NW; ++wi) {
      const float l = sh_l[wi][g] + (COLS > G ? sh_l[wi][COLS - G + g] : 0.f);
      const float f = l > 0.f ? fast_exp2((sh_m[wi][g] - M) * LOG2E) * 0x1p-7f : 0.f;   // and the weights' 2^7 off again
      L = fmaf(l, f, L);
      if (sh_ly[wi][g] > 0.f) LY = fmaf(sh_ly[wi][g], fast_exp2((sh_my[wi][g] - MY) * LOG2E), LY);
      sh_f[wi][g] = f;
    }
    // sums of -1, which no softmax has, tell the closing kernel that rows are missing
    *reinterpret_cast<float4*>(part + g * PSTRIDE) = lost ? make_float4(-INFINITY, -1.f, -INFINITY, -1.f) : make_float4(M, L, MY, LY);
  }
  __syncthreads();
  for (int idx = tid; idx < G * D; idx += NT) {
    const int g = idx / D, c = idx % D;
    float sum = 0.f;
#pragma unroll
    for (int wi = 0; wi < NW; ++wi) {
      const float* of = reinterpret_cast<const float*>(dyn_smem + (size_t)wi * 2 * TILE_BYTES);
      sum = fmaf(of[idx] + (COLS > G ? of[(COLS - G) * D + idx] : 0.f), sh_f[wi][g], sum);
    }
    part[g * PSTRIDE + 4 + c] = sum;
  }
}

template <int D>
__global__ void __launch_bounds__(512, 1) packed_close_wide_kernel(const __grid_constant__ PackedParams P) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int u = blockIdx.x;
  const int len = P.len[u];
  if (len < 0 || len > P.k) return;
  combine_and_evict_group<D, 512, 1, 8, true>(P, u, len);   // 4096 entries in one round
}

template <int D, int G>
__global__ void __launch_bounds__(close_threads(D, G), G == 1 ? 6 : (G == 8 ? 1 : 2)) packed_close_kernel(const __grid_constant__ PackedParams P) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int u = blockIdx.x;
  const int len = P.len[u];
  if (len < 0 || len > P.k) return;
  if constexpr (G == 1) combine_and_evict<D, 128, 1>(P, u, len);
  else combine_and_evict_group<D, close_threads(D, G), G, 4, true>(P, u, len);
}

template <int D, int G>
cudaError_t launch_one(const PackedParams& P, int units, cudaStream_t stream) {
  // Programmatic stream serialization on both launches, as for the binary16 kernels.
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)P.splits, (unsigned)(P.H / G), (unsigned)(units / (P.H / G)));
  cfg.blockDim = dim3(NW * 32);
  cfg.dynamicSmemBytes = NW * 2 * TILE * packed_slot_bytes(D);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  auto kern = P.noise_mode == 0 ? packed_stream_kernel<D, G, true> : packed_stream_kernel<D, G, false>;
  cudaError_t e = cudaSuccess;
  if (cfg.dynamicSmemBytes > 32 * 1024) {   // with the static part (up to 22 KB) above what every kernel may have; asked for once per device
    static std::atomic<uint64_t> asked{0};
    int dev = 0;
    e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev >= 64 || !(asked.load(std::memory_order_relaxed) >> dev & 1))) {
      e = cudaFuncSetAttribute(packed_stream_kernel<D, G, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes);
      if (e == cudaSuccess)
        e = cudaFuncSetAttribute(packed_stream_kernel<D, G, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes);
      if (e == cudaSuccess && dev < 64) asked.fetch_or((uint64_t)1 << dev, std::memory_order_relaxed);
    }
  }
  if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, kern, P);
  if (e != cudaSuccess) return e;
  cfg.dynamicSmemBytes = 0;
  cfg.gridDim = dim3((unsigned)units);
  cfg.blockDim = dim3(close_threads(D, G));
  if constexpr (G == 1) {
    if (close_is_wide(units, P.k)) {
      cfg.blockDim = dim3(512);
      return cudaLaunchKernelEx(&cfg, packed_close_wide_kernel<D>, P);
    }
  }
  return cudaLaunchKernelEx(&cfg, packed_close_kernel<D, G>, P);
}

template <int D>
cudaError_t launch_dim(const PackedParams& P, int units, cudaStream_t stream) {
  switch (P.group) {
    case 1: return launch_one<D, 1>(P, units, stream);
    case 2: return launch_one<D, 2>(P, units, stream);
    case 4: return launch_one<D, 4>(P, units, stream);
    case 8: return launch_one<D, 8>(P, units, stream);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace

void decode_packed_plan(int units, int budget_k, int head_dim, int* splits_out, int* tiles_per_split_out) {
  const int tiles = (budget_k + TILE - 1) / TILE;
  constexpr int ROUND = NW * SPAN / TILE;   // tiles of a round of the CTA's warps
  // Many caches: about three waves of CTAs (two CTAs for each of 1024 caches; one each 86.7 us, two 86.6, three 90.3).  Few: as many
  // CTAs as give every warp at least one round (32 caches of 4096: 16 CTAs each 13.7 us, 10 15.0, 8 17.3).
  // The rule does not look at the heads per cache nor at d.  256 full caches of 1999 slots in 1, 2, 4 and 8 (the rule's) CTAs: four heads, d 64 60, 37, 38,
  // 39 us, d 128 76, 47, 47, 48; eight heads, d 128 97, 87, 79, 77: it is within 5 % of the best (one head, d 64 28, 25, 24, 27: 11 %).  At d 256, where
  // an SM holds two CTAs, fewer would do better: one head 50, 53, 57, 64, four 69, 73, 82, 92, eight 105, 111, 122, 130.  32 caches of
  // 4096, 16 CTAs each (the rule's) against 8: d 128 13.0 and 16.4, four heads 18.7 and 24.9; d 256 22.7 and 20.1.
  const int target_ctas = units >= 148 ? 148 * 13 : 148 * 8;
  int splits = (target_ctas + units - 1) / units;
  splits = std::max(1, std::min(splits, std::min(MAX_SPLITS, (tiles + ROUND - 1) / ROUND)));
  int tps = (tiles + splits - 1) / splits;
  tps = (tps + ROUND - 1) / ROUND * ROUND;
  *splits_out = (tiles + tps - 1) / tps;
  *tiles_per_split_out = tps;
}

cudaError_t launch_decode_packed(const PackedParams& P, int head_dim, int units, cudaStream_t stream) {
  if (P.splits < 1 || P.splits > MAX_SPLITS) return cudaErrorInvalidValue;
  switch (head_dim) {
    case 64: return launch_dim<64>(P, units, stream);
    case 128: return launch_dim<128>(P, units, stream);
    case 256: return launch_dim<256>(P, units, stream);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kf
