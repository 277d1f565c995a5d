// Causal attention over prompts of different lengths that lie one after the other without padding (kf_prefill_attend_ragged):
// out_i = sum_{j <= i} softmax_j(x_ij) v_j within each sequence, in one pass over its keys.
//
// The structure is that of kf_prefill_attend1p.cu (tcgen05 MMAs with accumulators in tensor memory, TMA loads through a ring, a thread
// per query row, references that move only when a row outgrows them by 2^8); what differs:
//   - Operands are binary16 or bfloat16 and lie in any order of heads and tokens (tensor maps with the caller's strides).
//   - Blocks of 128 query rows start at the sequence's own first token.  The grid is laid out without knowing the lengths (slot_sequence);
//     a CTA whose slot holds nothing leaves at once.
//   - A block of 128 rows holds `pack` query heads of a key/value head x 128 / pack tokens, so that a short sequence still fills
//     its rows: row r is token r / pack, head r % pack, which is what a TMA box of 64 features x pack heads x tokens writes.
//   - What stands behind the last key of a sequence belongs to others.  Its logits are masked like any later key's; its value rows
//     are overwritten with zeros in shared memory, because 0 * NaN is NaN.
//   - head_dim 256: one block of 128 rows per CTA and key tiles of 64 rows (tensor memory: 2 x 64 columns of S and 256 of O; the logits
//     of the next tile are formed while the current one's softmax runs).
// Output weights are taken times 2^7, so that binary16 holds them from 2^-32 of a row's largest on; bfloat16 (the type V has, which the
// MMA wants for both) rounds them to 8 bits, as much as the output itself is rounded.
#include "kf_pages.cuh"
#include "kf_tc.cuh"

namespace kf {

namespace {

// A group of four warps for the TMA loads and the MMAs (one warp each), one per block of query rows.  With two blocks the registers of the launch
// (384 x 168) are dealt out again: a compute thread holds its whole row of logits.
constexpr int threads_of(int blocks) { return 128 * (blocks + 1); }
constexpr int FEW_REGS = 72, MANY_REGS = 216;
static_assert(128 * FEW_REGS + 256 * MANY_REGS <= 384 * 168, "registers of the launch");
constexpr int RING = 5;                 // slots that K and V tiles go through in the order of use
constexpr uint32_t TMEM_COLS = 512;
constexpr float HEADROOM = 7.0f;        // log2 units a weight stands above its distance from the reference
constexpr float LOWEST = -1e30f;
constexpr float SLACK = 8.0f;           // log2 units a row's maximum may exceed its reference before the reference moves

struct RaggedParams {
  CUtensorMap tmQ, tmK, tmV;   // [heads][tokens] rows of d; boxes of 64 features x (pack heads x 128 / pack tokens; KT tokens), 128-byte swizzle
  void* out;
  const int32_t* begin;
  const float* slopes;
  int64_t out_token, out_head;
  int32_t tokens, S, pack, log_pack, group;
  float a_scale;               // logit scale * log2(e)
  bool fail_first_wait;
};

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if (BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <int D, bool ALIBI, bool BF16>
__global__ void __launch_bounds__(threads_of(D == 256 ? 1 : 2), 1) ragged_kernel(const __grid_constant__ RaggedParams P) {
  constexpr int NB = D == 256 ? 1 : 2;     // blocks of 128 query rows
  constexpr int KT = D == 256 ? 64 : 128;  // rows of a key tile
  constexpr int KCH = D / 64;              // 64-feature boxes per row
  constexpr int QBOX = 128 * 128, Q_BYTES = KCH * QBOX;
  constexpr int KBOX = KT * 128, SLOT = KCH * KBOX;
  constexpr int AHEAD = NB == 1 ? 2 : 1;   // logit tiles of a block in tensor memory (the two blocks take turns, one block alone looks ahead)
  constexpr uint32_t O_COL = 256;          // S tiles from 0 (block or parity x KT), O of block b at 256 + b D
  constexpr uint32_t TYPES = BF16 ? (1u << 7) | (1u << 10) : 0u;
  constexpr uint32_t IDESC_QK = umma_idesc_kk(KT) | TYPES;
  constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24) | TYPES;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* sQ = smem;
  unsigned char* sR = sQ + NB * Q_BYTES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(sR + (size_t)RING * SLOT);
  uint64_t* q_full = bars;
  uint64_t* r_full = q_full + 1;
  uint64_t* r_empty = r_full + RING;
  uint64_t* s_full = r_empty + RING;      // [2] per block, or per parity of the tile
  uint64_t* p_full = s_full + 2;          // [2][2]: the halves of a tile's weights
  uint64_t* o_full = p_full + 4;          // [2]
  uint64_t* v_done = o_full + 2;          // one block: the value MMAs of a tile have completed
  uint64_t* v_clean = v_done + 1;         // value rows behind the sequence have been overwritten
  uint64_t* drain = v_clean + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* issued = const_cast<int*>(abort_flag) + 1;   // ring positions whose loads have been issued

  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int tb = 128 >> P.log_pack;                // tokens of a block
  constexpr int ROW_SHIFT = NB == 2 ? 8 : 7;       // rows of a CTA
  const int slot = (int)(gridDim.x - 1 - blockIdx.x);   // the longest CTAs of a sequence start first
  const int seq = slot_sequence(P.begin, P.S, slot, P.pack, ROW_SHIFT, 1);
  const int row0 = P.begin[seq], row_end = P.begin[seq + 1];
  const int64_t local = slot - slot_start(P.begin, seq, P.pack, ROW_SHIFT, 1);
  if (row0 < 0 || row_end > P.tokens || row0 >= row_end || local < 0) return;
  const int n = row_end - row0;
  const int64_t first64 = local * (NB * tb);       // first token of the CTA within the sequence
  if (first64 >= n) return;
  const int first = (int)first64;
  const bool has1 = NB == 2 && first + tb < n;
  const int T0 = (min(first + tb, n) + KT - 1) / KT;                              // key tiles of block 0
  const int T = has1 ? (min(first + 2 * tb, n) + KT - 1) / KT : T0;               // key tiles the CTA walks: step u takes tile T - 1 - u
  const int U0 = T - T0;                                                          // the step at which block 0 joins
  const bool clean = T * KT > n && row0 + n < P.tokens;                           // rows of others in the last tile, the first to be walked
  const int head0 = blockIdx.y * P.pack, kv_head = head0 / P.group;

  if (tid == 0) {
    mbar_init(q_full, 1);
    for (int s = 0; s < RING; ++s) { mbar_init(r_full + s, 1); mbar_init(r_empty + s, 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(s_full + b, 1); mbar_init(p_full + 2 * b, 4); mbar_init(p_full + 2 * b + 1, 4); mbar_init(o_full + b, 1); }
    mbar_init(v_done, 1);
    mbar_init(v_clean, 1);
    mbar_init(drain, 1);
    *abort_flag = 0;
    issued[0] = 0;
    mbar_fence_init();
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  // Ring position 0 is the K tile of step 0; then, as the MMA warp needs them, the K tile of step u + AHEAD before the V tile of step u.  With one step of
  // look-ahead position 2u + 1 is K of step u + 1 and 2u + 2 V of step u; with two, positions 0 and 1 are K, 2u + 2 is V of step u and 2u + 3 K of step u + 2.
  if (warp < 4) {
    if (NB == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(FEW_REGS));
   if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    bool ok = true;
    if (lane == 0) {
      mbar_expect_tx(q_full, has1 ? 2 * Q_BYTES : Q_BYTES);
      for (int b = 0; b < (has1 ? 2 : 1); ++b)
        for (int kc = 0; kc < KCH; ++kc) tma_load_3d(sQ + b * Q_BYTES + kc * QBOX, &P.tmQ, kc * 64, head0, row0 + first + b * tb, q_full);
      for (int j = 0; ok && j <= 2 * T; ++j) {
        const bool is_v = j >= 2 && (j & 1) == 0;
        const int u = is_v ? (j - 2) >> 1 : (AHEAD == 1 ? (j == 0 ? 0 : (j + 1) >> 1) : (j < 2 ? j : (j + 1) >> 1));
        if (u >= T) continue;                                  // a K tile behind the last one
        const int s = j % RING;
        if (j >= RING) ok = wait_bar(r_empty + s, (uint32_t)((j / RING - 1) & 1), abort_flag);
        if (!ok) break;
        mbar_expect_tx(r_full + s, SLOT);
        const CUtensorMap* tm = is_v ? &P.tmV : &P.tmK;
        for (int kc = 0; kc < KCH; ++kc) tma_load_3d(sR + (size_t)s * SLOT + kc * KBOX, tm, kc * 64, row0 + (T - 1 - u) * KT, kv_head, r_full + s);
        issued[0] = j + 1;
      }
      if (!ok) *abort_flag = 1;
    }
   } else if (warp == 2) {
    // ------------------------------------------------------------ value rows of others, in the tile of step 0, become zeros
    if (clean) {
      constexpr int s = 2;                                     // its ring position
      if (__all_sync(0xffffffffu, wait_bar_eager(r_full + s, 0, abort_flag))) {
        unsigned char* tile = sR + (size_t)s * SLOT;
        const int from = n - (T - 1) * KT;                     // rows of the tile that are the sequence's
        for (int kc = 0; kc < KCH; ++kc)
          for (int i = from * 8 + lane; i < KT * 8; i += 32) reinterpret_cast<uint4*>(tile + kc * KBOX)[i] = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(v_clean);
      } else if (lane == 0) {
        *abort_flag = 1;
      }
    }
   } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer: the warp runs along together, one lane issues
    const uint32_t leader = warp_leader();
    const int Tu = __shfl_sync(0xffffffffu, T, 0), U0u = __shfl_sync(0xffffffffu, U0, 0);
    const bool two = __shfl_sync(0xffffffffu, has1 ? 1 : 0, 0) != 0, clean_u = __shfl_sync(0xffffffffu, clean ? 1 : 0, 0) != 0;
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
    auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bar_eager(bar, parity, abort_flag)) != 0; };
    // Where a tile lies: its slot of the ring and the parity of the slot's use.  Two positions on is the next tile of its kind.
    struct Cursor {
      int slot, parity;
      __device__ __forceinline__ void next() {
        slot += 2;
        if (slot >= RING) { slot -= RING; parity ^= 1; }
      }
    };
    bool ok = wait(q_full, 0);
    const uint64_t qd0 = umma_smem_desc(smem_u32(sQ)), kd0 = umma_smem_desc(smem_u32(sR));
    const uint64_t vd0 = umma_desc_mn(smem_u32(sR), KBOX, 1024);   // descriptors of other slots / offsets: + bytes / 16
    // S = Q_b K_t^T (K-major operands, 16 features per MMA) into tile buffer sb
    auto qk = [&](int b, int sb, int slot) {
      const uint64_t kd = kd0 + (uint64_t)((slot * SLOT) >> 4), qd = qd0 + (uint64_t)((b * Q_BYTES) >> 4);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        const uint32_t in_box = (uint32_t)((kk & 3) * 32);
        umma_f16_warp(leader, tmem + (uint32_t)(sb * KT), qd + ((uint32_t)((kk >> 2) * QBOX) + in_box) / 16, kd + ((uint32_t)((kk >> 2) * KBOX) + in_box) / 16,
                      IDESC_QK, kk > 0 ? 1u : 0u);
      }
      umma_commit_warp(leader, s_full + sb);
    };
    // O_b += P V_t (A = P from tensor memory, 16 keys = 8 columns per MMA; B = V, MN-major).  The weights arrive in two halves: the first
    // half's products run while the second is still being formed.
    auto pv = [&](int b, int sb, int slot, uint32_t parity, bool first) {
      const uint64_t vd = vd0 + (uint64_t)((slot * SLOT) >> 4);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (!wait(p_full + 2 * sb + half, parity)) return false;
        tc_fence_after();
#pragma unroll
        for (int kk = half * (KT / 32); kk < (half + 1) * (KT / 32); ++kk)
          umma_f16_ts_warp(leader, tmem + O_COL + (uint32_t)(b * D), tmem + (uint32_t)(sb * KT + kk * 8), vd + (uint64_t)((kk * 16 * 128) >> 4), IDESC_PV,
                           (!first || kk > 0) ? 1u : 0u);
      }
      return true;
    };
    // The tensor pipe must never run dry between two groups of MMAs, so the waits for tiles stand behind the group before the one that
    // needs them.  A slot is handed back by a commit placed right after the last MMA that reads it.
    Cursor kc{0, 0}, vc{2, 0};
    for (int u = 0; ok && u < min(AHEAD, Tu); ++u) {
      ok = wait(r_full + kc.slot, kc.parity);
      if (!ok) break;
      tc_fence_after();
      if (u >= U0u) qk(0, NB == 2 ? 0 : u, kc.slot);
      if (two) qk(1, 1, kc.slot);
      umma_commit_warp(leader, r_empty + kc.slot);
      kc = Cursor{2 * u + 1, 0};                                   // K of step u + 1 stands at 2u + 1
    }
    if (ok && AHEAD < Tu) ok = wait(r_full + kc.slot, kc.parity);
    if (ok) ok = wait(r_full + vc.slot, vc.parity);
    if (ok && clean_u) ok = wait(v_clean, 0);
    for (int u = 0; ok && u < Tu; ++u) {
      const bool more = u + AHEAD < Tu;
      const int kslot = kc.slot, vslot = vc.slot;
      kc.next();
      vc.next();
      const int own = u - U0u;                                     // block 0's step
      if (own >= 0) {
        if (!pv(0, NB == 2 ? 0 : (own & 1), vslot, (uint32_t)(NB == 2 ? own & 1 : own >> 1 & 1), own == 0)) { ok = false; break; }
        if (!two) umma_commit_warp(leader, r_empty + vslot);
        if (NB == 1) umma_commit_warp(leader, v_done);
        if (u == Tu - 1) umma_commit_warp(leader, o_full);
      }
      if (more && own + AHEAD >= 0) qk(0, NB == 2 ? 0 : (own & 1), kslot);
      if (u + AHEAD + 1 < Tu) {
        ok = wait(r_full + kc.slot, kc.parity);
        if (!ok) break;
      }
      if (two) {
        if (!pv(1, 1, vslot, (uint32_t)(u & 1), u == 0)) { ok = false; break; }
        if (more) qk(1, 1, kslot);
        else umma_commit_warp(leader, o_full + 1);
        umma_commit_warp(leader, r_empty + vslot);               // both blocks' value MMAs of the step have been issued
      }
      if (more) umma_commit_warp(leader, r_empty + kslot);       // every logit MMA that reads it has been issued
      if (u + 1 < Tu) ok = wait(r_full + vc.slot, vc.parity);
    }
    if (!ok && lane == 0) *abort_flag = 1;
    umma_commit_warp(leader, drain);
    (void)wait_bar(drain, 0, abort_flag);
   }
  } else {
    if (NB == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(MANY_REGS));
    // ------------------------------------------------------------ compute warps: a thread is a query row
    const int b = NB == 2 ? (warp - 4) >> 2 : 0;
    const int quarter = warp & 3;
    const int row = quarter * 32 + lane;
    const int block0 = first + b * tb;               // the block's first token within the sequence
    const int i = block0 + (row >> P.log_pack);      // this row's token and head
    const int head = head0 + (row & (P.pack - 1));
    const int warp_i = block0 + ((quarter * 32) >> P.log_pack);
    const int Ub = b ? 0 : U0;                       // the block's first step
    const bool active = b == 0 || has1;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t o_addr = lane_addr + O_COL + (uint32_t)(b * D);
    const float A = P.a_scale;
    float sb = 0.f;
    if (ALIBI) sb = P.slopes[head] * LOG2E;
    float bias[32];                                  // ALIBI: slope times the column within 32
    if (ALIBI) {
#pragma unroll
      for (int e = 0; e < 32; ++e) bias[e] = sb * (float)e;
    }
    bool ok = !P.fail_first_wait;                    // the self-test: as if the first wait had run out
    float m_ref = 0.f, l0 = 0.f, l1 = 0.f;
    for (int u = Ub; active && ok && u < T; ++u) {
      const int t = T - 1 - u, own = u - Ub;         // key tile, and how many the block has done
      const int buf = NB == 2 ? b : (own & 1);
      const uint32_t s_addr = lane_addr + (uint32_t)(buf * KT);
      const uint32_t phase = NB == 2 ? (uint32_t)(own & 1) : (uint32_t)((own >> 1) & 1);
      ok = __all_sync(0xffffffffu, wait_bar_eager(s_full + buf, phase, abort_flag));
      if (!ok) break;
      tc_fence_after();
      // ---- the row of logits, and its maximum in log2 units (the scale is positive: maximum of the raw logits first, scale after)
      uint32_t r[KT];
      tmem_ld_row(s_addr, r);
      // x2 = a_scale x + slope (j - i) log2 e: the part of the bias that depends on the column within 32 enters here, the rest with the reference
      if (ALIBI) {
#pragma unroll
        for (int e = 0; e < KT; e += 2) {
          float x0, x1;
          fma2v(x0, x1, __uint_as_float(r[e]), __uint_as_float(r[e + 1]), A, bias[e & 31], bias[(e & 31) + 1]);
          r[e] = __float_as_uint(x0);
          r[e + 1] = __float_as_uint(x1);
        }
      }
      if (t * KT + KT - 1 > block0) {                // some row of the block does not see the whole tile
        const int lim = i - t * KT, edge = (warp_i - t * KT) >> 5;      // the mask cuts the same 32 columns for the whole warp
#pragma unroll
        for (int c = 0; c < KT / 32; ++c) {
          const int last = c < edge ? 31 : (c == edge ? (lim & 31) : -1);
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (e > last) r[c * 32 + e] = 0xff800000u;     // -infinity
        }
      }
      const float from = ALIBI ? sb * (float)(t * KT - i) : 0.f;      // of the tile's first column
      float tmax = -INFINITY;
#pragma unroll
      for (int c = 0; c < KT / 32; ++c) {
        float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          m0 = max3(m0, __uint_as_float(r[c * 32 + e]), __uint_as_float(r[c * 32 + e + 1]));
          m1 = max3(m1, __uint_as_float(r[c * 32 + e + 2]), __uint_as_float(r[c * 32 + e + 3]));
        }
        if (ALIBI) tmax = fmaxf(tmax, fmaxf(m0, m1) + fmaf(sb, (float)(c * 32), from));
        else tmax = max3(tmax, m0, m1);
      }
      if (!ALIBI) tmax *= A;
      // ---- the reference: set by the first tile, moved (the row of O and its sum rescaled) when the maximum exceeds it by more than the slack
      if (own == 0) {
        m_ref = fmaxf(tmax, LOWEST) - HEADROOM;      // finite where the tile holds no key for a row yet
      } else {
        const bool move = tmax > m_ref + (HEADROOM + SLACK);
        if (__any_sync(0xffffffffu, move)) {
          const float fac = move ? fast_exp2(m_ref - (tmax - HEADROOM)) : 1.f;
          if (move) m_ref = tmax - HEADROOM;
          l0 *= fac;
          l1 *= fac;
          // rows of O are accumulator lanes of these same threads.  With two blocks the value MMAs of the tiles before have completed (their
          // commit precedes the one that published S); one block that looks ahead has to wait for them.
          if (NB == 1) {
            ok = __all_sync(0xffffffffu, wait_bar(v_done, (uint32_t)((own - 1) & 1), abort_flag));
            if (!ok) break;
            tc_fence_after();
          }
#pragma unroll 1
          for (int oc = 0; oc < D / 16; ++oc) {
            uint32_t w[16];
            tmem_ld_32x16(o_addr + (uint32_t)(oc * 16), w);
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * fac);
            tmem_st_32x16(o_addr + (uint32_t)(oc * 16), w);
          }
          tmem_wait_st();
        }
      }
      // ---- weights 2^(x2 - m_ref), their sum (of the unrounded values), and P over the first half of S in two steps
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int c = half * (KT / 64); c < (half + 1) * (KT / 64); ++c) {
          uint32_t packed[16];
          const float shift = (ALIBI ? fmaf(sb, (float)(c * 32), from) : 0.f) - m_ref;
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            float y0, y1;
            fma2(y0, y1, __uint_as_float(r[c * 32 + e]), __uint_as_float(r[c * 32 + e + 1]), ALIBI ? 1.f : A, shift);
            const float p0 = fast_exp2(y0), p1 = fast_exp2(y1);
            add2(l0, l1, p0, p1);
            packed[e / 2] = pack2<BF16>(p0, p1);
          }
          tmem_st_32x16(s_addr + (uint32_t)(c * 16), packed);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + 2 * buf + half);
      }
    }
    const float l = l0 + l1;
    // ---- output: O / l; NaN where the rows did not arrive
    if (active && ok) ok = __all_sync(0xffffffffu, wait_bar(o_full + b, 0, abort_flag));
    if (active) {
      tc_fence_after();
      const float inv_l = ok ? 1.f / l : nan_f32();
#pragma unroll 1
      for (int oc = 0; oc < D / 32; ++oc) {
        float v[32];
        if (ok) {
          tmem_ld_32x32(o_addr + (uint32_t)(oc * 32), v);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = 0.f;
        }
        if (i < n) {
          uint4* dst = reinterpret_cast<uint4*>(static_cast<unsigned short*>(P.out) + (int64_t)(row0 + i) * P.out_token + (int64_t)head * P.out_head + oc * 32);
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack2<BF16>(v[8 * q4 + 2 * e] * inv_l, v[8 * q4 + 2 * e + 1] * inv_l);
            dst[q4] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
      tc_fence_before();
    }
    if (!ok && lane == 0) *abort_flag = 1;
  }

  // ---- teardown: on the failure path give the copies still in flight a bounded wait, then free tensor memory
  __syncthreads();
  if (tid == 0 && *abort_flag) {
    const int nj = issued[0];
    for (int j = nj > RING ? nj - RING : 0; j < nj; ++j) {
      const bool is_v = j >= 2 && (j & 1) == 0;
      const int u = is_v ? (j - 2) >> 1 : (AHEAD == 1 ? (j == 0 ? 0 : (j + 1) >> 1) : (j < 2 ? j : (j + 1) >> 1));
      if (u >= T) continue;                                    // a position that is never loaded
      (void)mbar_wait_bounded(r_full + (j % RING), (uint32_t)((j / RING) & 1), TC_WAIT_LIMIT);
    }
    (void)mbar_wait_bounded(q_full, 0, TC_WAIT_LIMIT);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, TMEM_COLS);
  }
}

template <int D, bool BF16>
cudaError_t launch_ragged_d(const RaggedParams& P, int64_t slots, int groups, cudaStream_t st) {
  constexpr int NB = D == 256 ? 1 : 2, KT = D == 256 ? 64 : 128;
  constexpr size_t smem = 1024 + (size_t)NB * 128 * D * 2 + (size_t)RING * KT * D * 2 + 32 * 8 + 64;
  static_assert(smem <= 227 * 1024, "shared memory budget of one CTA");
  constexpr size_t smem_req = smem < 120 * 1024 ? 120 * 1024 : smem;   // one CTA per SM: it takes all of tensor memory
  auto go = [&](auto kern) -> cudaError_t {
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_req);
    if (e != cudaSuccess) return e;
    kern<<<dim3((unsigned)slots, (unsigned)groups), threads_of(NB), smem_req, st>>>(P);
    return cudaGetLastError();
  };
  return P.slopes ? go(ragged_kernel<D, true, BF16>) : go(ragged_kernel<D, false, BF16>);
}

}  // namespace

cudaError_t launch_ragged(const RaggedArgs& a, cudaStream_t stream) {
  const int D = a.head_dim, KT = D == 256 ? 64 : 128, group = a.H / a.Hkv;
  RaggedParams P{};
  P.pack = 1;
  while (P.pack < 8 && group % (2 * P.pack) == 0) P.pack *= 2;
  P.log_pack = P.pack == 8 ? 3 : P.pack == 4 ? 2 : P.pack - 1;
  const CUtensorMapDataType type = a.bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  auto map = [&](CUtensorMap* m, const void* base, uint64_t d1, uint64_t s1, uint64_t d2, uint64_t s2, uint32_t b1, uint32_t b2) {
    const uint64_t dims[3] = {(uint64_t)D, d1, d2}, strides[2] = {s1 * 2, s2 * 2};
    const uint32_t box[3] = {64, b1, b2};
    return make_tensor_map(m, type, 3, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
  };
  const uint64_t T = (uint64_t)a.tokens;
  if (!map(&P.tmQ, a.q, (uint64_t)a.H, (uint64_t)a.q_head, T, (uint64_t)a.q_token, (uint32_t)P.pack, 128u >> P.log_pack) ||
      !map(&P.tmK, a.k, T, (uint64_t)a.k_token, (uint64_t)a.Hkv, (uint64_t)a.k_head, (uint32_t)KT, 1) ||
      !map(&P.tmV, a.v, T, (uint64_t)a.v_token, (uint64_t)a.Hkv, (uint64_t)a.v_head, (uint32_t)KT, 1))
    return cudaErrorNotSupported;
  P.out = a.out; P.begin = a.begin; P.slopes = a.slopes;
  P.out_token = a.out_token; P.out_head = a.out_head;
  P.tokens = a.tokens; P.S = a.sequences; P.group = group;
  P.a_scale = a.scale * LOG2E;
  P.fail_first_wait = a.fail_first_wait;
  const int64_t slots = (((int64_t)a.tokens * P.pack) >> (D == 256 ? 7 : 8)) + a.sequences;
  const int groups = a.H / P.pack;
  switch (D) {
    case 64: return a.bf16 ? launch_ragged_d<64, true>(P, slots, groups, stream) : launch_ragged_d<64, false>(P, slots, groups, stream);
    case 128: return a.bf16 ? launch_ragged_d<128, true>(P, slots, groups, stream) : launch_ragged_d<128, false>(P, slots, groups, stream);
    case 256: return a.bf16 ? launch_ragged_d<256, true>(P, slots, groups, stream) : launch_ragged_d<256, false>(P, slots, groups, stream);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kf
