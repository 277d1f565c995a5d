// Causal attention over prompts of different lengths that lie one after the other without padding (kf_prefill_attend_ragged):
// out_i = sum_{j <= i} softmax_j(x_ij) v_j within each sequence, in one pass over its keys.
//
// As in kf_prefill_attend1p.cu a thread is a query row: S = Q K^T and O += P V are tcgen05 MMAs with accumulators in tensor memory (two blocks of 128
// rows: S 2 x 128 columns, O 2 x head_dim), K and V tiles come by TMA through one ring of five slots, and no thread exchanges a maximum or a sum with another.
// What is particular to this kernel:
//   - Operands are binary16 or bfloat16 and lie in any order of heads and tokens (tensor maps with the caller's strides).
//   - A block of 128 rows holds `pack` query heads of a key/value head x 128 / pack tokens, so that a short sequence still fills
//     its rows: row r is token r / pack, head r % pack, which is what a TMA box of 64 features x pack heads x tokens writes.
//   - The grid is laid out without knowing the lengths (slot_sequence).  A CTA per SM starts with its own place and then claims places that
//     have not been launched (cluster launch control); its roles run on across the borders, so that the next queries, keys and logits are there
//     when a block's outputs have been written.  Against a CTA per place: 64 prompts of 256 tokens 152 -> 118 us.
//   - Key tiles are walked from the diagonal back: with ALiBi the nearest keys have the largest logits, so that a row's reference, which
//     only moves when a maximum exceeds it by 2^8, hardly ever moves (MPT-like layer 504 -> 440 us).  The bias enters by one packed multiply-add.
//   - A compute thread reads its whole row of S into registers (the launch's registers are dealt out again between the roles), so that the maximum is
//     known before the first exponential and nothing is done twice; P is handed over in two halves, the second half's exponentials run while
//     the first half's products do.
//   - The warp that issues MMAs runs along together and one lane issues: descriptors then stay in uniform registers (a single
//     thread took 100 cycles per MMA: 1083 -> 960 us for two documents of 8192).
//   - What stands behind the last key of a sequence belongs to others.  Its logits are masked like any later key's; its value rows
//     are overwritten with zeros in shared memory, because 0 * NaN is NaN.
//   - head_dim 256: one block of 128 rows per CTA and key tiles of 64 rows (tensor memory: 2 x 64 columns of S and 256 of O; the logits
//     of the next tile are formed while the current one's softmax runs).
// Output weights are taken times 2^7, so that binary16 holds them from 2^-32 of a row's largest on; bfloat16 (the type V has, which the
// MMA wants for both) rounds them to 8 bits, as much as the output itself is rounded.
//
// What bounds it: two documents of 8192 tokens (32 heads on 8, d 128) take 815 to 966 us from machine to machine, 1.14 to 1.35 PFLOP/s.  A round of both blocks is
// 2800 cycles: the chain of one block (logits to registers, maximum, two halves of exponentials, the last products, the next logits), while the tensor pipe
// is busy for 61 % and the exponential unit for 60 %; back to back the 1000 W limit takes the clock from 1.9 to about 1.5 GHz.  Short prompts (48 of up to
// 97 tokens, 22 us) are three to four items of 6800 cycles per SM, a third of them the stores of the outputs.  Not taken: a share of the exponentials as polynomials
// (1 to 3 % at head_dim 64, nothing at 128); for sequences of one block, the blocks of two groups of heads in one item (200 prompts of 60 tokens, one cache per
// head, 162 -> 119 us, but 64 of 256 4 % slower, 16 of 1024 and head_dim 64 1 to 3 %).
#include "kf_pages.cuh"
#include "kf_tc.cuh"

namespace kf {

namespace {

// A group of four warps for the TMA loads and the MMAs (one warp each), one per block of query rows.  With two blocks the registers of the launch
// (384 x 168) are dealt out again: a compute thread holds its whole row of logits.
constexpr int threads_of(int blocks) { return 128 * (blocks + 1); }
constexpr int FEW_REGS = 40, MANY_REGS = 232;
static_assert(128 * FEW_REGS + 256 * MANY_REGS <= 384 * 168, "registers of the launch");
constexpr int RING = 5;                 // slots that K and V tiles go through in the order of use
constexpr uint32_t TMEM_COLS = 512;
constexpr float HEADROOM = 7.0f;        // log2 units a weight stands above its distance from the reference
constexpr float LOWEST = -1e30f;        // far below every logit that binary32 tells from its neighbours (2^22: there the reference is off by a quarter at most)
constexpr float SLACK = 8.0f;           // log2 units a row's maximum may exceed its reference before the reference moves

struct RaggedParams {
  CUtensorMap tmQ, tmK, tmV;   // [heads][tokens] rows of d; boxes of 64 features x (pack heads x 128 / pack tokens; KT tokens), 128-byte swizzle
  void* out;
  const int32_t* begin;
  const float* slopes;
  int64_t out_token, out_head;
  int32_t tokens, S, pack, log_pack, group;
  int32_t slots, groups;       // of the grid: places per group of heads, groups
  float a_scale;               // logit scale * log2(e)
  bool wide;                   // output rows are aligned to 32 bytes
  int32_t fail_item, leave_item;   // the self-test's: items of a CTA, -1: none
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

// One of the two steps (S = 1, 2) that transpose four sectors of eight words each between four neighbouring threads: afterwards thread j of them holds
// in sector o what was sector j of thread o.
template <int S>
__device__ __forceinline__ void quad_exchange(uint32_t* w) {
  const bool upper = (threadIdx.x & S) != 0;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    if (a & S) continue;
    uint32_t *lo = w + 8 * a, *hi = w + 8 * (a + S);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t got = __shfl_xor_sync(0xffffffffu, upper ? lo[e] : hi[e], S);
      if (upper) lo[e] = got; else hi[e] = got;
    }
  }
}

// What a CTA works on: one pair of blocks (head_dim 256: one block) of one sequence and group of heads.
struct Item {
  int valid;                 // 0: there is nothing more
  int row0, n;               // the sequence's first row and tokens
  int first;                 // the first block's first token within it
  int T, U0;                 // key tiles to walk (step u takes tile T - 1 - u), and the step at which block 0 joins
  int has1, clean;           // whether there is a second block; whether the tile of step 0 holds rows of others
  int head0, kv_head;
};

// Asks for the coordinates of a CTA of this grid that has not been launched, and then never is; 16 bytes to shared memory.
__device__ __forceinline__ void claim_issue(void* answer, uint64_t* bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
               ::"r"(smem_u32(answer)), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ bool claim_read(const void* answer, int& x) {
  uint32_t got, cx;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\t"
      "ld.shared.b128 r, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
      "selp.u32 %1, 1, 0, p;\n\t"
      "mov.u32 %0, 0;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%0, _, _, _}, r;\n\t}"
      : "=&r"(cx), "=&r"(got) : "r"(smem_u32(answer)) : "memory");
  x = (int)cx;
  return got != 0;
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
  constexpr int READERS = 2 + 4 * NB;      // warps that take an item: loads, MMAs, compute
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* sQ = smem;
  unsigned char* sR = sQ + NB * Q_BYTES;
  unsigned char* claim = sR + (size_t)RING * SLOT;                  // the answer to a claim, 16 bytes
  Item* items = reinterpret_cast<Item*>(claim + 16);                // [2]
  uint64_t* bars = reinterpret_cast<uint64_t*>(reinterpret_cast<unsigned char*>(items) + 2 * sizeof(Item));
  uint64_t* item_full = bars;             // [2]
  uint64_t* item_empty = item_full + 2;   // [2]
  uint64_t* claimed = item_empty + 2;
  uint64_t* q_full = claimed + 1;
  uint64_t* q_empty = q_full + 1;
  uint64_t* r_full = q_empty + 1;
  uint64_t* r_empty = r_full + RING;
  uint64_t* s_full = r_empty + RING;      // [2] per block, or per parity of the step
  uint64_t* p_full = s_full + 2;          // [2][2]: the halves of a tile's weights
  uint64_t* o_full = p_full + 4;          // [2]
  uint64_t* o_empty = o_full + 2;         // [2]
  uint64_t* v_done = o_empty + 2;         // one block: the value MMAs of a step have completed
  uint64_t* drain = v_done + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* issued = abort_flag + 1;   // loads that have been issued: of the ring, and of queries
  volatile int* left = issued + 2;         // a role has given up waiting for an item
  volatile int* looked = left + 1;         // the scheduler's claims when it last met a place that holds nothing

  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int tb = 128 >> P.log_pack;                // tokens of a block

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) { mbar_init(item_full + i, 1); mbar_init(item_empty + i, READERS); }
    mbar_init(claimed, 1);
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int s = 0; s < RING; ++s) { mbar_init(r_full + s, 1); mbar_init(r_empty + s, 1); }
    for (int b = 0; b < 2; ++b) {
      mbar_init(s_full + b, 1);
      mbar_init(p_full + 2 * b, 4);
      mbar_init(p_full + 2 * b + 1, 4);
      mbar_init(o_full + b, 1);
      mbar_init(o_empty + b, 4);
    }
    mbar_init(v_done, 1);
    mbar_init(drain, 1);
    *abort_flag = 0;
    issued[0] = issued[1] = 0;
    *left = *looked = 0;
    items[0].T = items[1].T = 0;
    mbar_fence_init();
  }
  // Tensor memory only behind the kernel before: one that lets this one launch early may still have to take its own, and this one waits for its end.
  after_earlier_kernels();
  if (warp == 1) {
    tmem_alloc(tmem_slot, TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  // Every role takes the items in order; number k lies in items[k & 1].  A wait for an item, or for all roles to be done with one, lasts as long as the
  // two items before may (64 times 2^16 polls for every key tile), and begins anew while the scheduler meets places that hold nothing, of which there may be any
  // number.  It does not end when a role has given up a wait within an item: all roles then pass over what is left, up to the item that says there is no more, so
  // that nothing claimed goes without its output.  A role that gives up the wait for an item leaves, and so do all others then; rows that not all of them
  // took become NaN at the end.
  auto wait_item = [&](uint64_t* bar, int k) {
    for (int tries = 0, seen = -1;;) {
      if (__builtin_expect(mbar_wait_bounded(bar + (k & 1), (uint32_t)(k >> 1 & 1), 1u << 16), 1)) return true;
      const int now = *looked;
      tries = now == seen ? tries + 1 : 0;
      seen = now;
      const volatile Item* two = items;
      if (*left || tries > 64 * (1 + two[0].T + two[1].T)) return false;
    }
  };
  auto leave = [&]() {
    if (lane == 0) *left = *abort_flag = 1;
    return false;
  };
  auto take = [&](int k, Item& item) {
    if (__builtin_expect(!__all_sync(0xffffffffu, wait_item(item_full, k)), 0)) return leave();
    item = items[k & 1];
    return item.valid != 0;
  };
  auto release = [&](int k) {
    __syncwarp();
    if (lane == 0) mbar_arrive(item_empty + (k & 1));
  };

  int handed = 0;                                      // the scheduler's: items
  // The ring's order within an item, as the MMA warp needs the tiles: K of step 0; then K of step u + 1 and V of step u in turn; V of the last step.
  if (warp < 4) {
    if (NB == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(FEW_REGS));
    if (warp == 3) {
      // ---------------------------------------------------------- scheduler: this CTA's own place in the grid, then places that it claims
      int place = blockIdx.x, claims = 0;
      bool own = true, more = true;
      constexpr int ROW_SHIFT = NB == 2 ? 8 : 7;           // rows of a place
      int64_t used = P.slots;                              // slots up to the end of the last sequence: the rows of a buffer need not all be somebody's
      for (int k = 0; more; ++k) {
        // the slot of item k - 2 first: nothing is claimed long before it can be worked on
        if (k >= 2 && !__all_sync(0xffffffffu, wait_item(item_empty, k - 2))) {
          (void)leave();
          break;
        }
        Item item{};
        for (;;) {
          if (!own) {
            more = *abort_flag == 0;
            more = __all_sync(0xffffffffu, more) != 0;
            if (!more) break;
            if (lane == 0) {
              mbar_expect_tx(claimed, 16);
              claim_issue(claim, claimed);
            }
            if (claims == 0) {
              const int last = P.begin[P.S];
              if (last >= 0 && last <= P.tokens) used = slot_start(&last, 0, P.pack, ROW_SHIFT, 0) + P.S;
            }
            // as long as two bounded waits: a place that came after that would be nobody's
            more = __all_sync(0xffffffffu, mbar_wait_bounded(claimed, (uint32_t)(claims & 1), 1u << 23)) != 0;
            if (!more && lane == 0) *abort_flag = 1;
            if (!more) break;
            ++claims;
            more = claim_read(claim, place);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the answer has been read before the next one may come
            __syncwarp();
            if (!more) break;
          }
          own = false;
          // The place as a pair of blocks of a sequence; some places hold nothing.
          // All groups of heads of a slot, then the next slot; the slots of a sequence from its end on, so that the longest come first.  (One group
          // after the other, which keeps fewer keys and values in use at a time, ends with a few long places: 416 instead of 373 us for six
          // prompts of up to 4096 tokens and 32 heads, and no gain for 32768 tokens: 8.0 against 7.7 ms.)
          const int slot = P.slots - 1 - place / P.groups, heads = place % P.groups;
          if (slot >= used) {                              // no search: 430 tokens in a buffer of 131072 take 63 instead of 80 us
            if (lane == 0) *looked = claims;
            continue;
          }
          const int seq = slot_sequence(P.begin, P.S, slot, P.pack, ROW_SHIFT, 1);
          const int row0 = P.begin[seq], row_end = P.begin[seq + 1];
          const int64_t local = (slot - slot_start(P.begin, seq, P.pack, ROW_SHIFT, 1)) * (NB * tb);
          if (row0 < 0 || row_end > P.tokens || row0 >= row_end || local < 0 || local >= (int64_t)row_end - row0) {
            if (lane == 0) *looked = claims;
            continue;
          }
          item.valid = 1;
          item.row0 = row0;
          item.n = row_end - row0;
          item.first = (int)local;
          item.has1 = NB == 2 && item.first + tb < item.n;
          const int T0 = (min(item.first + tb, item.n) + KT - 1) / KT;
          item.T = item.has1 ? (min(item.first + 2 * tb, item.n) + KT - 1) / KT : T0;
          item.U0 = item.T - T0;
          item.clean = item.T * KT > item.n && row_end < P.tokens;
          item.head0 = heads * P.pack;
          item.kv_head = item.head0 / P.group;
          break;
        }
        if (lane == 0) {
          items[k & 1] = item;
          mbar_arrive(item_full + (k & 1));
        }
        handed = k + item.valid;
        __syncwarp();
      }
    } else if (warp == 0) {
      // ---------------------------------------------------------- TMA producer
      Item item;
      int slot = 0, count = 0;                                       // ring slot, and loads before
      uint32_t parity = 1;                                           // of the use of the slot before: none yet, such a wait passes at once
      bool ok = true;
      for (int k = 0; take(k, item); ++k) {
        if (lane == 0 && ok) {
          if (k > 0) ok = wait_bar(q_empty, (uint32_t)((k - 1) & 1), abort_flag);
          if (ok) {
            mbar_expect_tx(q_full, item.has1 ? 2 * Q_BYTES : Q_BYTES);
            for (int b = 0; b < (item.has1 ? 2 : 1); ++b)
              for (int kc = 0; kc < KCH; ++kc) tma_load_3d(sQ + b * Q_BYTES + kc * QBOX, &P.tmQ, kc * 64, item.head0, item.row0 + item.first + b * tb, q_full);
            issued[1] = k + 1;
          }
          for (int j = 0; ok && j < 2 * item.T; ++j) {
            const bool is_k = j == 0 || ((j & 1) && (j + 1) / 2 < item.T);
            const int u = is_k ? (j + 1) / 2 : ((j & 1) ? item.T - 1 : (j - 2) / 2);
            ok = wait_bar(r_empty + slot, parity, abort_flag);
            if (!ok) break;
            mbar_expect_tx(r_full + slot, SLOT);
            const CUtensorMap* tm = is_k ? &P.tmK : &P.tmV;
            for (int kc = 0; kc < KCH; ++kc)
              tma_load_3d(sR + (size_t)slot * SLOT + kc * KBOX, tm, kc * 64, item.row0 + (item.T - 1 - u) * KT, item.kv_head, r_full + slot);
            issued[0] = ++count;
            if (++slot == RING) { slot = 0; parity ^= 1; }
          }
          if (!ok) *abort_flag = 1;
        }
        release(k);
      }
    } else if (warp == 1) {
      // ---------------------------------------------------------- MMA issuer: the warp runs along together, one lane issues
      const uint32_t leader = warp_leader();
      const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
      auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bar_eager(bar, parity, abort_flag)) != 0; };
      const uint64_t qd0 = umma_smem_desc(smem_u32(sQ)), kd0 = umma_smem_desc(smem_u32(sR));
      const uint64_t vd0 = umma_desc_mn(smem_u32(sR), KBOX, 1024);   // descriptors of other slots / offsets: + bytes / 16
      // the next tile of the ring: its slot, once it is there
      int ring = 0;
      uint32_t ring_parity = 0;
      auto next_tile = [&](int& slot) {
        slot = ring;
        if (!wait(r_full + ring, ring_parity)) return false;
        if (++ring == RING) { ring = 0; ring_parity ^= 1; }
        return true;
      };
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
      // What stands behind a sequence belongs to others: its value rows become zeros before a product reads them.
      auto clean_rows = [&](int slot, int from) {
        unsigned char* tile = sR + (size_t)slot * SLOT;
        for (int kc = 0; kc < KCH; ++kc)
          for (int i = from * 8 + lane; i < KT * 8; i += 32) reinterpret_cast<uint4*>(tile + kc * KBOX)[i] = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      };
      Item item;
      int steps0 = 0, steps1 = 0, items0 = 0, items1 = 0;            // of the blocks, over all items
      bool ok = true;
      for (int k = 0; take(k, item); ++k) {
        const int T = __shfl_sync(0xffffffffu, item.T, 0), U0 = __shfl_sync(0xffffffffu, item.U0, 0);
        const bool two = NB == 2 && __shfl_sync(0xffffffffu, item.has1, 0) != 0;
        int kslot = 0, vslot = 0, next_k = 0;
        if (ok) ok = wait(q_full, (uint32_t)(k & 1));
        // Logits of the first step (of the first two), then per step and block the value MMAs and the next logits.  The tensor pipe must never run dry
        // between two groups of MMAs, so the waits for tiles stand behind the group before the one that needs them.  A slot is handed back by a commit
        // placed right after the last MMA that reads it.
        for (int u = 0; ok && u < min(AHEAD, T); ++u) {
          ok = next_tile(kslot);
          if (!ok) break;
          tc_fence_after();
          if (u >= U0) qk(0, NB == 2 ? 0 : (steps0 + u) & 1, kslot);
          if (two) qk(1, 1, kslot);
          umma_commit_warp(leader, r_empty + kslot);
        }
        if (ok && T <= AHEAD) umma_commit_warp(leader, q_empty);
        if (ok && NB == 2 && T > 1) ok = next_tile(kslot);
        if (ok) ok = next_tile(vslot);
        if (ok && item.clean) clean_rows(vslot, item.n - (T - 1) * KT);
        if (ok && NB == 1 && T > 2) ok = next_tile(kslot);
        // O of the item before has been read
        if (ok && items0 > 0) ok = wait(o_empty, (uint32_t)((items0 - 1) & 1));
        if (ok && two && items1 > 0) ok = wait(o_empty + 1, (uint32_t)((items1 - 1) & 1));
        for (int u = 0; ok && u < T; ++u) {
          const bool more = u + AHEAD < T;
          const int at0 = steps0 + u - U0, at1 = steps1 + u;         // steps of the blocks, over all items
          const int sb0 = NB == 2 ? 0 : at0 & 1;
          if (u >= U0) {
            if (!pv(0, sb0, vslot, (uint32_t)((NB == 2 ? at0 : at0 >> 1) & 1), u == U0)) { ok = false; break; }
            if (!two) umma_commit_warp(leader, r_empty + vslot);
            if (NB == 1) umma_commit_warp(leader, v_done);
            if (u == T - 1) umma_commit_warp(leader, o_full);
          }
          if (more && u + AHEAD >= U0) qk(0, sb0, kslot);
          if (NB == 2 && u + 2 < T && !next_tile(next_k)) { ok = false; break; }
          if (two) {
            if (!pv(1, 1, vslot, (uint32_t)(at1 & 1), u == 0)) { ok = false; break; }
            if (more) qk(1, 1, kslot);
            else umma_commit_warp(leader, o_full + 1);
            umma_commit_warp(leader, r_empty + vslot);               // both blocks' value MMAs of the step have been issued
          }
          if (more) umma_commit_warp(leader, r_empty + kslot);       // every logit MMA that reads it has been issued
          if (u + AHEAD == T - 1) umma_commit_warp(leader, q_empty);
          if (u + 1 < T) ok = next_tile(vslot);
          if (NB == 1 && ok && u + 3 < T) ok = next_tile(next_k);
          kslot = next_k;
        }
        steps0 += T - U0;
        ++items0;
        if (two) { steps1 += T; ++items1; }
        if (!ok && lane == 0) *abort_flag = 1;
        release(k);
      }
      umma_commit_warp(leader, drain);
      (void)mbar_wait_bounded(drain, 0, TC_WAIT_LIMIT);
    }
  } else {
    if (NB == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(MANY_REGS));
    // ------------------------------------------------------------ compute warps: a thread is a query row
    const int b = NB == 2 ? (warp - 4) >> 2 : 0;
    const int quarter = warp & 3;
    const int row = quarter * 32 + lane;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t o_addr = lane_addr + O_COL + (uint32_t)(b * D);
    const float A = P.a_scale;
    Item item;
    int steps = 0, done = 0;                           // of this block, over all items: steps, items
    bool ok = true;
    for (int k = 0; k != P.leave_item ? take(k, item) : leave(); ++k) {
      if (k == P.fail_item) {                          // the self-test: as if a wait had run out
        ok = false;
        if (lane == 0) *abort_flag = 1;
      }
      if (b == 1 && !item.has1) {
        release(k);
        continue;
      }
      const int T = item.T, n = item.n;
      const int block0 = item.first + b * tb;          // the block's first token within the sequence
      const int i = block0 + (row >> P.log_pack);      // this row's token and head
      const int head = item.head0 + (row & (P.pack - 1));
      const int warp_i = block0 + ((quarter * 32) >> P.log_pack);
      const int Ub = b ? 0 : item.U0;                  // the block's first step
      float sb = 0.f;
      if (ALIBI) sb = P.slopes[head] * LOG2E;
      float bias[32];                                  // ALIBI: slope times the column within 32
      if (ALIBI) {
#pragma unroll
        for (int e = 0; e < 32; ++e) bias[e] = sb * (float)e;
      }
      float m_ref = 0.f, l0 = 0.f, l1 = 0.f;
      uint32_t r[128];
      for (int u = Ub; ok && u < T; ++u) {
        const int t = T - 1 - u, at = steps + u - Ub;  // key tile; step over all items
        const int buf = NB == 2 ? b : (at & 1);
        const uint32_t s_addr = lane_addr + (uint32_t)(buf * KT);
        ok = __all_sync(0xffffffffu, wait_bar_eager(s_full + buf, (uint32_t)((NB == 2 ? at : at >> 1) & 1), abort_flag));
        if (!ok) break;
        tc_fence_after();
        // ---- the row of logits, and its maximum in log2 units (the scale is positive: maximum of the raw logits first, scale after)
        uint32_t(&x)[KT] = reinterpret_cast<uint32_t(&)[KT]>(r);
        tmem_ld_row(s_addr, x);
        // x2 = a_scale x + slope (j - i) log2 e: the part of the bias that depends on the column within 32 enters here, the rest with the reference
        if (ALIBI) {
#pragma unroll
          for (int e = 0; e < KT; e += 2) {
            float x0, x1;
            fma2v(x0, x1, __uint_as_float(x[e]), __uint_as_float(x[e + 1]), A, bias[e & 31], bias[(e & 31) + 1]);
            x[e] = __float_as_uint(x0);
            x[e + 1] = __float_as_uint(x1);
          }
        }
        const bool second_empty = ((warp_i - t * KT) >> 5) < KT / 64;
        if (t * KT + KT - 1 > block0) {                // some row of the block does not see the whole tile
          const int lim = i - t * KT, edge = (warp_i - t * KT) >> 5;      // the mask cuts the same 32 columns for the whole warp
#pragma unroll
          for (int c = 0; c < KT / 32; ++c) {
            const int last = c < edge ? 31 : (c == edge ? (lim & 31) : -1);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (e > last) x[c * 32 + e] = 0xff800000u;     // -infinity
          }
        }
        const float from = ALIBI ? sb * (float)(t * KT - i) : 0.f;        // of the tile's first column
        float tmax = -INFINITY;
#pragma unroll
        for (int c = 0; c < KT / 32; ++c) {
          float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            m0 = max3(m0, __uint_as_float(x[c * 32 + e]), __uint_as_float(x[c * 32 + e + 1]));
            m1 = max3(m1, __uint_as_float(x[c * 32 + e + 2]), __uint_as_float(x[c * 32 + e + 3]));
          }
          if (ALIBI) tmax = fmaxf(tmax, fmaxf(m0, m1) + fmaf(sb, (float)(c * 32), from));
          else tmax = max3(tmax, m0, m1);
        }
        if (!ALIBI) tmax *= A;
        // ---- the reference: set by the first tile, moved (the row of O and its sum rescaled) when the maximum exceeds it by more than the slack
        if (u == Ub) {
          m_ref = fmaxf(tmax, LOWEST) - HEADROOM;      // finite where the tile holds no key for a row yet
        } else {
          const bool move = tmax > m_ref + (HEADROOM + SLACK);
          if (__any_sync(0xffffffffu, move)) {
            const float fac = move ? fast_exp2(m_ref - (tmax - HEADROOM)) : 1.f;
            if (move) m_ref = tmax - HEADROOM;
            l0 *= fac;
            l1 *= fac;
            // rows of O are accumulator lanes of these same threads.  With two blocks the value MMAs of the steps before have completed (their
            // commit precedes the one that published S); one block that looks ahead has to wait for them.
            if (NB == 1) {
              ok = __all_sync(0xffffffffu, wait_bar_eager(v_done, (uint32_t)((at - 1) & 1), abort_flag));
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
          // The second half may hold no key that a row of the warp sees.  The branch also keeps its exponentials behind the first half's hand-over (two
          // documents of 8192: 972 us without it, 935 with).
          if (half == 1 && second_empty) {
            const uint32_t none[16] = {};
#pragma unroll
            for (int c = KT / 64; c < KT / 32; ++c) tmem_st_32x16(s_addr + (uint32_t)(c * 16), none);
          } else {
#pragma unroll
            for (int c = half * (KT / 64); c < (half + 1) * (KT / 64); ++c) {
              uint32_t packed[16];
              const float shift = (ALIBI ? fmaf(sb, (float)(c * 32), from) : 0.f) - m_ref;
#pragma unroll
              for (int e = 0; e < 32; e += 2) {
                float y0, y1;
                fma2(y0, y1, __uint_as_float(x[c * 32 + e]), __uint_as_float(x[c * 32 + e + 1]), ALIBI ? 1.f : A, shift);
                const float p0 = fast_exp2(y0), p1 = fast_exp2(y1);
                add2(l0, l1, p0, p1);
                packed[e / 2] = pack2<BF16>(p0, p1);
              }
              tmem_st_32x16(s_addr + (uint32_t)(c * 16), packed);
            }
          }
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full + 2 * buf + half);
        }
      }
      steps += T - Ub;
      // ---- output: O / l; NaN where the rows did not arrive
      if (ok) ok = __all_sync(0xffffffffu, wait_bar_eager(o_full + b, (uint32_t)(done & 1), abort_flag));
      ++done;
      if (ok) tc_fence_after();
      else if (lane == 0) *abort_flag = 1;
      const float inv_l = ok ? 1.f / (l0 + l1) : nan_f32();
      constexpr int PIECE = D < 128 ? D : 128;
#pragma unroll
      for (int oc = 0; oc < D; oc += PIECE) {
        uint32_t(&v)[PIECE] = reinterpret_cast<uint32_t(&)[PIECE]>(r);
        if (ok) {
          tmem_ld_row(o_addr + (uint32_t)oc, v);
          if (oc + PIECE == D) {                       // the next item's products may write O
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_empty + b);
          }
        } else {
#pragma unroll
          for (int e = 0; e < PIECE; ++e) v[e] = 0u;
        }
        uint32_t w[PIECE / 2];                         // the thread's row, rounded
#pragma unroll
        for (int e = 0; e < PIECE / 2; ++e) w[e] = pack2<BF16>(__uint_as_float(v[2 * e]) * inv_l, __uint_as_float(v[2 * e + 1]) * inv_l);
        if (P.wide && block0 + tb <= n) {
          // Whole blocks: four threads exchange sectors of 32 bytes, so that together they store 128 consecutive bytes of a row, as a store takes as many
          // cycles as it touches lines (16 prompts of 1024: 192 -> 177 us).  Where rows are missing the exchange costs more than it saves.
#pragma unroll
          for (int g = 0; g < PIECE / 2; g += 32) {
            quad_exchange<1>(w + g);
            quad_exchange<2>(w + g);
#pragma unroll
            for (int o = 0; o < 4; ++o) {              // row o of the quad, sector lane & 3 of these four
              const int rr = quarter * 32 + (lane & 28) + o, ii = block0 + (rr >> P.log_pack);
              unsigned short* dst = static_cast<unsigned short*>(P.out) + (int64_t)(item.row0 + ii) * P.out_token +
                                    (int64_t)(item.head0 + (rr & (P.pack - 1))) * P.out_head + oc + 2 * g + (lane & 3) * 16;
              store_sector(dst, w + g + 8 * o);
            }
          }
        } else if (i < n) {
          unsigned short* dst = static_cast<unsigned short*>(P.out) + (int64_t)(item.row0 + i) * P.out_token + (int64_t)head * P.out_head + oc;
#pragma unroll
          for (int q = 0; q < PIECE / 16; ++q) {
            if (P.wide) {
              store_sector(dst + 16 * q, w + 8 * q);
            } else {
              reinterpret_cast<uint4*>(dst)[2 * q] = make_uint4(w[8 * q], w[8 * q + 1], w[8 * q + 2], w[8 * q + 3]);
              reinterpret_cast<uint4*>(dst)[2 * q + 1] = make_uint4(w[8 * q + 4], w[8 * q + 5], w[8 * q + 6], w[8 * q + 7]);
            }
          }
        }
      }
      release(k);
    }
  }

  // ---- teardown: on the failure path give the copies still in flight a bounded wait and rows that not every role took NaN, then free tensor memory
  tc_fence_before();
  __syncthreads();
  if (__builtin_expect(warp == 3 && *abort_flag, 0))
    for (int k = max(handed - 2, 0); k < handed; ++k) {
      if (mbar_test(item_empty + (k & 1), (uint32_t)(k >> 1 & 1))) continue;
      const Item item = items[k & 1];                  // of this slot the last one that was handed out: the next would have waited for it
      const int rows = min(NB * tb, item.n - item.first), pieces = D / 8;
      for (int e = lane; e < rows * P.pack * pieces; e += 32) {
        const int row = e / pieces, i = item.row0 + item.first + (row >> P.log_pack), head = item.head0 + (row & (P.pack - 1));
        *reinterpret_cast<uint4*>(static_cast<unsigned short*>(P.out) + (int64_t)i * P.out_token + (int64_t)head * P.out_head + e % pieces * 8) =
            make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
      }
    }
  if (tid == 0 && *abort_flag) {
    for (int j = issued[0] > RING ? issued[0] - RING : 0; j < issued[0]; ++j)
      (void)mbar_wait_bounded(r_full + (j % RING), (uint32_t)((j / RING) & 1), TC_WAIT_LIMIT);
    if (issued[1] > 0) (void)mbar_wait_bounded(q_full, (uint32_t)((issued[1] - 1) & 1), TC_WAIT_LIMIT);
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, TMEM_COLS);
  }
}

template <int D, bool BF16>
cudaError_t launch_ragged_d(const RaggedParams& P, cudaStream_t st) {
  constexpr int NB = D == 256 ? 1 : 2, KT = D == 256 ? 64 : 128;
  constexpr size_t smem = 1024 + (size_t)NB * 128 * D * 2 + (size_t)RING * KT * D * 2 + 16 + 2 * sizeof(Item) + 32 * 8 + 64;
  static_assert(smem <= 227 * 1024, "shared memory budget of one CTA");
  constexpr size_t smem_req = smem < 120 * 1024 ? 120 * 1024 : smem;   // one CTA per SM: it takes all of tensor memory
  auto go = [&](auto kern) -> cudaError_t {
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_req);
    if (e != cudaSuccess) return e;
    return launch_early(kern, dim3((unsigned)(P.slots * P.groups)), threads_of(NB), smem_req, st, P);
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
  P.wide = reinterpret_cast<uintptr_t>(a.out) % 32 == 0 && a.out_token % 16 == 0 && a.out_head % 16 == 0;
  P.tokens = a.tokens; P.S = a.sequences; P.group = group;
  P.a_scale = a.scale * LOG2E;
  P.fail_item = a.fail_item;
  P.leave_item = a.leave_item;
  const int64_t slots = (((int64_t)a.tokens * P.pack) >> (D == 256 ? 7 : 8)) + a.sequences;
  P.groups = a.H / P.pack;
  if (slots * P.groups > INT32_MAX) return cudaErrorInvalidValue;
  P.slots = (int32_t)slots;
  switch (D) {
    case 64: return a.bf16 ? launch_ragged_d<64, true>(P, stream) : launch_ragged_d<64, false>(P, stream);
    case 128: return a.bf16 ? launch_ragged_d<128, true>(P, stream) : launch_ragged_d<128, false>(P, stream);
    case 256: return a.bf16 ? launch_ragged_d<256, true>(P, stream) : launch_ragged_d<256, false>(P, stream);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kf
