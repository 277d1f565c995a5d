// The closing stage of a generation step, shared by the kernels that follow a streaming kernel: merge the split
// partials, normalise the scores, add them into f_theta, pick the entry to evict and write the new token's row into
// the freed slot.  PARAMS is DecodeParams (binary16 rows) or a type derived from it that brings a row format of its
// own: the struct CloseRow is what differs between the two.
#pragma once

#include "kf_decode.cuh"

namespace kf {

namespace {

constexpr int MAX_SPLITS = 64;   // CTAs per unit (the closing CTA keeps one weight per split in shared memory)

// Threads of a closing CTA.  Few units with long caches take the 512-thread form.
inline bool close_is_wide(int units, int k) { return units <= 148 && k >= 2048; }
__host__ __device__ constexpr int close_threads(int d, int g) { return g == 1 ? 128 : (128 * (g < 4 ? g : 4) < d ? d : 128 * (g < 4 ? g : 4)); }

// What a row format adds to the closing stage; the primary template is the binary16 cache.  A thread holds the columns
// tid + i NT of the new token's row.
template <class PARAMS, int D, int NT, int CPT>
struct CloseRow {
  __half kn[CPT], vn[CPT];
  static __device__ __forceinline__ float noise(const PARAMS& P, uint32_t b, uint32_t lh, uint32_t i, uint32_t j) {
    return noise_for(P, b, lh, i, j);
  }
  // Called by every thread with the columns loaded, before the streaming kernel's results are waited for.
  __device__ __forceinline__ void prepare(const PARAMS&, int) {}
  // Whether the streaming kernel marks the statistics of a split that it could not finish (sums of -1); the context's
  // kernels report through its error word instead.
  static constexpr bool MARKS_FAILURES = false;
  // Called by every thread of a full unit that has no entry to evict.
  static __device__ __forceinline__ void nothing_to_evict(const PARAMS& P, int) {
    if (threadIdx.x == 0) atomicExch(P.err, ERR_BOUNDS);
  }
  // Called once by every thread: the row goes to `slot`, or nowhere if slot is -1.
  __device__ __forceinline__ void store(const PARAMS& P, int u, int slot) const {
    if (slot < 0) return;
    __half* Kr = const_cast<__half*>(P.K) + ((size_t)u * P.k + slot) * D;
    __half* Vr = const_cast<__half*>(P.V) + ((size_t)u * P.k + slot) * D;
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int c = threadIdx.x + i * NT;
      if (c < D) { Kr[c] = kn[i]; Vr[c] = vn[i]; }
    }
  }
};

__device__ __forceinline__ unsigned long long evict_key(float a, int pos) {
  // smallest key = smallest accumulated score; equal scores: the higher position leaves
  return ((unsigned long long)__float_as_uint(a) << 32) | (unsigned long long)(0xFFFFFFFFu - (uint32_t)pos);
}

// A unit whose rows did not all arrive: its outputs and scores say so, its state stays as it was.
template <int D, int NT, int G, class PARAMS>
__device__ __forceinline__ void report_failure(const PARAMS& P, int u, int len) {
  const float nan = __int_as_float(0x7fc00000);
  for (int c = threadIdx.x; c < G * D; c += NT) P.out[(size_t)u * G * D + c] = __float2half_rn(nan);
  if (P.score_opt)
    for (int j = threadIdx.x; j <= len; j += NT) P.score_opt[(size_t)u * (P.k + 1) + j] = nan;
  if (P.slot_opt && threadIdx.x == 0) P.slot_opt[u] = ERR_TIMEOUT;
}

// The eviction decision and the replacement, common to every form of the closing stage: `best` / `best_j` are the
// thread's smallest eviction key (accumulated score, inverted position) among its non-recent entries and its slot,
// z_new the new token's own score, `row` the new token's row.
template <int D, int NT, int CPT, class PARAMS>
__device__ __forceinline__ void evict_and_replace(const PARAMS& P, int u, int len, unsigned long long best, int best_j,
                                                  float z_new, const CloseRow<PARAMS, D, NT, CPT>& row) {
  __shared__ unsigned long long sh_key[NT / 32];
  __shared__ int sh_j[NT / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int BATCH = 8;
  float* __restrict__ acc = P.acc + (size_t)u * P.k;
  int32_t* __restrict__ pos = P.pos + (size_t)u * P.k;
  const unsigned long long key_new = evict_key(z_new, P.p);
  int slot;   // where the new token's row goes
  if (len < P.k) {  // cache not full yet: append
    slot = len;
    if (tid == 0) P.len[u] = len + 1;
  } else {
    // smallest key over the CTA: warp minimum by shuffles, the owning lane publishes it with its slot
    const unsigned long long mine = best;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o);
      best = other < best ? other : best;
    }
    if (best == ~0ull ? lane == 0 : mine == best) { sh_key[warp] = best; sh_j[warp] = best_j; }   // keys are unique
    __syncthreads();
    best = sh_key[0];
    slot = sh_j[0];
#pragma unroll
    for (int wi = 1; wi < NT / 32; ++wi)
      if (sh_key[wi] < best) { best = sh_key[wi]; slot = sh_j[wi]; }
    if (P.w == 0 && key_new < best) { row.store(P, u, -1); return; }  // the new token itself has the lowest score: it is not stored
    if (best == ~0ull || slot < 0 || slot >= len) {  // not with 0 <= w <= k and distinct positions before the new one: report it instead of guessing
      row.nothing_to_evict(P, u);
      return;
    }
  }
  if (P.place) {
    // the entries behind the one that leaves move up one place; the new token takes the last place
    int32_t* __restrict__ place = P.place + (size_t)u * P.k;
    if (len >= P.k) {
      const int pos_out = (int)(0xffffffffu - (uint32_t)best);   // the key's low word is 2^32 - 1 - position
      for (int j0 = tid; j0 < len; j0 += NT * BATCH) {   // loads of a batch first, so that they overlap
        int pp[BATCH], pl[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const int j = j0 + i * NT;
          pp[i] = j < len ? pos[j] : -1;
          pl[i] = j < len ? place[j] : 0;
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const int j = j0 + i * NT;
          if (j != slot && pp[i] > pos_out) place[j] = pl[i] - 1;   // pp = -1 beyond the end never passes
        }
      }
    }
    if (tid == 0) place[slot] = len < P.k ? len : P.k - 1;
  }
  if (tid == 0) { pos[slot] = P.p; acc[slot] = z_new; }
  row.store(P, u, slot);
}

// Closing a unit: merge splits, normalise, accumulate, evict, replace.  Everything that does not depend on the
// streaming kernel (scores and positions of the entries, the new token's own logit) is requested before
// `griddepcontrol.wait`, i.e. while the streaming kernel's last CTAs are still running.
// G query heads share the unit's cache (G = 1: the method as printed): every head has its own split partials,
// adjusted logits and output row; the score added to f_theta is the mean of the heads' softmaxes (Eq. 11).
template <int D, int NT, int G, class PARAMS>
__device__ void combine_and_evict(const PARAMS& P, int u, int len) {
  const int tid = threadIdx.x, lane = tid & 31;
  const int Hkv = P.H / G;
  const uint32_t b = (uint32_t)(u / Hkv), h0 = (uint32_t)(u % Hkv) * G, lh0 = (uint32_t)P.layer * P.H + h0;
  const __half* q = P.q + (size_t)u * G * D;
  const __half* kn = P.knew + (size_t)u * D;
  const __half* vn = P.vnew + (size_t)u * D;
  constexpr int PSTRIDE = 4 + D;
  constexpr int CPT = (D + NT - 1) / NT;   // output columns per thread
  constexpr float INV_G = 1.0f / (float)G;
  const float* part = P.partials + (size_t)u * P.splits * G * PSTRIDE;   // [split][head][4 + D]
  float* __restrict__ acc = P.acc + (size_t)u * P.k;
  int32_t* __restrict__ pos = P.pos + (size_t)u * P.k;
  const float* __restrict__ ys = P.y_scratch + (size_t)u * G * (P.k + 1);   // [head][k + 1]

  // ---- independent of the streaming kernel: scores and positions of the first batch of entries, the new
  //      token's row, its own logit and adjusted logit (every warp computes these for itself: no hand-over)
  constexpr int BATCH = 8;   // 64 registers per thread keep all closing CTAs of 1024 units resident at once
  float yv[BATCH], av[BATCH];
  int pv[BATCH];
#pragma unroll
  for (int i = 0; i < BATCH; ++i) {
    const int j = tid + i * NT;
    const bool in = j < len;
    av[i] = in ? acc[j] : 0.f;
    pv[i] = in ? pos[j] : 0x7fffffff;
  }
  // entries beyond the first batch: pull their scores and positions into L2 (one request per 128-byte line)
  for (int line = tid + (NT * BATCH) / 32; line * 32 < len; line += NT) {
    asm volatile("prefetch.global.L2 [%0];" ::"l"(acc + line * 32));
    asm volatile("prefetch.global.L2 [%0];" ::"l"(pos + line * 32));
  }
  CloseRow<PARAMS, D, NT, CPT> row;
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    const int c = tid + i * NT;
    row.kn[i] = c < D ? kn[c] : __float2half(0.f);
    row.vn[i] = c < D ? vn[c] : __float2half(0.f);
  }
  row.prepare(P, u);
  float x_new[G], y_new[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    float s = 0.f;
    for (int c = lane; c < D; c += 32) s = fmaf(__half2float(q[g * D + c]), __half2float(kn[c]), s);
    x_new[g] = warp_sum(s) * P.scale;  // bias(p, p) = 0
    float yn = 0.f;
    if (lane == 0) yn = (x_new[g] + CloseRow<PARAMS, D, NT, CPT>::noise(P, b, lh0 + g, (uint32_t)P.p, (uint32_t)P.p)) * P.inv_tau;
    y_new[g] = __shfl_sync(0xffffffffu, yn, 0);
  }

  asm volatile("griddepcontrol.wait;" ::: "memory");   // the streaming kernel has finished; its writes are visible

  // ---- everything the streaming kernel produced is requested at once
  if (G == 1) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int j = tid + i * NT;
      yv[i] = j < len ? __ldcg(ys + j) : 0.f;
    }
  }
  float my[G], inv_ly[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    // (max, sum) pairs of both softmaxes: split `lane` and split `lane + 32`
    float4 ps0 = make_float4(-INFINITY, 0.f, -INFINITY, 0.f), ps1 = ps0;
    if (lane < P.splits) ps0 = __ldcg(reinterpret_cast<const float4*>(part + ((size_t)lane * G + g) * PSTRIDE));
    if (lane + 32 < P.splits) ps1 = __ldcg(reinterpret_cast<const float4*>(part + ((size_t)(lane + 32) * G + g) * PSTRIDE));
    if constexpr (CloseRow<PARAMS, D, NT, CPT>::MARKS_FAILURES) {
      if (__any_sync(0xffffffffu, ps0.y < 0.f || ps1.y < 0.f)) {   // every warp looks at the same statistics
        report_failure<D, NT, G>(P, u, len);
        return;
      }
    }
    const float mx = warp_max(fmaxf(x_new[g], fmaxf(ps0.y > 0.f ? ps0.x : -INFINITY, ps1.y > 0.f ? ps1.x : -INFINITY)));
    my[g] = warp_max(fmaxf(y_new[g], fmaxf(ps0.w > 0.f ? ps0.z : -INFINITY, ps1.w > 0.f ? ps1.z : -INFINITY)));
    const float w0 = ps0.y > 0.f ? fast_exp2((ps0.x - mx) * LOG2E) : 0.f;   // weight of split `lane` in the output
    const float w1 = ps1.y > 0.f ? fast_exp2((ps1.x - mx) * LOG2E) : 0.f;
    float lx = fmaf(ps0.y, w0, ps1.y * w1);
    float ly = (ps0.w > 0.f ? ps0.w * fast_exp2((ps0.z - my[g]) * LOG2E) : 0.f) + (ps1.w > 0.f ? ps1.w * fast_exp2((ps1.z - my[g]) * LOG2E) : 0.f);
    const float inv_lx = 1.f / (warp_sum(lx) + fast_exp2((x_new[g] - mx) * LOG2E));
    inv_ly[g] = 1.f / (warp_sum(ly) + fast_exp2((y_new[g] - my[g]) * LOG2E));

    // ---- attention output of this head (Eq. 1): merged partial sums plus the new token's own value row
    float o[CPT];
#pragma unroll
    for (int i = 0; i < CPT; ++i) o[i] = fast_exp2((x_new[g] - mx) * LOG2E) * __half2float(row.vn[i]);
#pragma unroll 4
    for (int sp = 0; sp < P.splits; ++sp) {
      const float w = __shfl_sync(0xffffffffu, sp < 32 ? w0 : w1, sp & 31);
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        const int c = tid + i * NT;
        if (c < D) o[i] = fmaf(__ldcg(part + ((size_t)sp * G + g) * PSTRIDE + 4 + c), w, o[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int c = tid + i * NT;
      if (c < D) P.out[((size_t)u * G + g) * D + c] = __float2half_rn(o[i] * inv_lx);
    }
  }

  // ---- score (Eq. 11; the mean over the group's heads), accumulation and the eviction candidate
  float* __restrict__ sc = P.score_opt ? P.score_opt + (size_t)u * (P.k + 1) : nullptr;
  unsigned long long best = ~0ull;
  int best_j = -1;
  const int cutoff = P.p - P.w;  // entries with pos <= cutoff are outside the recent window
  for (int j0 = tid; j0 < len; j0 += NT * BATCH) {
    if (j0 != tid) {   // the first batch was loaded above
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int j = j0 + i * NT;
        const bool in = j < len;
        if (G == 1) yv[i] = in ? __ldcg(ys + j) : 0.f;
        av[i] = in ? acc[j] : 0.f;
        pv[i] = in ? pos[j] : 0x7fffffff;
      }
    }
    float zv[BATCH];
    if (G == 1) {
#pragma unroll
      for (int i = 0; i < BATCH; ++i) zv[i] = fast_exp2((yv[i] - my[0]) * LOG2E) * inv_ly[0];
    } else {
#pragma unroll
      for (int i = 0; i < BATCH; ++i) zv[i] = 0.f;
#pragma unroll
      for (int g = 0; g < G; ++g) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const int j = j0 + i * NT;
          yv[i] = j < len ? __ldcg(ys + (size_t)g * (P.k + 1) + j) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) zv[i] = fmaf(fast_exp2((yv[i] - my[g]) * LOG2E), inv_ly[g], zv[i]);
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) zv[i] *= INV_G;
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int j = j0 + i * NT;
      if (j < len) {
        const float z = zv[i];
        const float a = av[i] + z;
        acc[j] = a;
        if (sc) sc[j] = z;
        if (pv[i] <= cutoff) {
          const unsigned long long key = evict_key(a, pv[i]);
          if (key < best) { best = key; best_j = j; }
        }
      }
    }
  }
  float z_new = 0.f;
#pragma unroll
  for (int g = 0; g < G; ++g) z_new = fmaf(fast_exp2((y_new[g] - my[g]) * LOG2E), inv_ly[g], z_new);
  if (G > 1) z_new *= INV_G;
  if (sc && tid == 0) sc[len] = z_new;
  evict_and_replace<D, NT, CPT>(P, u, len, best, best_j, z_new, row);
}

// The closing stage with many threads per unit (NT = 128 * min(G, 4) for G > 1 query heads on one cache, so that the heads are
// worked on side by side instead of one after the other; 512 for a single head with a long cache and few units): warp n merges the split statistics of head n and leaves them in shared
// memory; then every thread owns one (head, column) of the outputs and a few entries of the score update, all of whose
// loads are issued together.
// BATCH: entries per thread and round.  EARLY: the adjusted logits of the first round are requested together with the
// split statistics instead of after them (G * BATCH more registers).
template <int D, int NT, int G, int BATCH = 4, bool EARLY = false, class PARAMS>
__device__ void combine_and_evict_group(const PARAMS& P, int u, int len) {
  static_assert(NT >= 32 * G && NT >= D, "one warp per head for the statistics, one thread per column of the new row");
  __shared__ float sh_mx[G], sh_inv_lx[G], sh_my[G], sh_inv_ly[G], sh_xnew[G], sh_ynew[G];
  __shared__ float sh_w[G][MAX_SPLITS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int Hkv = P.H / G;
  const uint32_t b = (uint32_t)(u / Hkv), h0 = (uint32_t)(u % Hkv) * G, lh0 = (uint32_t)P.layer * P.H + h0;
  const __half* q = P.q + (size_t)u * G * D;
  const __half* kn = P.knew + (size_t)u * D;
  const __half* vn = P.vnew + (size_t)u * D;
  constexpr int PSTRIDE = 4 + D;
  constexpr float INV_G = 1.0f / (float)G;
  const float* part = P.partials + (size_t)u * P.splits * G * PSTRIDE;   // [split][head][4 + D]
  float* __restrict__ acc = P.acc + (size_t)u * P.k;
  int32_t* __restrict__ pos = P.pos + (size_t)u * P.k;
  const float* __restrict__ ys = P.y_scratch + (size_t)u * G * (P.k + 1);   // [head][k + 1]

  // ---- independent of the streaming kernel
  float av[BATCH];
  int pv[BATCH];
#pragma unroll
  for (int i = 0; i < BATCH; ++i) {
    const int j = tid + i * NT;
    const bool in = j < len;
    av[i] = in ? acc[j] : 0.f;
    pv[i] = in ? pos[j] : 0x7fffffff;
  }
  for (int line = tid + (NT * BATCH) / 32; line * 32 < len; line += NT) {
    asm volatile("prefetch.global.L2 [%0];" ::"l"(acc + line * 32));
    asm volatile("prefetch.global.L2 [%0];" ::"l"(pos + line * 32));
  }
  CloseRow<PARAMS, D, NT, 1> row;
  row.kn[0] = tid < D ? kn[tid] : __float2half(0.f);
  row.vn[0] = tid < D ? vn[tid] : __float2half(0.f);
  row.prepare(P, u);
  float x_new = 0.f, y_new = 0.f;
  if (warp < G) {   // warp n: head n's logit of the new token against itself
    float s = 0.f;
    for (int c = lane; c < D; c += 32) s = fmaf(__half2float(q[warp * D + c]), __half2float(kn[c]), s);
    x_new = warp_sum(s) * P.scale;  // bias(p, p) = 0
    if (lane == 0) y_new = (x_new + CloseRow<PARAMS, D, NT, 1>::noise(P, b, lh0 + warp, (uint32_t)P.p, (uint32_t)P.p)) * P.inv_tau;
    y_new = __shfl_sync(0xffffffffu, y_new, 0);
  }

  asm volatile("griddepcontrol.wait;" ::: "memory");   // the streaming kernel has finished; its writes are visible

  float yv[G][BATCH];
  auto load_y = [&](int j0) {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int j = j0 + i * NT;
        yv[g][i] = j < len ? __ldcg(ys + (size_t)g * (P.k + 1) + j) : 0.f;
      }
  };
  if (EARLY) load_y(tid);
  bool lost = false;
  if (warp < G) {
    const int g = warp;
    float4 ps0 = make_float4(-INFINITY, 0.f, -INFINITY, 0.f), ps1 = ps0;
    if (lane < P.splits) ps0 = __ldcg(reinterpret_cast<const float4*>(part + ((size_t)lane * G + g) * PSTRIDE));
    if (lane + 32 < P.splits) ps1 = __ldcg(reinterpret_cast<const float4*>(part + ((size_t)(lane + 32) * G + g) * PSTRIDE));
    if constexpr (CloseRow<PARAMS, D, NT, 1>::MARKS_FAILURES) lost = __any_sync(0xffffffffu, ps0.y < 0.f || ps1.y < 0.f);
    const float mx = warp_max(fmaxf(x_new, fmaxf(ps0.y > 0.f ? ps0.x : -INFINITY, ps1.y > 0.f ? ps1.x : -INFINITY)));
    const float my = warp_max(fmaxf(y_new, fmaxf(ps0.w > 0.f ? ps0.z : -INFINITY, ps1.w > 0.f ? ps1.z : -INFINITY)));
    const float w0 = ps0.y > 0.f ? fast_exp2((ps0.x - mx) * LOG2E) : 0.f;
    const float w1 = ps1.y > 0.f ? fast_exp2((ps1.x - mx) * LOG2E) : 0.f;
    const float lx = fmaf(ps0.y, w0, ps1.y * w1);
    const float ly = (ps0.w > 0.f ? ps0.w * fast_exp2((ps0.z - my) * LOG2E) : 0.f) + (ps1.w > 0.f ? ps1.w * fast_exp2((ps1.z - my) * LOG2E) : 0.f);
    const float inv_lx = 1.f / (warp_sum(lx) + fast_exp2((x_new - mx) * LOG2E));
    const float inv_ly = 1.f / (warp_sum(ly) + fast_exp2((y_new - my) * LOG2E));
    sh_w[g][lane] = w0;
    sh_w[g][lane + 32] = w1;
    if (lane == 0) { sh_mx[g] = mx; sh_inv_lx[g] = inv_lx; sh_my[g] = my; sh_inv_ly[g] = inv_ly; sh_xnew[g] = x_new; sh_ynew[g] = y_new; }
  }
  if constexpr (CloseRow<PARAMS, D, NT, 1>::MARKS_FAILURES) {
    if (__syncthreads_or(lost)) {
      report_failure<D, NT, G>(P, u, len);
      return;
    }
  } else {
    __syncthreads();
  }

  // ---- attention outputs (Eq. 1): one (head, column) per thread and round
  for (int idx = tid; idx < G * D; idx += NT) {
    const int g = idx / D, c = idx % D;
    float o = fast_exp2((sh_xnew[g] - sh_mx[g]) * LOG2E) * __half2float(vn[c]);
    const float* col = part + (size_t)g * PSTRIDE + 4 + c;
#pragma unroll 8
    for (int sp = 0; sp < P.splits; ++sp) o = fmaf(__ldcg(col + (size_t)sp * G * PSTRIDE), sh_w[g][sp], o);
    P.out[((size_t)u * G + g) * D + c] = __float2half_rn(o * sh_inv_lx[g]);
  }

  // ---- score (Eq. 11; the mean over the group's heads), accumulation and the eviction candidate
  float my[G], inv_ly[G];
#pragma unroll
  for (int g = 0; g < G; ++g) { my[g] = sh_my[g]; inv_ly[g] = sh_inv_ly[g] * INV_G; }
  float* __restrict__ sc = P.score_opt ? P.score_opt + (size_t)u * (P.k + 1) : nullptr;
  unsigned long long best = ~0ull;
  int best_j = -1;
  const int cutoff = P.p - P.w;  // entries with pos <= cutoff are outside the recent window
  for (int j0 = tid; j0 < len; j0 += NT * BATCH) {
    if (j0 != tid) {
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int j = j0 + i * NT;
        const bool in = j < len;
        av[i] = in ? acc[j] : 0.f;
        pv[i] = in ? pos[j] : 0x7fffffff;
      }
    }
    if (!EARLY || j0 != tid) load_y(j0);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int j = j0 + i * NT;
      if (j < len) {
        float z = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) z = fmaf(fast_exp2((yv[g][i] - my[g]) * LOG2E), inv_ly[g], z);
        const float a = av[i] + z;
        acc[j] = a;
        if (sc) sc[j] = z;
        if (pv[i] <= cutoff) {
          const unsigned long long key = evict_key(a, pv[i]);
          if (key < best) { best = key; best_j = j; }
        }
      }
    }
  }
  float z_new = 0.f;
#pragma unroll
  for (int g = 0; g < G; ++g) z_new = fmaf(fast_exp2((sh_ynew[g] - my[g]) * LOG2E), inv_ly[g], z_new);
  if (sc && tid == 0) sc[len] = z_new;
  evict_and_replace<D, NT, 1>(P, u, len, best, best_j, z_new, row);
}

}  // namespace

}  // namespace kf
