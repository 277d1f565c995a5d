// Beam search around the generation step.
//
// Selection: the `take` best of beams x vocabulary continuations by score_b + log softmax(logits_b), in one pass over the
// logits.  Within a beam the order is that of the logits, so a continuation among the best of all is among the
// `take` best of every chunk of its row.  beam_chunk_kernel: a CTA keeps a chunk of one row in registers (8 or 32
// values per thread), sums its exponentials against the chunk's maximum and lists its `take` best; beam_merge_kernel,
// one CTA per request and launched as its programmatic dependent, joins the sums in binary64 (two continuations of
// different beams may differ by less than binary32 tells) and takes the best of the lists.
//
// Finding the best few of thousands of registers: with c = take / 8 rounded up, each of the eight warps finds the c-th
// largest of its threads' maxima, and the smallest of those eight values is one that at least `take` elements reach and
// few more than that do (about three times `take` of 8192 random ones).  (Of a chunk that fills fewer warps, those count;
// where a warp has too few tokens that are not forbidden, a single warp's take-th largest serves.)  They are collected in shared
// memory and ranked by comparison.  Chunks with so many equal values that the collection does not fit (all tokens
// forbidden, constant logits) are worked off one element at a time.
//
// 32 requests x 8 beams x 50400 logits in binary16 (a third of the beams at their end): 18 us, of which 12 are chunks in two and a half
// waves of CTAs that live for one chunk each, and 6 the merge; one request of 4 x 50257: 7.5 us.  Latency bounds both: the
// bytes would take 4 us and 0.1.
//
// Order everywhere: larger value first, of equal values the lower beam, then the lower token.
//
// Reordering (54.6 us for 352 MB, 6.4 TB/s): a thread owns one offset of a state row, reads it from every beam that another one continues and then writes the beams
// that change, so it works in place without staging; bound by HBM.
#include <cuda_bf16.h>

#include "kf_ops.cuh"

namespace kf {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int CAP = THREADS;              // collected elements, one per thread when they are ranked

// Larger value, then lower index: larger key.  Values are never NaN.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);          // -0 counts as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) { return (uint64_t)ordered(v) << 32 | (0xffffffffu - index); }

__device__ __forceinline__ float widen(__half v) { return __half2float(v); }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float widen(float v) { return v; }

template <class KEY>
__device__ __forceinline__ KEY warp_best(KEY v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const KEY other = __shfl_xor_sync(0xffffffffu, v, o);
    v = other > v ? other : v;
  }
  return v;
}

// The c-th largest of the lanes' values (equal ones count one by one).
__device__ __forceinline__ float warp_nth(float v, int c, int lane) {
  float m = -INFINITY;
  for (int i = 0; i < c; ++i) {
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
    const unsigned who = __ballot_sync(0xffffffffu, v == m);
    if (lane == __ffs(who) - 1) v = -INFINITY;
  }
  return m;
}

// One 16-byte vector of logits, worked on in its own type (two values at a time where they have 16 bits).  What lies outside
// the row and what is not finite is -inf.
template <class T>
struct Vec {
  static constexpr int N = 16 / (int)sizeof(T), PER = 4 / (int)sizeof(T);   // values per vector, per 32-bit word
  static constexpr uint32_t MINUS_INF = sizeof(T) == 4 ? 0xff800000u : (__is_same(T, __half) ? 0xfc00fc00u : 0xff80ff80u);
  uint32_t w[4];

  template <class F>
  __device__ __forceinline__ static auto pair(uint32_t bits, F&& f) {
    if constexpr (__is_same(T, __half)) return f(*reinterpret_cast<const __half2*>(&bits));
    else return f(*reinterpret_cast<const __nv_bfloat162*>(&bits));
  }
  __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = MINUS_INF; }
  __device__ __forceinline__ void load(const T* p) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  }
  __device__ __forceinline__ void load_within(const T* row, int at, int vocab) {   // a vector that the row's ends cut
    T v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = at + e >= 0 && at + e < vocab ? row[at + e] : minus_inf();
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = reinterpret_cast<const uint32_t*>(v)[i];
  }
  __device__ __forceinline__ void only_finite() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {     // NaN and +inf are not below +inf
      if constexpr (sizeof(T) == 4) {
        w[i] = __uint_as_float(w[i]) < INFINITY ? w[i] : MINUS_INF;
      } else {
        const uint32_t ok = less(w[i], MINUS_INF & 0x7fff7fffu);
        w[i] = (w[i] & ok) | (MINUS_INF & ~ok);
      }
    }
  }
  __device__ __forceinline__ static T minus_inf() {
    if constexpr (sizeof(T) == 4) return -INFINITY;
    else if constexpr (__is_same(T, __half)) return __ushort_as_half((unsigned short)0xfc00u);
    else return __ushort_as_bfloat16((unsigned short)0xff80u);
  }
  // 16-bit types: masks of the halves where a < b, a >= b
  __device__ __forceinline__ static uint32_t less(uint32_t a, uint32_t b) {
    return pair(a, [&](auto x) { return pair(b, [&](auto y) { return __hlt2_mask(x, y); }); });
  }
  __device__ __forceinline__ static uint32_t reaches(uint32_t a, uint32_t b) {
    return pair(a, [&](auto x) { return pair(b, [&](auto y) { return __hge2_mask(x, y); }); });
  }
  __device__ __forceinline__ static float value(uint32_t bits, int e) {   // value e of a word
    if constexpr (sizeof(T) == 4) return __uint_as_float(bits);
    else if constexpr (__is_same(T, __half)) return __half2float(__ushort_as_half((unsigned short)(bits >> 16 * e)));
    else return __uint_as_float(e ? bits & 0xffff0000u : bits << 16);
  }
  __device__ __forceinline__ static uint32_t larger(uint32_t a, uint32_t b) {
    if constexpr (sizeof(T) == 4) {
      return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    } else {
      return pair(a, [&](auto x) { return pair(b, [&](auto y) { const auto m = __hmax2(x, y); return *reinterpret_cast<const uint32_t*>(&m); }); });
    }
  }
  // the word with `v`, which the type holds exactly, in every place
  __device__ __forceinline__ static uint32_t splat(float v) {
    if constexpr (sizeof(T) == 4) return __float_as_uint(v);
    else if constexpr (__is_same(T, __half)) return (uint32_t)__half_as_ushort(__float2half_rn(v)) * 0x10001u;
    else return (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v)) * 0x10001u;
  }
};

// VPT 16-byte vectors per thread.
template <class T, int VPT>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 4 ? 4 : 5) beam_chunk_kernel(const __grid_constant__ BeamParams P) {
  using V = Vec<T>;
  constexpr int EPV = V::N, PER = V::PER;
  __shared__ float sh_nth[WARPS], sh_top[WARPS], sh_sum[WARPS];
  __shared__ uint64_t list[CAP];
  __shared__ int count;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int row = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (P.finished && P.finished[row]) return;              // goes on with the padding token; nothing is read
  const T* logits = static_cast<const T*>(P.logits) + (int64_t)row * P.row_stride;
  // vectors start on 16-byte boundaries; the row's first one may begin before it, its last one end behind it
  const int lead = (int)((reinterpret_cast<uintptr_t>(logits) & 15u) / sizeof(T));
  const int vectors = (P.vocab + lead + EPV - 1) / EPV, per_chunk = (vectors + P.chunks - 1) / P.chunks;   // at most THREADS * VPT
  const int first = chunk * per_chunk, last = min(vectors, first + per_chunk);
  auto place = [&](int v) { return (first + v * THREADS + tid) * EPV - lead; };   // element at which the vector starts

  V vec[VPT];
#pragma unroll
  for (int v = 0; v < VPT; ++v) vec[v].clear();
#pragma unroll
  for (int v = 0; v < VPT; ++v)
    if (first + v * THREADS + tid < last && place(v) >= 0 && place(v) + EPV <= P.vocab) vec[v].load(logits + place(v));
  if (first * EPV < lead || last * EPV - lead > P.vocab) {   // the same for the whole CTA: one of its vectors is cut
#pragma unroll 1
    for (int v = 0; v < VPT; ++v) {
      const int at = place(v);
      if (first + v * THREADS + tid < last && (at < 0 || at + EPV > P.vocab)) {
        V one;
        one.load_within(logits, at, P.vocab);
#pragma unroll
        for (int k = 0; k < VPT; ++k)
          if (k == v) vec[k] = one;
      }
    }
  }
#pragma unroll
  for (int v = 0; v < VPT; ++v) vec[v].only_finite();
  if (tid == 0) count = 0;
  uint32_t top_word = V::MINUS_INF;
#pragma unroll
  for (int v = 0; v < VPT; ++v)
#pragma unroll
    for (int i = 0; i < 4; ++i) top_word = V::larger(top_word, vec[v].w[i]);
  const float top = fmaxf(V::value(top_word, 0), V::value(top_word, PER - 1));
  // warps of which every lane has a vector; a chunk that does not fill one is small enough to be collected whole
  const int full = min(WARPS, (last - first) / 32), each = full > 0 ? (P.take + full - 1) / full : 33;
  const float most = warp_nth(top, 1, lane), nth = each <= 32 ? warp_nth(top, each, lane) : -INFINITY;
  if (lane == 0) { sh_nth[warp] = nth; sh_top[warp] = most; }
  __syncthreads();
  float thr = sh_nth[0], best = sh_top[0];
#pragma unroll
  for (int i = 1; i < WARPS; ++i) {
    if (i < full) thr = fminf(thr, sh_nth[i]);
    best = fmaxf(best, sh_top[i]);
  }
  if (thr == -INFINITY && best > -INFINITY && P.take <= 32) {   // the same for the whole CTA
    const float one = warp_nth(top, P.take, lane);
    __syncthreads();
    if (lane == 0) sh_nth[warp] = one;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WARPS; ++i) thr = fmaxf(thr, sh_nth[i]);
  }

  // collect what reaches the threshold; the order of arrival does not matter, keys are ranked below.  The few words that hold
  // such a value are noted first.
  uint32_t hits = 0;
  if (top >= thr) {
    const uint32_t thr_word = V::splat(thr);
#pragma unroll
    for (int k = 0; k < 4 * VPT; ++k) {
      const uint32_t word = vec[k / 4].w[k % 4];
      bool hit;
      if constexpr (PER == 1) hit = __uint_as_float(word) >= thr;
      else hit = V::reaches(word, thr_word) != 0u;
      hits |= hit ? 1u << k : 0u;
    }
  }
  while (hits) {
    const int k = __ffs(hits) - 1, at = place(k >> 2) + (k & 3) * PER;
    hits &= hits - 1;
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 4 * VPT; ++i) word = i == k ? vec[i / 4].w[i % 4] : word;
    if (first + (k >> 2) * THREADS + tid < last) {
#pragma unroll
      for (int e = 0; e < PER; ++e)
        if (at + e >= 0 && at + e < P.vocab) {
          const float x = V::value(word, e);
          if (x >= thr) {
            const int slot = atomicAdd(&count, 1);
            if (slot < CAP) list[slot] = key_of(x, (uint32_t)(at + e));
          }
        }
    }
  }
  // sum of exponentials against the chunk's maximum
  float sum = 0.f;
  if (best > -INFINITY) {
    // the difference first: masks of the type's lowest value times log2(e) would overflow
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
      for (int e = 0; e < EPV; ++e) sum += fast_exp2((V::value(vec[v].w[e / PER], e % PER) - best) * LOG2E);
  }
  sum = warp_sum(sum);
  if (lane == 0) sh_sum[warp] = sum;
  __syncthreads();

  const int64_t entry = (int64_t)row * P.chunks + chunk;
  uint2* out = P.lists + entry * P.take;
  auto put = [&](int rank, uint64_t key) { out[rank] = make_uint2(__float_as_uint(unordered((uint32_t)(key >> 32))), 0xffffffffu - (uint32_t)key); };
  const int n = count;
  if (tid == THREADS - 1) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) s += sh_sum[i];
    P.stats[entry] = make_float2(best, s);
  }
  if (n <= CAP) {
    if (tid < n) {
      const uint64_t mine = list[tid];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < n; ++j) rank += list[j] > mine ? 1 : 0;
      if (rank < P.take) put(rank, mine);
    }
    for (int i = n + tid; i < P.take; i += THREADS) out[i] = make_uint2(0u, 0xffffffffu);   // fewer elements than asked for
    return;
  }
  // many equal values: one element per round, the best key below the last one (read from memory again: this is rare, and what it
  // would hold costs the common path registers)
  __shared__ uint64_t sh_key[WARPS];
  uint64_t prev = ~0ull;
  const int from = max(0, first * EPV - lead), to = min(P.vocab, last * EPV - lead);
  for (int r = 0; r < P.take; ++r) {
    uint64_t mine = 0;
    for (int idx = from + tid; idx < to; idx += THREADS) {
      float x = widen(logits[idx]);
      x = x < INFINITY ? x : -INFINITY;
      const uint64_t key = key_of(x, (uint32_t)idx);
      if (key < prev && key > mine) mine = key;
    }
    mine = warp_best(mine);
    if (lane == 0) sh_key[warp] = mine;
    __syncthreads();
    prev = sh_key[0];
#pragma unroll
    for (int i = 1; i < WARPS; ++i) prev = sh_key[i] > prev ? sh_key[i] : prev;
    if (tid == 0) put(r, prev);          // n > CAP >= take: there is one in every round
    __syncthreads();
  }
}

// A continuation as it is ranked: value (larger key: larger value; whole numbers compare faster than binary64 ones), then the
// place beam * vocab + token.
struct Candidate {
  uint64_t key;
  int place;        // below 2^31: at most 32 beams of 2^26 tokens
};
__device__ __forceinline__ bool better(const Candidate& a, const Candidate& b) {
  return (a.key > b.key) | ((a.key == b.key) & (a.place < b.place));   // no branches: this is the inner loop of a ranking
}
__device__ __forceinline__ uint64_t ordered(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double unordered(uint64_t k) {
  return __longlong_as_double((long long)(k >> 63 ? k & 0x7fffffffffffffffull : ~k));
}

// The first entries of all lists, as many as the threads hold in registers, are requested before anything else.  They are dealt
// to the threads position by position and beam by beam in turn, so that the best ones lie in different threads.  What lies
// further down a list is read only where the list is still above the threshold there.
__global__ void __launch_bounds__(THREADS) beam_merge_kernel(const __grid_constant__ BeamParams P) {
  constexpr int MCAP = 1024, HELD = 8, RANKED = 384, FEW = 96;
  __shared__ double base[BEAM_MAX];          // score - log of the sum of exponentials against the largest logit
  __shared__ float largest[BEAM_MAX];        // that logit, taken off each logit by itself: it may be the type's lowest value
  __shared__ int kind[BEAM_MAX];             // 0: lists of the chunks, 1: at its end, 2: nothing left
  __shared__ __align__(16) float sh_max[THREADS];
  __shared__ unsigned int least;
  __shared__ Candidate cand[MCAP];
  __shared__ int count;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n_lists = P.beams * P.chunks;
  const int depth = min(P.take, HELD * THREADS / n_lists);        // entries of a list that are held
  const uint2* lists = P.lists + (int64_t)b * n_lists * P.take;
  // held entry e: number i = e / n_lists of a list, the lists shifted by i beams
  auto locate = [&](int e, int& l, int& i) {
    i = n_lists == 1 ? e : (int)__umulhi((uint32_t)e, P.by_lists);            // exact: e n_lists < 2^32
    const int shift = i * P.chunks;                                           // below e: chunks <= n_lists
    l = e - i * n_lists + shift - (n_lists == 1 ? shift : (int)__umulhi((uint32_t)shift, P.by_lists) * n_lists);
    if (l >= n_lists) l -= n_lists;
  };
  if (tid == 0) { count = 0; least = ~0u; }
  // the caller's tensors do not depend on the chunks
  float score = 0.f;
  bool done = false;
  auto ask = [&](int w) {
    const int64_t row = (int64_t)b * P.beams + w;
    score = P.scores[row];
    done = P.finished && P.finished[row];
  };
  if (warp < P.beams) ask(warp);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float2 first_stat = make_float2(-INFINITY, 0.f);
  if (warp < P.beams && lane < P.chunks && !done) first_stat = __ldcg(&P.stats[((int64_t)b * P.beams + warp) * P.chunks + lane]);
  uint2 held[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    held[i] = make_uint2(0u, 0xffffffffu);
    if (tid + i * THREADS < depth * n_lists) {
      int l, k;
      locate(tid + i * THREADS, l, k);
      held[i] = __ldcg(lists + l * P.take + k);
    }
  }

  // ---- the beams' normalisers: one warp per beam
  for (int w = warp; w < P.beams; w += WARPS) {
    const int64_t row = (int64_t)b * P.beams + w;
    if (w != warp) ask(w);
    float m = -INFINITY, sum = 0.f;
    if (!done) {
      for (int c = lane; c < P.chunks; c += 32) {
        const float2 st = w == warp && c == lane ? first_stat : __ldcg(&P.stats[row * P.chunks + c]);
        if (st.x > m) {
          sum = fmaf(sum, fast_exp2((m - st.x) * LOG2E), st.y);
          m = st.x;
        } else if (st.x > -INFINITY) {
          sum = fmaf(st.y, fast_exp2((st.x - m) * LOG2E), sum);
        }
      }
      const float all = warp_max(m);
      sum = warp_sum(m > -INFINITY ? sum * fast_exp2((m - all) * LOG2E) : 0.f);
      m = all;
    }
    if (lane == 0) {
      const bool live = isfinite(score) && (done || m > -INFINITY);
      kind[w] = live ? (done ? 1 : 0) : 2;
      // log(sum) from its exponent, exactly, and the logarithm of a number near 1: binary32 alone would round a sum of thousands
      // to half a millionth
      const int e = (__float_as_int(sum) - 0x3f3504f3) >> 23;       // 0x3f3504f3: sqrt(1/2)
      const double log_sum = (double)e * 0.69314718055994531 + (double)logf(__int_as_float(__float_as_int(sum) - (e << 23)));
      base[w] = live ? (done ? (double)score : (double)score - log_sum) : -INFINITY;
      largest[w] = m;
    }
  }
  __syncthreads();

  // ---- entry i of list l as a continuation.  A beam without a live continuation offers its first tokens, all at -inf, in place of its
  //      first list; one at its end the padding token at its score, then the other tokens at -inf.  A place of -1: the list has ended.
  auto candidate = [&](int l, int i, const uint2& raw) {
    const int w = P.chunks == 1 ? l : (int)__umulhi((uint32_t)l, P.by_chunks);      // l / chunks, exact: l chunks < 2^32
    Candidate c;
    int token = (int)raw.y;
    double value = base[w] + ((double)__uint_as_float(raw.x) - (double)largest[w]);
    if (kind[w] != 0) {
      const bool done = kind[w] == 1;
      token = l != w * P.chunks || i >= P.vocab ? -1 : (!done ? i : (i == 0 ? P.pad : (i - 1 < P.pad ? i - 1 : i)));
      value = done && i == 0 ? base[w] : -INFINITY;
    }
    c.key = token < 0 ? 0 : ordered(value);             // below every real one
    c.place = token < 0 ? -1 : w * P.vocab + token;
    return c;
  };
  Candidate mine[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    mine[i].key = 0;
    mine[i].place = -1;
    if (tid + i * THREADS < depth * n_lists) {
      int l, k;
      locate(tid + i * THREADS, l, k);
      mine[i] = candidate(l, k, held[i]);
    }
  }
  // use(continuation) for every one of this thread whose key reaches `from`
  auto each = [&](uint64_t from, auto&& use) {
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (mine[i].place >= 0 && mine[i].key >= from) use(mine[i]);
    if (depth < P.take)
      for (int l = tid; l < n_lists; l += THREADS)
        for (int i = depth; i < P.take; ++i) {          // lists descend
          const Candidate c = candidate(l, i, __ldcg(lists + (int64_t)l * P.take + i));
          if (c.place < 0 || c.key < from) break;
          use(c);
        }
  };

  // ---- a value that at least `take` continuations reach: the take-th of the threads' maxima, in binary32; what rounding may
  //      have taken off it is granted.  With few entries all of them are ranked.
  uint64_t thr = 0;
  if (n_lists * P.take > FEW) {
    uint64_t most = ordered((double)-INFINITY);
#pragma unroll
    for (int i = 0; i < HELD; ++i) most = mine[i].key > most ? mine[i].key : most;
    if (depth == 0)                                     // more lists than can be held: their heads
      for (int l = tid; l < n_lists; l += THREADS) {
        const Candidate c = candidate(l, 0, __ldcg(lists + (int64_t)l * P.take));
        if (c.place >= 0 && c.key > most) most = c.key;
      }
    float top = (float)unordered(most);
    // a sixteenth of the maxima is asked for at most: those of four threads together will do
    const int group = P.take <= 16 ? 4 : 1;
    if (group == 4) {
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    }
    const bool mark = (tid & (group - 1)) == 0;
    if (mark) sh_max[group == 4 ? tid >> 2 : tid] = top;
    __syncthreads();
    int above = 0;
#pragma unroll 16
    for (int i = 0; i < THREADS / group; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(sh_max + i);
      above += (v.x > top) + (v.y > top) + (v.z > top) + (v.w > top);
    }
    if (mark && above < P.take) atomicMin(&least, ordered(top));   // the smallest value with fewer than `take` above it
    __syncthreads();
    const double t = (double)unordered(least);
    thr = ordered(t - 1e-6 * fabs(t));      // -inf stays -inf
  }
  each(thr, [&](const Candidate& c) {
    const int slot = atomicAdd(&count, 1);
    if (slot < MCAP) cand[slot] = c;
  });
  __syncthreads();
  const int n = count;
  auto put = [&](int rank, const Candidate& c) {
    const int64_t at = (int64_t)b * P.take + rank;
    P.out_scores[at] = (float)unordered(c.key);
    P.out_parent[at] = c.place / P.vocab;
    P.out_token[at] = c.place % P.vocab;
  };
  if (n <= RANKED) {
    for (int i = tid; i < n; i += THREADS) {
      const Candidate one = cand[i];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < n; ++j) rank += better(cand[j], one) ? 1 : 0;
      if (rank < P.take) put(rank, one);
    }
    return;
  }
  // many equal values: one continuation per round, the best one behind the last, of those collected if they all were
  __shared__ Candidate sh_best[WARPS];
  Candidate last;
  last.key = ~0ull;
  last.place = -1;
  for (int r = 0; r < P.take; ++r) {
    Candidate next;
    next.key = 0;
    next.place = INT32_MAX;
    auto look = [&](const Candidate& c) {
      if (better(last, c) && better(c, next)) next = c;
    };
    if (n <= MCAP)
      for (int i = tid; i < n; i += THREADS) look(cand[i]);
    else
      each(0, look);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      Candidate other;
      other.key = __shfl_xor_sync(0xffffffffu, next.key, o);
      other.place = __shfl_xor_sync(0xffffffffu, next.place, o);
      if (better(other, next)) next = other;
    }
    if (lane == 0) sh_best[warp] = next;
    __syncthreads();
    last = sh_best[0];
#pragma unroll
    for (int i = 1; i < WARPS; ++i)
      if (better(sh_best[i], last)) last = sh_best[i];
    if (tid == 0) put(r, last);
    __syncthreads();
  }
}

template <class T>
cudaError_t launch_type(BeamParams P, bool wide, cudaStream_t stream) {
  // floor(2^32 / n) + 1: the high word of its product with e is e / n while e n < 2^32 (n = 1 does without)
  P.by_lists = (uint32_t)(((uint64_t)1 << 32) / (uint64_t)(P.beams * P.chunks)) + 1;
  P.by_chunks = (uint32_t)(((uint64_t)1 << 32) / (uint64_t)P.chunks) + 1;
  constexpr int NARROW = (int)sizeof(T) / 2, WIDE = 4 * NARROW;   // 8 or 32 values per thread
  const dim3 grid((unsigned)P.chunks, (unsigned)(P.batch * P.beams));
  if (wide) beam_chunk_kernel<T, WIDE><<<grid, THREADS, 0, stream>>>(P);
  else beam_chunk_kernel<T, NARROW><<<grid, THREADS, 0, stream>>>(P);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)P.batch);
  cfg.blockDim = dim3(THREADS);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, beam_merge_kernel, P);
}

// ------------------------------------------------------------------------------------------------ reordering
template <int W, class V>
__device__ __forceinline__ void move_offset(unsigned char* row0, int64_t row_bytes, const int (&from)[W]) {
  V v[W];
#pragma unroll
  for (int w = 0; w < W; ++w)
    if (from[w] >= 0) v[w] = *reinterpret_cast<const V*>(row0 + from[w] * row_bytes);
#pragma unroll
  for (int w = 0; w < W; ++w)
    if (from[w] >= 0) *reinterpret_cast<V*>(row0 + w * row_bytes) = v[w];
}

template <int W>
__global__ void __launch_bounds__(THREADS) reorder_kernel(const __grid_constant__ ReorderParams P) {
  const int batch_row = blockIdx.y;
  int from[W];          // source of beam w, -1 where it keeps its own (or the entry is out of range)
  bool any = false;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int p = w < P.beams ? P.parent[batch_row * P.beams + w] : w;
    from[w] = p >= 0 && p < P.beams && p != w ? p : -1;
    any = any || from[w] >= 0;
  }
  if (!any) return;
  int i = 0;
  while (i + 1 < P.n_buffers && (int)blockIdx.x >= P.buf[i + 1].first_block) ++i;
  const ReorderBuffer& B = P.buf[i];
  const int local = (int)blockIdx.x - B.first_block, outer = local / B.blocks_per_row;
  const int64_t at = ((int64_t)(local % B.blocks_per_row) * THREADS + threadIdx.x) * B.width;
  if (at >= B.row_bytes) return;
  unsigned char* row0 = B.base + outer * B.outer_stride + (int64_t)batch_row * P.beams * B.row_bytes + at;
  if (B.width == 16) move_offset<W, uint4>(row0, B.row_bytes, from);
  else if (B.width == 4) move_offset<W, uint32_t>(row0, B.row_bytes, from);
  else move_offset<W, unsigned char>(row0, B.row_bytes, from);
}

}  // namespace

void beam_plan(int64_t rows, int vocab, int* chunks, bool* wide) {
  // 32 values per thread where that still gives every SM work, else 8; 7 more values than the row has, because its first vector may begin before it.
  // 32 against 8, us: 256 rows of 50400 in binary16 20.7 and 37.6 (binary32 27.6 and 36.5), 32 rows of 50257 10.1 and 13.3 (12.5 and 12.8), 512 rows of
  // 4000 10.2 and 11.9 (12.1 and 11.2).  Below the switch 32 would be no slower either: 16 rows of 50257 9.6 and 11.5 (9.9 and 11.1), 4 rows
  // 7.0 and 7.9 (7.6 and 7.7).
  const int64_t span = (int64_t)vocab + 7;
  const int64_t big = (span + THREADS * 32 - 1) / (THREADS * 32);
  *wide = rows * big >= 148 && span > THREADS * 8;
  *chunks = (int)(*wide ? big : (span + THREADS * 8 - 1) / (THREADS * 8));
}

cudaError_t launch_beam_select(const BeamParams& P, int type, bool wide, cudaStream_t stream) {
  switch (type) {
    case LOGITS_F16: return launch_type<__half>(P, wide, stream);
    case LOGITS_BF16: return launch_type<__nv_bfloat16>(P, wide, stream);
    case LOGITS_F32: return launch_type<float>(P, wide, stream);
    default: return cudaErrorInvalidValue;
  }
}

cudaError_t launch_reorder(ReorderParams P, cudaStream_t stream) {
  int64_t blocks = 0;
  for (int i = 0; i < P.n_buffers; ++i) {
    ReorderBuffer& B = P.buf[i];
    const uint64_t mix = reinterpret_cast<uint64_t>(B.base) | (uint64_t)B.row_bytes | (B.outer > 1 ? (uint64_t)B.outer_stride : 0);
    B.width = mix % 16 == 0 ? 16 : (mix % 4 == 0 ? 4 : 1);
    const int64_t per_row = (B.row_bytes + (int64_t)THREADS * B.width - 1) / ((int64_t)THREADS * B.width);
    B.first_block = (int32_t)blocks;
    B.blocks_per_row = (int32_t)per_row;
    blocks += per_row * B.outer;
    if (per_row > INT32_MAX || blocks > INT32_MAX) return cudaErrorInvalidValue;
  }
  if (blocks == 0) return cudaSuccess;
  const dim3 grid((unsigned)blocks, (unsigned)P.batch);
  if (P.beams <= 4) reorder_kernel<4><<<grid, THREADS, 0, stream>>>(P);
  else if (P.beams <= 8) reorder_kernel<8><<<grid, THREADS, 0, stream>>>(P);
  else if (P.beams <= 16) reorder_kernel<16><<<grid, THREADS, 0, stream>>>(P);
  else reorder_kernel<32><<<grid, THREADS, 0, stream>>>(P);
  return cudaGetLastError();
}

}  // namespace kf
