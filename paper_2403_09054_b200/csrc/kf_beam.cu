// Beam search around the generation step.
//
// Selection: the `take` best of beams x vocabulary continuations by score_b + log softmax(logits_b), in one pass over the
// logits.  Within a beam the order is that of the logits, so a continuation among the best of all is among the
// `take` best of every chunk of its row.  beam_chunk_kernel: a CTA keeps a chunk of one row in registers (8 or 32
// values per thread), sums its exponentials against the chunk's maximum and lists its `take` best; beam_merge_kernel,
// one CTA per request and launched as its programmatic dependent, joins the sums in binary64 (two continuations of
// different beams may differ by less than binary32 tells) and takes the best of the lists.
//
// Finding the best few of thousands of registers: the largest values of the threads are sorted within their warp and the
// eight largest of each warp ranked against one another; the take-th of those 64 is a value that at least `take`
// elements reach, and few more than that do.  Those are collected in shared memory and ranked by comparison.  Rows with so
// many equal values that the collection does not fit (all tokens forbidden, constant logits) are worked off one
// element at a time.
//
// Order everywhere: larger value first, of equal values the lower beam, then the lower token.
//
// Reordering: a thread owns one offset of a state row, reads it from every beam that another one continues and then writes the beams
// that change, so it works in place without staging; bound by HBM.
#include <cuda_bf16.h>

#include "kf_ops.cuh"

namespace kf {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int TOP = 8;                    // maxima each warp contributes; WARPS * TOP >= BEAM_TAKE_MAX
constexpr int CAP = 512;                  // collected elements
static_assert(WARPS * TOP >= BEAM_TAKE_MAX, "the threshold needs `take` maxima");

// Larger value, then lower index: larger key.  Values are never NaN.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);          // -0 counts as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) { return (uint64_t)ordered(v) << 32 | (0xffffffffu - index); }

__device__ __forceinline__ float usable(float v) { return v < INFINITY ? v : -INFINITY; }   // NaN and +inf count as -inf

template <class T>
__device__ __forceinline__ float one_logit(const T* p);
template <> __device__ __forceinline__ float one_logit<__half>(const __half* p) { return __half2float(*p); }
template <> __device__ __forceinline__ float one_logit<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }
template <> __device__ __forceinline__ float one_logit<float>(const float* p) { return *p; }

template <class T>
__device__ __forceinline__ void widen(const uint4& v, float* x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      x[i] = __uint_as_float(w[i]);
    } else {
      float2 f;
      if constexpr (__is_same(T, __half)) f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      else f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}

// Descending sort of one value per lane (bitonic network).
__device__ __forceinline__ float sort_lanes(float v, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll
    for (int o = size >> 1; o > 0; o >>= 1) {
      const float other = __shfl_xor_sync(0xffffffffu, v, o);
      const bool keep_max = ((lane & o) == 0) == ((lane & size) == 0 || size == 32);
      v = keep_max ? fmaxf(v, other) : fminf(v, other);
    }
  }
  return v;
}

template <class KEY>
__device__ __forceinline__ KEY warp_best(KEY v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const KEY other = __shfl_xor_sync(0xffffffffu, v, o);
    v = other > v ? other : v;
  }
  return v;
}

// The take-th largest of the values that the warps left in `tops` (WARPS x TOP, each warp's in descending order): a
// threshold that at least `take` of the CTA's elements reach.  Every thread of the CTA calls it.
template <class V>
__device__ __forceinline__ V threshold_of(const V (&tops)[WARPS * TOP], V* where, int take) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (tid < WARPS * TOP) {
    const V mine = tops[tid];
    int rank = 0;
#pragma unroll
    for (int i = 0; i < WARPS * TOP; ++i) rank += (tops[i] > mine || (tops[i] == mine && i < tid)) ? 1 : 0;
    if (rank == take - 1) *where = mine;
  }
  __syncthreads();
  return *where;
}

// VPT 16-byte vectors per thread.
template <class T, int VPT>
__global__ void __launch_bounds__(THREADS) beam_chunk_kernel(const __grid_constant__ BeamParams P) {
  constexpr int EPV = 16 / (int)sizeof(T), E = EPV * VPT;
  __shared__ float tops[WARPS * TOP];
  __shared__ float sh_thr, sh_sum[WARPS];
  __shared__ uint64_t list[CAP];
  __shared__ int count;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int row = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (P.finished && P.finished[row]) return;              // goes on with the padding token; nothing is read
  const T* logits = static_cast<const T*>(P.logits) + (int64_t)row * P.row_stride;
  // vectors start on 16-byte boundaries; the first one may begin before the row, the last one end behind it
  const int lead = (int)((reinterpret_cast<uintptr_t>(logits) & 15u) / sizeof(T));
  const int first = chunk * (THREADS * E) - lead;         // element at which the chunk's first vector starts

  float x[E];
  float top = -INFINITY;
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    const int at = first + (v * THREADS + tid) * EPV;
    if (at >= 0 && at + EPV <= P.vocab) {
      widen<T>(__ldg(reinterpret_cast<const uint4*>(logits + at)), x + v * EPV);
    } else {
#pragma unroll
      for (int e = 0; e < EPV; ++e) x[v * EPV + e] = at + e >= 0 && at + e < P.vocab ? one_logit<T>(logits + at + e) : -INFINITY;
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    x[e] = usable(x[e]);
    top = fmaxf(top, x[e]);
  }
  const float sorted = sort_lanes(top, lane);
  if (lane < TOP) tops[warp * TOP + lane] = sorted;
  if (tid == 0) count = 0;
  const float thr = threshold_of(tops, &sh_thr, P.take);
  float best = tops[0];
#pragma unroll
  for (int i = 1; i < WARPS; ++i) best = fmaxf(best, tops[i * TOP]);

  // sum of exponentials against the chunk's maximum
  float sum = 0.f;
  if (best > -INFINITY) {
    const float off = best * LOG2E;
#pragma unroll
    for (int e = 0; e < E; ++e) sum += fast_exp2(fmaf(x[e], LOG2E, -off));
  }
  sum = warp_sum(sum);
  if (lane == 0) sh_sum[warp] = sum;

  // collect what reaches the threshold
  auto index_of = [&](int e) { return first + ((e / EPV) * THREADS + tid) * EPV + e % EPV; };
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int idx = index_of(e);
    if (x[e] >= thr && idx >= 0 && idx < P.vocab) {
      const int slot = atomicAdd(&count, 1);              // the order of arrival does not matter: keys are ranked below
      if (slot < CAP) list[slot] = key_of(x[e], (uint32_t)idx);
    }
  }
  __syncthreads();
  const int64_t entry = (int64_t)row * P.chunks + chunk;
  uint2* out = P.lists + entry * P.take;
  auto put = [&](int rank, uint64_t key) { out[rank] = make_uint2(__float_as_uint(unordered((uint32_t)(key >> 32))), 0xffffffffu - (uint32_t)key); };
  const int n = count;
  if (tid == 0) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) s += sh_sum[i];
    P.stats[entry] = make_float2(best, s);
  }
  if (n <= CAP) {
    for (int i = tid; i < n; i += THREADS) {
      const uint64_t mine = list[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += list[j] > mine ? 1 : 0;
      if (rank < P.take) put(rank, mine);
    }
    for (int i = n + tid; i < P.take; i += THREADS) out[i] = make_uint2(0u, 0xffffffffu);   // fewer elements than asked for
    return;
  }
  // many equal values: one element per round, the best key below the last one
  __shared__ uint64_t sh_key[WARPS];
  uint64_t last = ~0ull;
  for (int r = 0; r < P.take; ++r) {
    uint64_t mine = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int idx = index_of(e);
      if (idx >= 0 && idx < P.vocab) {
        const uint64_t key = key_of(x[e], (uint32_t)idx);
        if (key < last && key > mine) mine = key;
      }
    }
    mine = warp_best(mine);
    if (lane == 0) sh_key[warp] = mine;
    __syncthreads();
    last = sh_key[0];
#pragma unroll
    for (int i = 1; i < WARPS; ++i) last = sh_key[i] > last ? sh_key[i] : last;
    if (tid == 0) put(r, last);          // n > CAP >= take: there is one in every round
    __syncthreads();
  }
}

// A continuation as it is ranked: value, then the place beam * vocab + token.
struct Candidate {
  double value;
  int64_t place;
};
__device__ __forceinline__ bool better(const Candidate& a, const Candidate& b) {
  return a.value > b.value || (a.value == b.value && a.place < b.place);
}

__global__ void __launch_bounds__(THREADS) beam_merge_kernel(const __grid_constant__ BeamParams P) {
  constexpr int MCAP = 1024;
  __shared__ double base[BEAM_MAX];          // score - log of the sum of exponentials; -inf: no continuation counts
  __shared__ double tops[WARPS * TOP];
  __shared__ double sh_thr;
  __shared__ Candidate cand[MCAP];
  __shared__ int count;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (tid == 0) count = 0;

  // ---- the beams' normalisers: one warp per beam
  for (int w = warp; w < P.beams; w += WARPS) {
    const int64_t row = (int64_t)b * P.beams + w;
    double s = (double)P.scores[row], lse = 0.0;
    bool live = isfinite(s);
    if (!(P.finished && P.finished[row])) {
      float m = -INFINITY;
      for (int c = lane; c < P.chunks; c += 32) m = fmaxf(m, __ldcg(&P.stats[row * P.chunks + c]).x);
      m = warp_max(m);
      double sum = 0.0;
      if (m > -INFINITY)
        for (int c = lane; c < P.chunks; c += 32) {
          const float2 st = __ldcg(&P.stats[row * P.chunks + c]);
          if (st.x > -INFINITY) sum += (double)st.y * exp((double)st.x - (double)m);
        }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      live = live && m > -INFINITY;
      lse = live ? (double)m + log(sum) : 0.0;
    }
    if (lane == 0) base[w] = live ? s - lse : -INFINITY;
  }
  __syncthreads();

  // ---- entry i of list l.  A beam without a live continuation offers its first tokens, all at -inf; a finished one the
  //      padding token at its score, then the other tokens at -inf.  Lists end where entry() says so.
  const int lists = P.beams * P.chunks;
  auto entry = [&](int l, int i, Candidate& c) -> bool {
    const int w = l / P.chunks, ch = l % P.chunks;
    const int64_t row = (int64_t)b * P.beams + w;
    const bool dead = base[w] == -INFINITY, done = P.finished && P.finished[row];
    int token;
    double value;
    if (dead || done) {
      if (ch > 0 || i >= P.vocab) return false;
      token = dead ? i : (i == 0 ? P.pad : (i - 1 < P.pad ? i - 1 : i));
      value = dead || i > 0 ? -INFINITY : base[w];
    } else {
      const uint2 e = __ldcg(&P.lists[(row * P.chunks + ch) * P.take + i]);
      if (e.y == 0xffffffffu) return false;
      token = (int)e.y;
      value = base[w] + (double)__uint_as_float(e.x);
    }
    c.value = value;
    c.place = (int64_t)w * P.vocab + token;
    return true;
  };

  // ---- a value that at least `take` continuations reach, found as in the chunks: every thread takes its share of the
  //      entries, neighbouring entries of a list in different threads
  const int entries = lists * P.take;
  double left = -INFINITY;
  for (int i = tid; i < entries; i += THREADS) {
    Candidate c;
    if (entry(i / P.take, i % P.take, c) && c.value > left) left = c.value;
  }
  for (int i = 0; i < TOP; ++i) {
    const double m = warp_best(left);
    if (lane == 0) tops[warp * TOP + i] = m;
    const unsigned who = __ballot_sync(0xffffffffu, left == m);
    if (lane == __ffs(who) - 1) left = -INFINITY;
  }
  const double thr = threshold_of(tops, &sh_thr, P.take);

  for (int i = tid; i < entries; i += THREADS) {
    Candidate c;
    if (entry(i / P.take, i % P.take, c) && c.value >= thr) {
      const int slot = atomicAdd(&count, 1);
      if (slot < MCAP) cand[slot] = c;
    }
  }
  __syncthreads();
  const int n = count;
  auto put = [&](int rank, const Candidate& c) {
    const int64_t at = (int64_t)b * P.take + rank;
    P.out_scores[at] = (float)c.value;
    P.out_parent[at] = (int)(c.place / P.vocab);
    P.out_token[at] = (int)(c.place % P.vocab);
  };
  if (n <= MCAP) {
    for (int i = tid; i < n; i += THREADS) {
      const Candidate mine = cand[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += better(cand[j], mine) ? 1 : 0;
      if (rank < P.take) put(rank, mine);
    }
    return;
  }
  // many equal values: one continuation per round, the best one behind the last
  __shared__ Candidate sh_best[WARPS];
  Candidate last;
  last.value = INFINITY;
  last.place = -1;
  for (int r = 0; r < P.take; ++r) {
    Candidate mine;
    mine.value = -INFINITY;
    mine.place = (int64_t)1 << 62;
    for (int i = tid; i < entries; i += THREADS) {
      Candidate c;
      if (entry(i / P.take, i % P.take, c) && better(last, c) && better(c, mine)) mine = c;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      Candidate other;
      other.value = __shfl_xor_sync(0xffffffffu, mine.value, o);
      other.place = __shfl_xor_sync(0xffffffffu, mine.place, o);
      if (better(other, mine)) mine = other;
    }
    if (lane == 0) sh_best[warp] = mine;
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
cudaError_t launch_type(const BeamParams& P, bool wide, cudaStream_t stream) {
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
  // 32 values per thread where that still gives every SM work, else 8; 7 more values than the row has, because its
  // first vector may begin before it
  const int64_t span = (int64_t)vocab + 7;
  const int64_t big = (span + THREADS * 32 - 1) / (THREADS * 32);
  *wide = rows * big >= 148;
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
