// Launch interface and shared device code of the operators on ragged batches: attention over prompts of different lengths
// (kf_ragged.cu), 8-bit pages (kf_pages.cu: write, read, compact, update; kf_pages_attend.cu: one token per sequence).
//
// A page holds `page` consecutive tokens of one sequence: int8 codes [Hkv][2][page][d] (K tile, then V tile, of each head, so that a head's
// tile is contiguous) and a binary32 scale per head and side.  Scales that this library makes are powers of two: then codes are
// defined without a rounding of the scale, and bringing codes to a larger scale is one rounding each, at most half a step of a scale that
// has at least doubled, so that the steps a row may be off by form 1/2 + 1/4 + ... < 1 of the final one, however often its page grows.
#pragma once

#include <cuda_bf16.h>

#include "kf_common.cuh"

namespace kf {

// ---- prompts of different lengths
struct RaggedArgs {
  const void *q, *k, *v;
  void* out;
  const int32_t* begin;        // [S + 1]
  const float* slopes;         // [H] or null
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, out_token, out_head;   // strides in elements
  int32_t tokens, sequences, H, Hkv, head_dim;
  int32_t fail_item, leave_item;   // the self-test's (-1: none): the items of a CTA from which on waits for logits fail, or at which the wait for it fails
  bool bf16;
  float scale;
};
cudaError_t launch_ragged(const RaggedArgs& a, cudaStream_t stream);

// ---- pages
struct PageCache {
  signed char* codes;          // [pages][Hkv][2][page][d]
  float* scale;                // [pages][Hkv][2]
  int32_t pages, page, Hkv, d, S, W;
};
struct PageRows {
  void *k, *v;
  int64_t k_token, k_head, v_token, v_head;   // strides in elements
  int32_t tokens;
  bool bf16;
};
cudaError_t launch_pages_write(const PageCache& c, const PageRows& r, const int32_t* begin, const int32_t* length, const int32_t* table, cudaStream_t stream);
cudaError_t launch_pages_read(const PageCache& c, const PageRows& r, const int32_t* begin, const int32_t* first, const int32_t* table, cudaStream_t stream);
cudaError_t launch_pages_compact(const PageCache& c, int keep_width, int new_width, const int32_t* table, const int32_t* length, const int32_t* keep,
                                 const int32_t* n_keep, const int32_t* new_table, cudaStream_t stream);

constexpr int UPDATE_MAX_SEQUENCES = 8192;
struct PagesUpdate {
  PageCache c;
  int32_t layers, grow_all;
  int32_t *table, *length, *refs, *missing;
  const int32_t *parent, *grow;   // or null
  int32_t log_page;               // filled in by the launch
  int32_t *stays;                 // scratch [S][W]: the entries that stay, as read before anything is written
  int32_t *free_list;             // scratch [min(pages, S W)]
  int4* copies;                   // scratch [S]: (from, to, rows, 0) of a page that is filled in part; to = -1: none
};
cudaError_t launch_pages_update(const PagesUpdate& u, cudaStream_t stream);

struct PagesAttend {
  PageCache c;
  const void* q;
  void* out;
  const int32_t *table, *length;
  const float* slopes;            // [H] or null
  int64_t q_sequence, q_head, out_sequence, out_head;   // strides in elements
  int32_t H;
  int32_t fail_at;                // the self-test's (-1: none): a tile of every warp
  bool bf16;
  float scale;
  int4* splits;                   // scratch, two per share (warp): the unit that begins in it and goes on behind it, and the CTAs that it covers
  float* partials;                // scratch, pages_attend_partials floats
};
bool pages_attend_fits(const PageCache& c, int H);     // tiles are counted in 32 bits
int pages_attend_shares(const PageCache& c, int H);
size_t pages_attend_partials(const PageCache& c, int H);
cudaError_t launch_pages_attend(const PagesAttend& a, cudaStream_t stream);

#ifdef __CUDACC__

// A launch that may begin while the kernel before it on the stream still runs: a token's step is a row of kernels of a few microseconds each, and what a
// launch costs then hides behind the one before.  Every such kernel calls after_earlier_kernels() before it touches memory.
template <class Kernel, class... Args>
cudaError_t launch_early(Kernel kernel, dim3 grid, int threads, size_t smem, cudaStream_t stream, const Args&... args) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
// Waits until the kernels before have completed and what they wrote is seen.
__device__ __forceinline__ void after_earlier_kernels() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The next kernel may be launched (and wait) from here on.
__device__ __forceinline__ void let_next_kernel_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ void store_sector(void* at, const uint32_t* w) {   // 32 bytes, aligned to as many
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
               "r"(w[6]), "r"(w[7]) : "memory");
}

// The sequence that slot `slot` of a grid belongs to.  A grid that must cover ragged ranges without knowing their lengths on the
// host gives sequence s the slots from start(s) = (begin[s] >> shift) + extra * s on: as floor(a + b) - floor(a) >= floor(b), every
// sequence gets ceil(length / 2^shift) + extra - 1 of them at least.  All lanes of a warp call this and get the same answer, found 32 ways at a time;
// with ranges that descend it is some sequence within range.
__device__ __forceinline__ int64_t slot_start(const int32_t* begin, int s, int scale, int shift, int extra) {
  return (((int64_t)begin[s] * scale) >> shift) + (int64_t)extra * s;
}
__device__ __forceinline__ int slot_sequence(const int32_t* begin, int S, int64_t slot, int scale, int shift, int extra) {
  int lo = 0, hi = S;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, s = lo + (int)(threadIdx.x & 31) * step;
    const bool before = s < hi && slot_start(begin, s, scale, shift, extra) <= slot;
    const int n = __popc(__ballot_sync(0xffffffffu, before));
    lo += n > 0 ? (n - 1) * step : 0;
    hi = min(hi, lo + step);
  }
  return lo;
}

__device__ __forceinline__ float nan_f32() { return __int_as_float(0x7fffffff); }

#endif  // __CUDACC__

}  // namespace kf
