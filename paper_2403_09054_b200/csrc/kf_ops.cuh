// Launch interface of the operators around the generation step: norm and rotation of projections (kf_qk_norm.cu),
// beam selection and reordering (kf_beam.cu).
#pragma once

#include "kf_common.cuh"

namespace kf {

// ---- norm, rotation and head-major layout of projection rows
struct QkNormParams {
  const void* qkv;                    // [batch][n] rows of (H + 2 Hkv) heads, strides below
  const void* q_weight;               // [d] of the input's type, or null
  const void* k_weight;
  const int32_t* positions;           // [batch][n] or null: position0 + token
  __half* q;                          // [batch][H][n][d]
  __half* k;                          // [batch][Hkv][n][d]
  __half* v;                          // [batch][Hkv][n][d] or null
  int64_t batch_stride, token_stride; // elements
  int32_t batch, n, H, Hkv, position0;
  int32_t norm, rotary_dims, halves;
  float eps;
  double log2_base;
};
cudaError_t launch_qk_norm(const QkNormParams& P, int head_dim, bool bf16, cudaStream_t stream);

// ---- beam selection
constexpr int BEAM_MAX = 32, BEAM_TAKE_MAX = 64;
enum { LOGITS_F16 = 0, LOGITS_BF16 = 1, LOGITS_F32 = 2 };
struct BeamParams {
  const void* logits;           // [batch][beams] rows of `vocab` values, row_stride elements apart
  const float* scores;          // [batch][beams]
  const unsigned char* finished;   // [batch][beams] or null
  float* out_scores;            // [batch][take]
  int32_t* out_parent;
  int32_t* out_token;
  uint2* lists;                 // scratch: [row][chunk][take] (logit bits, token), best first
  float2* stats;                // scratch: [row][chunk] (maximum, sum of exponentials)
  int64_t row_stride;
  int32_t batch, beams, vocab, take, pad, chunks;
  uint32_t by_lists, by_chunks; // reciprocals for the merge, filled in by launch_beam_select
};
// Chunks a row of logits is cut into; `wide` is the form with 32 values per thread.
void beam_plan(int64_t rows, int vocab, int* chunks, bool* wide);
cudaError_t launch_beam_select(const BeamParams& P, int type, bool wide, cudaStream_t stream);

// ---- rows that follow their beam's parent, in place
constexpr int REORDER_BUFFERS = 8;
struct ReorderBuffer {
  unsigned char* base;      // [outer][batch * beams][row_bytes]
  int64_t row_bytes, outer_stride;
  int32_t outer, width;     // width: bytes moved per thread and row, 16, 4 or 1
  int32_t first_block, blocks_per_row;   // block range of this buffer in the grid
};
struct ReorderParams {
  ReorderBuffer buf[REORDER_BUFFERS];
  const int32_t* parent;    // [batch][beams]
  int32_t n_buffers, batch, beams;
};
// Fills in width, first_block and blocks_per_row and launches.
cudaError_t launch_reorder(ReorderParams P, cudaStream_t stream);

}  // namespace kf
