// The 4-bit cache ("packed" cache): its slot format, the conversions of a row, and the launch interface of the kernels
// that work on it (kf_pack.cu, kf_decode_packed.cu).
//
// A slot holds the K and the V row of one entry in 5d/4 bytes:
//   [0, d/2)          K codes, two features per byte, the even one in the low nibble
//   [d/2, d)          V codes
//   [d, 9d/8)         K groups: (scale, minimum), two binary16 numbers for every 32 features
//   [9d/8, 5d/4)      V groups
// A code c in 0..15 of a group (s, m) stands for the binary16 number s c + m, rounded once (one half-precision fma).
// s = (max - min) / 15 rounded down to binary16, so that no value exceeds the group's largest and nothing overflows;
// c = rint((x - m) * (1 / s)) in binary32, at most 15; s = 0 (a constant group) gives c = 0.  K and V of an entry lie
// together because every reader wants both: at d = 128 a slot is five whole 32-byte sectors.
#pragma once

#include "kf_decode.cuh"

namespace kf {

constexpr int PACK_GROUP = 32;
__host__ __device__ constexpr int packed_slot_bytes(int d) { return d + d / 4; }

struct PackedParams : DecodeParams {   // K, V, err, rope and place fields unused
  unsigned char* cache;   // [units][k][5d/4]
  int32_t* slot_opt;      // [units] or null: slot the new row went to, -1 if it was not stored, ERR_* where the step could not be taken
  __half* row_opt;        // [units][2][d] or null: the new K and V row as the values their codes stand for
};

void decode_packed_plan(int units, int budget_k, int head_dim, int* splits, int* tiles_per_split);
cudaError_t launch_decode_packed(const PackedParams& P, int head_dim, int units, cudaStream_t stream);

// Rows [units][n][d] <-> slots 0 .. n-1 of [units][k] (with `len`, only those below the unit's entry count).
cudaError_t launch_pack(const __half* K, const __half* V, const int32_t* len, unsigned char* cache, int64_t units, int n, int k,
                        int head_dim, cudaStream_t stream);
cudaError_t launch_unpack(const unsigned char* cache, const int32_t* len, __half* K, __half* V, int64_t units, int n, int k,
                          int head_dim, cudaStream_t stream);

#ifdef __CUDACC__

// (scale, minimum) of a group with these extremes.  A NaN or an infinity among the features arrives here as an extreme
// that is not finite: the whole group then reads back as NaN.
__device__ __forceinline__ __half2 packed_group(float low, float high) {
  const float range = __fsub_rn(high, low);
  const bool finite = range <= 131008.0f;   // the span of finite binary16 numbers; false for NaN too
  const __half nan = __ushort_as_half((unsigned short)0x7fffu);
  // range / 15, correctly rounded: a quotient by the rounded reciprocal and one correction by the remainder, which the
  // fused multiply-add gives exactly (Markstein 1990)
  const float q = __fmul_rn(range, 1.0f / 15.0f);
  const float span = fmaf(fmaf(-15.0f, q, range), 1.0f / 15.0f, q);
  return finite ? __halves2half2(__float2half_rd(span), __float2half_rn(low)) : __halves2half2(nan, nan);
}
// 1 / scale, or 0 where every code of the group is 0.
__device__ __forceinline__ float packed_inverse(__half scale) {
  const float s = __half2float(scale);
  float y;
  asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(s));   // to the last place; one Newton step with exact residual rounds it
  y = fmaf(y, fmaf(-s, y, 1.0f), y);
  return s > 0.f ? y : 0.f;              // false for NaN
}
__device__ __forceinline__ uint32_t packed_code(float x, float low, float inverse) {
  const float c = rintf(__fmul_rn(__fsub_rn(x, low), inverse));
  return (uint32_t)fminf(fmaxf(c, 0.f), 15.f);   // a NaN (group not finite) gives 0
}
__device__ __forceinline__ uint32_t h2_bits(__half2 v) { return *reinterpret_cast<const uint32_t*>(&v); }
__device__ __forceinline__ __half2 bits_h2(uint32_t v) { return *reinterpret_cast<const __half2*>(&v); }

// (w & mask) | bits in one instruction: both constants in registers, which the compiler does not do by itself.
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(bits));
  return r;
}
// Eight nibbles -> four pairs (nibble i, nibble i + 4) of binary16 integers 0..15, exact.  1024 + c has the bits
// 0x6400 | c, and 1024 + 16 c the bits 0x6400 | 16 c: one logic instruction per pair, and one arithmetic instruction
// that takes the offset off again.
__device__ __forceinline__ void nibble_pairs(uint32_t w, __half2 (&c)[4]) {
  const uint32_t w8 = w >> 8;
  const __half2 sixteenth = __floats2half2_rn(0.0625f, 0.0625f);
  c[0] = __hadd2(bits_h2(and_or(w, 0x000f000fu, 0x64006400u)), bits_h2(0xe400e400u));                  // - 1024
  c[1] = __hfma2(bits_h2(and_or(w, 0x00f000f0u, 0x64006400u)), sixteenth, bits_h2(0xd400d400u));       // / 16 - 64
  c[2] = __hadd2(bits_h2(and_or(w8, 0x000f000fu, 0x64006400u)), bits_h2(0xe400e400u));
  c[3] = __hfma2(bits_h2(and_or(w8, 0x00f000f0u, 0x64006400u)), sixteenth, bits_h2(0xd400d400u));
}

#endif  // __CUDACC__

}  // namespace kf
