// Conversion of cache rows between binary16 and the 4-bit slots of kf_packed.cuh.  Pure streaming: every row is read
// once and every slot written once, so HBM bounds both directions (4 d + 1.25 d bytes per slot).
//
// A thread owns eight features (one 16-byte chunk) of the K row and of the V row of a slot, so that two loads are in
// flight per thread and a group of 32 features is four neighbouring lanes: its extremes take two shuffles each.
//
// 1024 units of 2048 rows, d 128: unpack 210 us (6.7 TB/s, as fast as a copy), pack 325 us (4.3 TB/s): rounding 16 features to codes
// takes about 250 instructions a thread (issue slots 87 %); 415 us with a division and a reciprocal per chunk and codes shifted into
// place one by one.
#include "kf_packed.cuh"

namespace kf {

namespace {

constexpr int THREADS = 256;

// Extremes of the eight features; a NaN wins over every number, so that a group that holds one is recognised.
__device__ __forceinline__ void extremes8(const uint4& v, __half2& low, __half2& high) {
  const __half2 a = bits_h2(v.x), b = bits_h2(v.y), c = bits_h2(v.z), d = bits_h2(v.w);
  low = __hmin2_nan(__hmin2_nan(a, b), __hmin2_nan(c, d));
  high = __hmax2_nan(__hmax2_nan(a, b), __hmax2_nan(c, d));
}

// Eight codes.  Adding M = 1.5 * 2^23 rounds to whole numbers (to even, as rintf does) and leaves the code in the low bits of
// M's own; the eight words are shifted and added up as they are, and the M's taken off together (modulo 2^32).
constexpr float M = 12582912.f;
constexpr uint32_t M_BITS = 0x4b400000u;
template <bool CLAMP>
__device__ __forceinline__ uint32_t pack8(const uint4& v, float low, float inverse) {
  auto place = [&](float x) {
    float p = __fmul_rn(__fsub_rn(x, low), inverse);
    if (CLAMP) p = fminf(p, 15.f);
    return __float_as_uint(__fadd_rn(p, M));
  };
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t code = 0u - M_BITS * 0x11111111u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(bits_h2(w[i]));
    code += (place(f.x) << 8 * i) + (place(f.y) << (8 * i + 4));
  }
  return low == low ? code : 0u;   // not finite: every code 0
}

struct Group {
  __half2 params;   // (scale, minimum)
  float inverse;
  bool clamp;       // whether a code could pass 15 (scales of few bits, near the smallest binary16 numbers), of either group
};

// The groups that this lane's two chunks belong to; the four lanes of a group call it together.  The even lanes work out the
// K group, the odd ones the V group, and neighbours exchange: one division and one reciprocal per lane.
__device__ __forceinline__ void groups_of(const uint4& kv, const uint4& vv, Group& kg, Group& vg) {
  __half2 klo, khi, vlo, vhi;
  extremes8(kv, klo, khi);
  extremes8(vv, vlo, vhi);
  klo = __hmin2_nan(klo, __lowhigh2highlow(klo));
  khi = __hmax2_nan(khi, __lowhigh2highlow(khi));
  vlo = __hmin2_nan(vlo, __lowhigh2highlow(vlo));
  vhi = __hmax2_nan(vhi, __lowhigh2highlow(vhi));
  __half2 lo = __lows2half2(klo, vlo), hi = __lows2half2(khi, vhi);   // (K, V)
#pragma unroll
  for (int o = 1; o <= 2; o <<= 1) {
    lo = __hmin2_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = __hmax2_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const bool odd = threadIdx.x & 1;
  Group mine;
  const float low = __half2float(odd ? __high2half(lo) : __low2half(lo)), high = __half2float(odd ? __high2half(hi) : __low2half(hi));
  mine.params = packed_group(low, high);
  mine.inverse = packed_inverse(__low2half(mine.params));
  mine.clamp = !(__fmul_rn(__fsub_rn(high, low), mine.inverse) < 15.5f);   // the largest quotient of the group
  Group other;
  other.params = __shfl_xor_sync(0xffffffffu, mine.params, 1);
  other.inverse = __shfl_xor_sync(0xffffffffu, mine.inverse, 1);
  other.clamp = mine.clamp = __any_sync(0xffffffffu, mine.clamp);
  kg = odd ? other : mine;
  vg = odd ? mine : other;
}

// grid: chunks of a unit's rows, units (the rest of them in further rounds)
template <int D>
__global__ void __launch_bounds__(THREADS) pack_kernel(const __half* __restrict__ K, const __half* __restrict__ V,
                                                       const int32_t* __restrict__ len, unsigned char* __restrict__ cache,
                                                       int64_t units, int n, int k) {
  constexpr int CPR = D / 8;   // chunks per row
  const int64_t at = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  const int64_t j = at / CPR;
  const int c = (int)(at % CPR);
  for (int64_t u = blockIdx.y; u < units; u += gridDim.y) {
    const bool in = j < n && (!len || j < len[u]);
    const int64_t row = u * n + j;
    uint4 kv = make_uint4(0, 0, 0, 0), vv = kv;
    if (in) {
      kv = __ldcs(reinterpret_cast<const uint4*>(K + row * D) + c);
      vv = __ldcs(reinterpret_cast<const uint4*>(V + row * D) + c);
    }
    Group kg, vg;
    groups_of(kv, vv, kg, vg);   // whole warps: a group never straddles a row
    if (in) {
      unsigned char* slot = cache + ((size_t)u * k + j) * packed_slot_bytes(D);
      uint32_t kc, vc;
      if (kg.clamp) {            // the same for the whole warp
        kc = pack8<true>(kv, __high2float(kg.params), kg.inverse);
        vc = pack8<true>(vv, __high2float(vg.params), vg.inverse);
      } else {
        kc = pack8<false>(kv, __high2float(kg.params), kg.inverse);
        vc = pack8<false>(vv, __high2float(vg.params), vg.inverse);
      }
      *reinterpret_cast<uint32_t*>(slot + 4 * c) = kc;
      *reinterpret_cast<uint32_t*>(slot + D / 2 + 4 * c) = vc;
      if ((c & 3) == 0) {
        *reinterpret_cast<uint32_t*>(slot + D + c) = h2_bits(kg.params);
        *reinterpret_cast<uint32_t*>(slot + D + D / 8 + c) = h2_bits(vg.params);
      }
    }
  }
}

__device__ __forceinline__ uint4 unpack8(uint32_t w, __half2 group) {
  const __half2 s = __low2half2(group), m = __high2half2(group);
  __half2 c[4];
  nibble_pairs(w, c);
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = __hfma2(c[i], s, m);   // pairs (i, i + 4)
  uint4 out;
  out.x = h2_bits(__lows2half2(c[0], c[1]));
  out.y = h2_bits(__lows2half2(c[2], c[3]));
  out.z = h2_bits(__highs2half2(c[0], c[1]));
  out.w = h2_bits(__highs2half2(c[2], c[3]));
  return out;
}

template <int D>
__global__ void __launch_bounds__(THREADS) unpack_kernel(const unsigned char* __restrict__ cache, const int32_t* __restrict__ len,
                                                         __half* __restrict__ K, __half* __restrict__ V, int64_t units, int n, int k) {
  constexpr int CPR = D / 8;
  const int64_t at = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  const int64_t j = at / CPR;
  const int c = (int)(at % CPR);
  if (j >= n) return;
  for (int64_t u = blockIdx.y; u < units; u += gridDim.y) {
    if (len && j >= len[u]) continue;
    const int64_t row = u * n + j;
    const unsigned char* slot = cache + ((size_t)u * k + j) * packed_slot_bytes(D);
    const uint32_t kw = *reinterpret_cast<const uint32_t*>(slot + 4 * c), vw = *reinterpret_cast<const uint32_t*>(slot + D / 2 + 4 * c);
    const uint32_t kg = *reinterpret_cast<const uint32_t*>(slot + D + 4 * (c / 4));
    const uint32_t vg = *reinterpret_cast<const uint32_t*>(slot + D + D / 8 + 4 * (c / 4));
    __stcs(reinterpret_cast<uint4*>(K + row * D) + c, unpack8(kw, bits_h2(kg)));
    __stcs(reinterpret_cast<uint4*>(V + row * D) + c, unpack8(vw, bits_h2(vg)));
  }
}

inline dim3 grid_for(int64_t units, int n, int d) {
  return dim3((unsigned)(((int64_t)n * (d / 8) + THREADS - 1) / THREADS), (unsigned)(units < 65535 ? units : 65535));
}

}  // namespace

cudaError_t launch_pack(const __half* K, const __half* V, const int32_t* len, unsigned char* cache, int64_t units, int n, int k,
                        int head_dim, cudaStream_t stream) {
  const dim3 grid = grid_for(units, n, head_dim);
  switch (head_dim) {
    case 64: pack_kernel<64><<<grid, THREADS, 0, stream>>>(K, V, len, cache, units, n, k); break;
    case 128: pack_kernel<128><<<grid, THREADS, 0, stream>>>(K, V, len, cache, units, n, k); break;
    case 256: pack_kernel<256><<<grid, THREADS, 0, stream>>>(K, V, len, cache, units, n, k); break;
    default: return cudaErrorInvalidValue;
  }
  return cudaGetLastError();
}

cudaError_t launch_unpack(const unsigned char* cache, const int32_t* len, __half* K, __half* V, int64_t units, int n, int k,
                          int head_dim, cudaStream_t stream) {
  const dim3 grid = grid_for(units, n, head_dim);
  switch (head_dim) {
    case 64: unpack_kernel<64><<<grid, THREADS, 0, stream>>>(cache, len, K, V, units, n, k); break;
    case 128: unpack_kernel<128><<<grid, THREADS, 0, stream>>>(cache, len, K, V, units, n, k); break;
    case 256: unpack_kernel<256><<<grid, THREADS, 0, stream>>>(cache, len, K, V, units, n, k); break;
    default: return cudaErrorInvalidValue;
  }
  return cudaGetLastError();
}

}  // namespace kf
