// Conversion of cache rows between binary16 and the 4-bit slots of kf_packed.cuh.  Pure streaming: every row is read
// once and every slot written once, so HBM bounds both directions (4 d + 1.25 d bytes per slot).
//
// Packing, a thread owns sixteen features (two 16-byte chunks) of the K row and of the V row of a slot: four loads are in
// flight per thread, and a group of 32 features is two neighbouring lanes, one of which works out the K group and the other
// the V group.  Unpacking, it owns eight of each.
//
// 1024 units of 2048 rows, d 128: pack 218 us, 1.41 GB at the rate of a copy, unpack 231 us, 0.94 of it.  With eight features a thread
// packing took 325 us (four lanes worked out the same group, 250 instructions per 16 features); with a division and a reciprocal
// each and codes shifted into place one by one 415.  Unpacking sixteen features a thread takes 286 (stores in halves of 32 bytes).
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

// The groups that this lane's features belong to; the two lanes of a group call it together.  The even lane works out the K
// group, the odd one the V group, and they exchange: one division and one reciprocal per lane.
__device__ __forceinline__ void groups_of(const uint4 (&kv)[2], const uint4 (&vv)[2], Group& kg, Group& vg) {
  __half2 klo, khi, vlo, vhi, l2, h2;
  extremes8(kv[0], klo, khi);
  extremes8(kv[1], l2, h2);
  klo = __hmin2_nan(klo, l2);
  khi = __hmax2_nan(khi, h2);
  extremes8(vv[0], vlo, vhi);
  extremes8(vv[1], l2, h2);
  vlo = __hmin2_nan(vlo, l2);
  vhi = __hmax2_nan(vhi, h2);
  klo = __hmin2_nan(klo, __lowhigh2highlow(klo));
  khi = __hmax2_nan(khi, __lowhigh2highlow(khi));
  vlo = __hmin2_nan(vlo, __lowhigh2highlow(vlo));
  vhi = __hmax2_nan(vhi, __lowhigh2highlow(vhi));
  __half2 lo = __lows2half2(klo, vlo), hi = __lows2half2(khi, vhi);   // (K, V)
  lo = __hmin2_nan(lo, __shfl_xor_sync(0xffffffffu, lo, 1));
  hi = __hmax2_nan(hi, __shfl_xor_sync(0xffffffffu, hi, 1));
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

template <bool CLAMP>
__device__ __forceinline__ uint2 pack16(const uint4 (&v)[2], const Group& g) {
  return make_uint2(pack8<CLAMP>(v[0], __high2float(g.params), g.inverse), pack8<CLAMP>(v[1], __high2float(g.params), g.inverse));
}

// grid: chunks of a unit's rows, units (the rest of them in further rounds)
template <int D>
__global__ void __launch_bounds__(THREADS) pack_kernel(const __half* __restrict__ K, const __half* __restrict__ V,
                                                       const int32_t* __restrict__ len, unsigned char* __restrict__ cache,
                                                       int64_t units, int n, int k) {
  constexpr int TPR = D / 16;   // threads per row
  const int64_t at = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  const int64_t j = at / TPR;
  const int c = (int)(at % TPR);
  for (int64_t u = blockIdx.y; u < units; u += gridDim.y) {
    const bool in = j < n && (!len || j < len[u]);
    const int64_t row = u * n + j;
    uint4 kv[2], vv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      kv[i] = vv[i] = make_uint4(0, 0, 0, 0);
      if (in) {
        kv[i] = __ldcs(reinterpret_cast<const uint4*>(K + row * D) + 2 * c + i);
        vv[i] = __ldcs(reinterpret_cast<const uint4*>(V + row * D) + 2 * c + i);
      }
    }
    Group kg, vg;
    groups_of(kv, vv, kg, vg);   // whole warps: a group never straddles a row
    if (in) {
      unsigned char* slot = cache + ((size_t)u * k + j) * packed_slot_bytes(D);
      uint2 kc, vc;
      if (kg.clamp) {            // the same for the whole warp
        kc = pack16<true>(kv, kg);
        vc = pack16<true>(vv, vg);
      } else {
        kc = pack16<false>(kv, kg);
        vc = pack16<false>(vv, vg);
      }
      *reinterpret_cast<uint2*>(slot + 8 * c) = kc;
      *reinterpret_cast<uint2*>(slot + D / 2 + 8 * c) = vc;
      // one lane of the group writes its K parameters, the other its V parameters
      *reinterpret_cast<uint32_t*>(slot + D + (c & 1) * (D / 8) + (c >> 1) * 4) = h2_bits(c & 1 ? vg.params : kg.params);
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

inline dim3 grid_for(int64_t units, int n, int threads_per_row) {
  return dim3((unsigned)(((int64_t)n * threads_per_row + THREADS - 1) / THREADS), (unsigned)(units < 65535 ? units : 65535));
}

}  // namespace

cudaError_t launch_pack(const __half* K, const __half* V, const int32_t* len, unsigned char* cache, int64_t units, int n, int k,
                        int head_dim, cudaStream_t stream) {
  const dim3 grid = grid_for(units, n, head_dim / 16);
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
  const dim3 grid = grid_for(units, n, head_dim / 8);
  switch (head_dim) {
    case 64: unpack_kernel<64><<<grid, THREADS, 0, stream>>>(cache, len, K, V, units, n, k); break;
    case 128: unpack_kernel<128><<<grid, THREADS, 0, stream>>>(cache, len, K, V, units, n, k); break;
    case 256: unpack_kernel<256><<<grid, THREADS, 0, stream>>>(cache, len, K, V, units, n, k); break;
    default: return cudaErrorInvalidValue;
  }
  return cudaGetLastError();
}

}  // namespace kf
