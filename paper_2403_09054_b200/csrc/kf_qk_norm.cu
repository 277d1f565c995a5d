// From a model's projection rows to what the prompt phase and the generation step take: per head the root-mean-square
// norm of queries and keys (x r w, r = 1 / sqrt(mean(x^2) + eps)) and the rotary embedding, then head-major binary16
// rows; the values are only laid out.  Every value is read once and written once: HBM bounds it.
//
// A head's row is d / 8 neighbouring lanes with eight features (16 bytes) each, so that the sum of squares takes
// log2(d / 8) shuffles and a pair of features that turn together lies in one lane (pairs 2i, 2i + 1) or in two lanes
// R / 16 apart (pairs i, i + R / 2).  The angles of a token are shared by all of its heads: a CTA computes them once
// into shared memory.  Positions reach far, so angle / 2 pi is formed and reduced in binary64; what is left, at most
// half a turn, goes through binary32.
#include <cuda_bf16.h>

#include "kf_ops.cuh"

namespace kf {

namespace {

constexpr int THREADS = 256;
constexpr int MAX_TOKENS = 8;     // tokens per CTA (few heads: several, so that all threads have a row)
constexpr int UNROLL = 2;         // rows in flight per lane, and as many being worked on

template <class T>
__device__ __forceinline__ void widen(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 f;
    if constexpr (sizeof(T) == 2 && __is_same(T, __half)) f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    else f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

// A CTA works on one token, or, where a token has fewer rows than the CTA has places, on several with one row per
// place; either way a thread's token never changes, and its share of the token's angles and of the weights stays in registers.
template <int D, class T, bool HALVES>
__global__ void __launch_bounds__(THREADS, 4) qk_norm_kernel(const __grid_constant__ QkNormParams P, int tokens_per_cta) {
  constexpr int LPR = D / 8;                    // lanes per row
  constexpr int PLACES = THREADS / LPR;         // rows the CTA works on at a time
  constexpr int NCS = HALVES ? 8 : 4;           // pairs that this lane's features take part in
  __shared__ float2 turn[MAX_TOKENS][D / 2];    // (cos, sin)
  const int tid = threadIdx.x, lane = tid & 31, sub = lane % LPR, place = tid / LPR;
  const int64_t tokens = (int64_t)P.batch * P.n, first = (int64_t)blockIdx.x * tokens_per_cta;
  const int here = (int)(tokens - first < tokens_per_cta ? tokens - first : tokens_per_cta);
  const int half = P.rotary_dims / 2;
  const int rows_per_token = P.H + (P.v ? 2 : 1) * P.Hkv;
  const int tk = tokens_per_cta > 1 ? place / rows_per_token : 0;
  const int row0 = tokens_per_cta > 1 ? place % rows_per_token : place;
  const int rows = tk < here ? rows_per_token : 0;          // a place without a token takes part in the shuffles only
  const int64_t tok = first + (tk < here ? tk : 0), b = tok / P.n, t = tok % P.n;
  const T* src = static_cast<const T*>(P.qkv) + b * P.batch_stride + t * P.token_stride + sub * 8;

  uint4 raw[UNROLL];
  auto load = [&](int row) {
#pragma unroll
    for (int i = 0; i < UNROLL; ++i)
      raw[i] = row + i * PLACES < rows ? __ldcs(reinterpret_cast<const uint4*>(src + (int64_t)(row + i * PLACES) * D)) : make_uint4(0, 0, 0, 0);
  };
  load(row0);   // in flight while the angles are computed

  for (int idx = tid; idx < here * half; idx += THREADS) {
    const int tk2 = idx / half, i = idx % half;
    const int64_t tok2 = first + tk2;
    const int pos = P.positions ? P.positions[tok2] : P.position0 + (int)(tok2 % P.n);
    const double turns = (double)pos * (exp2(-P.log2_base * (double)i / (double)half) * 0.15915494309189535);
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    turn[tk2][i] = make_float2(c, s);
  }
  constexpr uint32_t ONES = __is_same(T, __half) ? 0x3c003c00u : 0x3f803f80u;
  uint4 wq = make_uint4(ONES, ONES, ONES, ONES), wk = wq;      // weights, as they came
  if (P.norm && P.q_weight) wq = __ldg(static_cast<const uint4*>(P.q_weight) + sub);
  if (P.norm && P.k_weight) wk = __ldg(static_cast<const uint4*>(P.k_weight) + sub);
  __syncthreads();
  // features that stay as they are turn by nothing
  const bool turns_here = 8 * sub < 2 * half;
  const bool low = 8 * sub < half;               // HALVES: this lane holds the first features of its pairs
  float cs[NCS], sn[NCS];
#pragma unroll
  for (int e = 0; e < NCS; ++e) {
    float2 v = make_float2(1.f, 0.f);
    if (turns_here) {
      if constexpr (!HALVES) v = turn[tk < here ? tk : 0][4 * sub + e];
      else v = turn[tk < here ? tk : 0][half == 4 ? e & 3 : (low ? 8 * sub : 8 * sub - half) + e];
    }
    cs[e] = v.x;
    // what the other feature of the pair is multiplied by: a c - b s for the first one, b c + a s for the second
    sn[e] = HALVES && (half == 4 ? e < 4 : low) ? -v.y : v.y;
  }

  const int rounds = (rows_per_token + PLACES - 1) / PLACES;
  for (int r0 = 0; r0 < rounds; r0 += UNROLL) {
    uint4 now[UNROLL];
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) now[i] = raw[i];
    if (r0 + UNROLL < rounds) load(row0 + (r0 + UNROLL) * PLACES);
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      if (r0 + i >= rounds) break;                // the same for the whole CTA
      const int head = row0 + (r0 + i) * PLACES;
      const bool is_q = head < P.H, is_v = head >= P.H + P.Hkv;
      float x[8];
      widen<T>(now[i], x);
      if (P.norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float r = rsqrtf(fmaf(ss, 1.0f / (float)D, P.eps));
        if (!is_v) {
          float w[8];
          widen<T>(is_q ? wq : wk, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= r * w[e];
        }
      }
      if (half > 0) {
        if constexpr (!HALVES) {
          if (!is_v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float a = x[2 * e], c = x[2 * e + 1];
              x[2 * e] = a * cs[e] - c * sn[e];
              x[2 * e + 1] = fmaf(a, sn[e], c * cs[e]);
            }
          }
        } else {
          float other[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) other[e] = half == 4 ? x[e ^ 4] : __shfl_xor_sync(0xffffffffu, x[e], half / 8);
          if (!is_v) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = fmaf(other[e], sn[e], x[e] * cs[e]);
          }
        }
      }
      if (head < rows) {
        __half* base = is_q ? P.q : (is_v ? P.v : P.k);
        const int64_t slab = is_q ? b * P.H + head : b * P.Hkv + head - P.H - (is_v ? P.Hkv : 0);
        __half* dst = base + (slab * P.n + t) * D;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const __half2 h = __floats2half2_rn(x[2 * e], x[2 * e + 1]);
          w[e] = *reinterpret_cast<const uint32_t*>(&h);
        }
        reinterpret_cast<uint4*>(dst)[sub] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}

template <int D>
cudaError_t launch_dim(const QkNormParams& P, bool bf16, cudaStream_t stream) {
  const int rows = P.H + (P.v ? 2 : 1) * P.Hkv;
  int per_cta = THREADS / (D / 8) / rows;
  per_cta = per_cta < 1 ? 1 : (per_cta > MAX_TOKENS ? MAX_TOKENS : per_cta);
  const int64_t tokens = (int64_t)P.batch * P.n;
  const unsigned grid = (unsigned)((tokens + per_cta - 1) / per_cta);
  if (bf16 && P.halves) qk_norm_kernel<D, __nv_bfloat16, true><<<grid, THREADS, 0, stream>>>(P, per_cta);
  else if (bf16) qk_norm_kernel<D, __nv_bfloat16, false><<<grid, THREADS, 0, stream>>>(P, per_cta);
  else if (P.halves) qk_norm_kernel<D, __half, true><<<grid, THREADS, 0, stream>>>(P, per_cta);
  else qk_norm_kernel<D, __half, false><<<grid, THREADS, 0, stream>>>(P, per_cta);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_qk_norm(const QkNormParams& P, int head_dim, bool bf16, cudaStream_t stream) {
  switch (head_dim) {
    case 64: return launch_dim<64>(P, bf16, stream);
    case 128: return launch_dim<128>(P, bf16, stream);
    case 256: return launch_dim<256>(P, bf16, stream);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kf
