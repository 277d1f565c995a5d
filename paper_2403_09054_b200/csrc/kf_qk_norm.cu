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
constexpr int UNROLL = 4;         // rows in flight per lane

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

template <int D, class T>
__global__ void __launch_bounds__(THREADS) qk_norm_kernel(const __grid_constant__ QkNormParams P, int tokens_per_cta) {
  constexpr int LPR = D / 8;                    // lanes per row
  constexpr int SLOTS = THREADS / LPR;          // rows the CTA works on at a time
  __shared__ float2 turn[MAX_TOKENS][D / 2];    // (cos, sin)
  const int tid = threadIdx.x, lane = tid & 31, sub = lane % LPR;
  const int64_t tokens = (int64_t)P.batch * P.n, first = (int64_t)blockIdx.x * tokens_per_cta;
  const int here = (int)(tokens - first < tokens_per_cta ? tokens - first : tokens_per_cta);
  const int half = P.rotary_dims / 2;
  const int rows_per_token = P.H + (P.v ? 2 : 1) * P.Hkv, total = here * rows_per_token;

  auto source = [&](int row) -> const uint4* {
    const int64_t tok = first + row / rows_per_token;
    const int64_t b = tok / P.n, t = tok % P.n;
    return reinterpret_cast<const uint4*>(static_cast<const T*>(P.qkv) + b * P.batch_stride + t * P.token_stride +
                                          (int64_t)(row % rows_per_token) * D) + sub;
  };
  uint4 raw[UNROLL];
  auto load = [&](int base) {
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      const int row = base + i * SLOTS + tid / LPR;
      raw[i] = row < total ? __ldcs(source(row)) : make_uint4(0, 0, 0, 0);
    }
  };
  load(0);   // in flight while the angles are computed

  for (int idx = tid; idx < here * half; idx += THREADS) {
    const int tk = idx / half, i = idx % half;
    const int64_t tok = first + tk;
    const int pos = P.positions ? P.positions[tok] : P.position0 + (int)(tok % P.n);
    const double turns = (double)pos * (exp2(-P.log2_base * (double)i / (double)half) * 0.15915494309189535);
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    turn[tk][i] = make_float2(c, s);
  }
  float wq[8], wk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) wq[e] = wk[e] = 1.f;
  if (P.norm && P.q_weight) widen<T>(__ldg(static_cast<const uint4*>(P.q_weight) + sub), wq);
  if (P.norm && P.k_weight) widen<T>(__ldg(static_cast<const uint4*>(P.k_weight) + sub), wk);
  __syncthreads();

  for (int base = 0; base < total; base += UNROLL * SLOTS) {
    if (base > 0) load(base);
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      const int row = base + i * SLOTS + tid / LPR;      // lanes without a row take part in the shuffles
      const int tk = row < total ? row / rows_per_token : 0, head = row % rows_per_token;
      const bool is_q = head < P.H, is_v = head >= P.H + P.Hkv;
      float x[8];
      widen<T>(raw[i], x);
      if (P.norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float r = rsqrtf(fmaf(ss, 1.0f / (float)D, P.eps));
        if (!is_v) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= r * (is_q ? wq[e] : wk[e]);
        }
      }
      if (half > 0) {
        if (!P.halves) {
          if (!is_v && 8 * sub < 2 * half) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 cs = turn[tk][4 * sub + e];
              const float a = x[2 * e], bb = x[2 * e + 1];
              x[2 * e] = a * cs.x - bb * cs.y;
              x[2 * e + 1] = fmaf(a, cs.y, bb * cs.x);
            }
          }
        } else if (half == 4) {
          if (!is_v && sub == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 cs = turn[tk][e];
              const float a = x[e], bb = x[e + 4];
              x[e] = a * cs.x - bb * cs.y;
              x[e + 4] = fmaf(a, cs.y, bb * cs.x);
            }
          }
        } else {
          const bool low = 8 * sub < half;               // this lane holds the first features of its pairs
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float other = __shfl_xor_sync(0xffffffffu, x[e], half / 8);
            if (!is_v && 8 * sub < 2 * half) {
              const float2 cs = turn[tk][(low ? 8 * sub : 8 * sub - half) + e];
              x[e] = low ? x[e] * cs.x - other * cs.y : fmaf(other, cs.y, x[e] * cs.x);
            }
          }
        }
      }
      if (row < total) {
        const int64_t tok = first + tk, b = tok / P.n, t = tok % P.n;
        __half* dst = is_q ? P.q + ((b * P.H + head) * P.n + t) * D
                           : (is_v ? P.v + ((b * P.Hkv + head - P.H - P.Hkv) * P.n + t) * D : P.k + ((b * P.Hkv + head - P.H) * P.n + t) * D);
        uint4 out;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const __half2 h = __floats2half2_rn(x[2 * e], x[2 * e + 1]);
          w[e] = *reinterpret_cast<const uint32_t*>(&h);
        }
        out = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(dst)[sub] = out;
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
  if (bf16) qk_norm_kernel<D, __nv_bfloat16><<<grid, THREADS, 0, stream>>>(P, per_cta);
  else qk_norm_kernel<D, __half><<<grid, THREADS, 0, stream>>>(P, per_cta);
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
