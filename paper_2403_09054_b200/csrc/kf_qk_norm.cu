// From a model's projection rows to what the prompt phase and the generation step take: per head the root-mean-square
// norm of queries and keys (x r w, r = 1 / sqrt(mean(x^2) + eps)) and the rotary embedding, then head-major binary16
// rows; the values are only laid out.  Every value is read once and written once: HBM bounds it.
//
// A head's row is d / 8 neighbouring lanes with eight features each, two runs of four that are chosen so that the features
// of a pair lie in one lane: [4 l, 4 l + 4) and [R/2 + 4 l, ...) of the rotary features for pairs (i, i + R/2), eight
// neighbours for pairs (2i, 2i + 1) and for what does not turn.  The sum of squares takes log2(d / 8) shuffles, the rotation
// none.  The angles of a token are shared by all of its heads: a CTA takes up to eight tokens and computes their angles
// first, one per thread, into shared memory.  Positions reach far, so angle / 2 pi is formed and reduced in binary64; what
// is left, at most half a turn, goes through binary32.
//
// 8 x 4096 tokens of 32 + 32 heads, d 128, whole heads turned (1.6 GB): 302 us = 5.3 TB/s, 0.83 of a copy; 32 tokens of 32 + 8 heads
// 3.3 us.  What it took: angles in registers instead of shared memory for every row 908 -> 382, pairs within a lane (no
// shuffles) 342, six rows requested ahead and streaming stores 302 (three 324, twelve 367: registers).  In bfloat16 the same prompt takes 341 us (halves; 325 in pairs) through the Python call, binary16 320; rows
// whose squares leave binary32 cost a second pass of their warp, looking for them 1 % (scaling them where they are met: 8 %).
#include <cuda_bf16.h>

#include <type_traits>

#include "kf_ops.cuh"

namespace kf {

namespace {

constexpr int THREADS = 256;
constexpr int MAX_TOKENS = 8;     // tokens per CTA
constexpr int AHEAD = 6;          // rows a lane requests before it works on the first

// Four values of a run.
template <class T>
__device__ __forceinline__ void widen(const uint2& v, float* x) {
  const uint32_t w[2] = {v.x, v.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float2 f;
    if constexpr (__is_same(T, __half)) f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    else f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint2 narrow(const float* x) {
  const __half2 a = __floats2half2_rn(x[0], x[1]), b = __floats2half2_rn(x[2], x[3]);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// A round of the CTA is one row for every place (d / 8 lanes): PLACES rows of one token, or, where a token has fewer rows than
// that, one row each of several tokens.
template <int D, class T, bool HALVES>
__global__ void __launch_bounds__(THREADS, 3) qk_norm_kernel(const __grid_constant__ QkNormParams P, int tokens_per_cta) {
  constexpr int LPR = D / 8;                    // lanes per row
  constexpr int PLACES = THREADS / LPR;
  __shared__ __align__(16) float2 turn[MAX_TOKENS][D / 2];    // (cos, sin)
  // bfloat16 reaches as far as binary32, so the squares of a row may leave it.  Where a mean square was not inside [2^-96, 2^96] (as words:
  // LOW + [0, SPAN]), the warp works on its rows of the token once more and scales such rows.
  constexpr bool FAR_ROWS = !__is_same(T, __half);
  constexpr uint32_t LOW = 0x0f800000u, SPAN = 0x60000000u;
  const int tid = threadIdx.x, sub = tid % LPR, place = tid / LPR;
  const int64_t tokens = (int64_t)P.batch * P.n, first = (int64_t)blockIdx.x * tokens_per_cta;
  const int here = (int)(tokens - first < tokens_per_cta ? tokens - first : tokens_per_cta);
  const int half = P.rotary_dims / 2;
  const int rows = P.H + (P.v ? 2 : 1) * P.Hkv;
  const int side = rows < PLACES ? PLACES / rows : 1;            // tokens side by side in a round
  const int my_token = rows < PLACES ? place / rows : 0, row0 = rows < PLACES ? place % rows : place;
  const bool idle = my_token >= side;                            // places left over; they take part in the shuffles
  // the lane's two runs of four features
  const bool turns = 8 * sub < P.rotary_dims;
  const int run0 = HALVES && turns ? 4 * sub : 8 * sub, run1 = HALVES && turns ? half + 4 * sub : 8 * sub + 4;

  for (int idx = tid; idx < here * half; idx += THREADS) {
    const int tk = idx / half, i = idx % half;
    const int64_t tok = first + tk;
    const int pos = P.positions ? P.positions[tok] : P.position0 + (int)(tok % P.n);
    const double turned = (double)pos * (exp2(-P.log2_base * (double)i / (double)half) * 0.15915494309189535);
    float s, c;
    sincospif(2.0f * (float)(turned - rint(turned)), &s, &c);
    turn[tk][i] = make_float2(c, s);
  }
  constexpr uint32_t ONES = __is_same(T, __half) ? 0x3c003c00u : 0x3f803f80u;
  uint2 wq[2] = {make_uint2(ONES, ONES), make_uint2(ONES, ONES)}, wk[2] = {wq[0], wq[0]};      // weights, as they came
  if (P.q_weight) {
    wq[0] = __ldg(reinterpret_cast<const uint2*>(static_cast<const T*>(P.q_weight) + run0));
    wq[1] = __ldg(reinterpret_cast<const uint2*>(static_cast<const T*>(P.q_weight) + run1));
  }
  if (P.k_weight) {
    wk[0] = __ldg(reinterpret_cast<const uint2*>(static_cast<const T*>(P.k_weight) + run0));
    wk[1] = __ldg(reinterpret_cast<const uint2*>(static_cast<const T*>(P.k_weight) + run1));
  }
  __syncthreads();

  uint32_t farthest = 0;
  auto walk = [&](auto again) {
    for (int group = 0; group < here; group += side) {
      const int tk = group + my_token;
      const bool there = !idle && tk < here;
      const int64_t tok = first + (there ? tk : 0), b = tok / P.n, t = tok % P.n;
      const T* src = static_cast<const T*>(P.qkv) + b * P.batch_stride + t * P.token_stride;
      const int mine = there ? rows : 0;
      const int64_t step = (int64_t)P.n * D;              // from a head's row to the next head's
      // row r of the token goes to one of these plus r steps
      __half* to_q = P.q + (b * P.H * P.n + t) * D;
      __half* to_k = P.k + (b * P.Hkv * P.n + t) * D - P.H * step;
      __half* to_v = P.v + (b * P.Hkv * P.n + t) * D - (P.H + P.Hkv) * step;
      float cs[4] = {}, sn[4] = {};                       // of the lane's four pairs
      if (turns) {
        const float4* at = reinterpret_cast<const float4*>(&turn[there ? tk : 0][4 * sub]);
        const float4 u = at[0], v = at[1];
        cs[0] = u.x; sn[0] = u.y; cs[1] = u.z; sn[1] = u.w;
        cs[2] = v.x; sn[2] = v.y; cs[3] = v.z; sn[3] = v.w;
      }
      auto request = [&](int row, uint2 (&raw)[2]) {
        raw[0] = raw[1] = make_uint2(ONES, ONES);
        if (row < mine) {
          raw[0] = __ldcs(reinterpret_cast<const uint2*>(src + (int64_t)row * D + run0));
          raw[1] = __ldcs(reinterpret_cast<const uint2*>(src + (int64_t)row * D + run1));
        }
      };
      auto work_on = [&](int row, const uint2 (&raw)[2]) {
        const bool is_q = row < P.H, is_v = row >= P.H + P.Hkv;
        float x[8];
        widen<T>(raw[0], x);
        widen<T>(raw[1], x + 4);
        if (!__all_sync(0xffffffffu, is_v)) {           // a warp of value rows only lays them out
          float r = 1.f;
          if (P.norm) {
            auto mean_square = [&](float eps) {
              float ss = 0.f;
#pragma unroll
              for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
              for (int o = 1; o < LPR; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
              return fmaf(ss, 1.0f / (float)D, eps);
            };
            float mean = mean_square(P.eps);
            if constexpr (decltype(again)::value) {     // a far row near 1 by a power of two, and eps with it; one with an infinity stays as it is
              float big = sqrtf(P.eps);
#pragma unroll
              for (int e = 0; e < 8; ++e) big = fmaxf(big, fabsf(x[e]));
#pragma unroll
              for (int o = 1; o < LPR; o <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
              const int exponent = __float_as_int(big) >> 23;
              const float by = !is_v && __float_as_uint(mean) - LOW > SPAN && exponent < 255 ? __int_as_float((254 - min(max(exponent, 1), 253)) << 23) : 1.f;
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] *= by;
              mean = mean_square(P.eps * by * by);
            } else if constexpr (FAR_ROWS) {
              farthest = __viaddmax_u32(__float_as_uint(mean), 0u - LOW, farthest);
            }
            r = rsqrtf(mean);
          }
          if (!is_v) {
            float w[8];
            widen<T>(is_q ? wq[0] : wk[0], w);
            widen<T>(is_q ? wq[1] : wk[1], w + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= r * w[e];
            if (turns) {      // what does not turn keeps its value (the other feature may be infinite)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float& a = HALVES ? x[e] : x[2 * e];
                float& c = HALVES ? x[e + 4] : x[2 * e + 1];
                const float a1 = a * cs[e] - c * sn[e];
                c = fmaf(a, sn[e], c * cs[e]);
                a = a1;
              }
            }
          }
        }
        if (row < mine) {
          __half* dst = (is_q ? to_q : (is_v ? to_v : to_k)) + row * step;
          __stcs(reinterpret_cast<uint2*>(dst + run0), narrow(x));
          __stcs(reinterpret_cast<uint2*>(dst + run1), narrow(x + 4));
        }
      };
      constexpr int ROUNDS = decltype(again)::value ? 1 : AHEAD;
      for (int r0 = 0; r0 < rows; r0 += ROUNDS * PLACES) {    // ROUNDS at a time, their rows requested first
        uint2 raw[ROUNDS][2];
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) request(r0 + i * PLACES + row0, raw[i]);
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
          if (r0 + i * PLACES >= rows) break;             // the same for the whole CTA
          work_on(r0 + i * PLACES + row0, raw[i]);
        }
      }
    }
  };
  walk(std::false_type{});
  if constexpr (FAR_ROWS)
    if (__any_sync(0xffffffffu, farthest > SPAN)) walk(std::true_type{});
}

template <int D>
cudaError_t launch_dim(const QkNormParams& P, bool bf16, cudaStream_t stream) {
  const int rows = P.H + (P.v ? 2 : 1) * P.Hkv, places = THREADS / (D / 8);
  const int64_t tokens = (int64_t)P.batch * P.n;
  // as many tokens side by side as fit; several one after the other only where that leaves every SM several CTAs
  int per_cta = rows < places ? places / rows : 1;
  per_cta = per_cta > MAX_TOKENS ? MAX_TOKENS : per_cta;
  while (per_cta * 2 <= 4 && tokens >= (int64_t)per_cta * 2 * 148 * 8) per_cta *= 2;
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
