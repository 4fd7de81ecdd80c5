// The product of a dense layer kept in 4 bits.
//
//   C[m][n] = act(ra[m] rb[n] sum_k A[m][k] B[n][k] + bias[n]),  A and B codes times their blocks' scales
//
// A product of two codes is a multiple of 1/4 up to 36, so a block's sum is exact in fp32.
#include "common.cuh"
#include "fp4.cuh"
#include "internal.h"
#include "rows.cuh"

namespace oscars {

namespace {

struct Fp4Args {
  const uint8_t *A, *sa, *B, *sb;
  const float *ra, *rb, *bias;
  void* C;
  int64_t lda, ldb, ldc;
  int M, N, K, mx, tiles, relu, bf16;
};

// sum x ra x rb: NV's sums lie between 2^-20 and 2^62 (or are 0), so their products with a row scale in [2^-96, 2^64] stay
// among fp32's normal numbers and only the result can leave them.  Other row scales are taken 2^64 nearer to 1, and the result
// gets that back.
__device__ __forceinline__ float near_one(float s) { return fabsf(s) > 0x1p64f ? s * 0x1p-64f : fabsf(s) < 0x1p-96f ? s * 0x1p64f : s; }
__device__ __forceinline__ float back(float s) { return fabsf(s) > 0x1p64f ? 0x1p64f : fabsf(s) < 0x1p-96f ? 0x1p-64f : 1.f; }

__device__ __forceinline__ float finish(const Fp4Args& a, float sum, float ra, float rb, float bias) {
  float v = sum * near_one(ra) * rb * back(ra);
  if (a.bias) v += bias;
  return a.relu && v < 0.f ? 0.f : v;
}

// ------------------------------------------------------------------ any sizes
// A warp takes one channel and MT tokens, a lane 32 codes of a row a turn: its blocks' sums in fp32, times their scales.
constexpr int kFewThreads = 256;

template <int MT>
__global__ void __launch_bounds__(kFewThreads) gemm_fp4_few_kernel(const __grid_constant__ Fp4Args a) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_trigger();
  const int n = blockIdx.x * (kFewThreads / 32) + warp;
  if (n >= a.N) return;
  const int groups = (a.K + 31) / 32;
  for (int m0 = blockIdx.y * MT; m0 < a.M; m0 += gridDim.y * MT) {
    float sum[MT] = {};
    for (int g = lane; g < groups; g += 32) {
      const uint4 w = *reinterpret_cast<const uint4*>(a.B + n * a.ldb + g * 16);
      const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
      auto scales = [&](const uint8_t* s, int64_t row, float& s0, float& s1) {   // of the group's two halves
        if (a.mx) {
          s0 = s1 = e8m0_value(s[fp4_scale_at(row, g >> 2, a.tiles) + (g & 3)]);
        } else {
          const float2 f = __half22float2(e4m3_pair(*reinterpret_cast<const uint16_t*>(s + fp4_scale_at(row, g >> 1, a.tiles) + 2 * (g & 1))));
          s0 = f.x, s1 = f.y;
        }
      };
      float b0, b1;
      scales(a.sb, n, b0, b1);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if (m0 + m >= a.M) break;
        const uint4 x = *reinterpret_cast<const uint4*>(a.A + (m0 + m) * a.lda + g * 16);
        const uint32_t xx[4] = {x.x, x.y, x.z, x.w};
        float s0, s1, part[2] = {};
        scales(a.sa, m0 + m, s0, s1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t p[4], q[4];
          eight_values(ww[i], p);
          eight_values(xx[i], q);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&p[j])), v = __half22float2(*reinterpret_cast<const __half2*>(&q[j]));
            part[i >> 1] = fmaf(u.y, v.y, fmaf(u.x, v.x, part[i >> 1]));
          }
        }
        sum[m] = fmaf(part[1], s1 * b1, fmaf(part[0], s0 * b0, sum[m]));
      }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float s = sum[m];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (lane == 0 && m0 + m < a.M) {
        const float y = finish(a, s, a.ra ? a.ra[m0 + m] : 1.f, a.rb ? a.rb[n] : 1.f, a.bias ? a.bias[n] : 0.f);
        if (a.bf16) static_cast<__nv_bfloat16*>(a.C)[(m0 + m) * a.ldc + n] = __float2bfloat16_rn(y);
        else static_cast<float*>(a.C)[(m0 + m) * a.ldc + n] = y;
      }
    }
  }
}

bool at_bytes(const void* p, int n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace
}  // namespace oscars

using namespace oscars;

extern "C" {

oscars_status oscars_gemm_fp4_nt(const uint8_t* A, int64_t lda, const uint8_t* scales_a, const float* row_a, const uint8_t* B,
                                 int64_t ldb, const uint8_t* scales_b, const float* row_b, int32_t format, const float* bias,
                                 int32_t relu, void* C, int64_t ldc, int32_t dtype, int32_t M, int32_t N, int32_t K, void* stream) {
  if (M < 0 || M > kFp4MaxSide || N < 1 || N > kFp4MaxSide || K < 1 || K > kFp4MaxSide || lda % 16 || ldb % 16 || lda < fp4_row_bytes(K) ||
      ldb < fp4_row_bytes(K) || ldc < N || (format != OSCARS_MXFP4 && format != OSCARS_NVFP4) || (dtype != OSCARS_F32 && dtype != OSCARS_BF16))
    return OSCARS_EINVAL;
  if (M == 0) return OSCARS_OK;
  if (!A || !B || !C || !scales_a || !scales_b || !at_bytes(A, 16) || !at_bytes(B, 16) || !at_bytes(scales_a, 16) || !at_bytes(scales_b, 16) ||
      !at_bytes(row_a, 4) || !at_bytes(row_b, 4) || !at_bytes(bias, 4) || !at_bytes(C, dtype == OSCARS_F32 ? 4 : 2))
    return OSCARS_EINVAL;
  Fp4Args a{A, scales_a, B, scales_b, row_a, row_b, bias, C, lda, ldb, ldc, M, N, K, format == OSCARS_MXFP4, fp4_tiles(K, format), relu,
            dtype == OSCARS_BF16};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  constexpr int kPer = kFewThreads / 32;
  const dim3 grid((N + kPer - 1) / kPer, (M + 3) / 4 < 65535 ? (M + 3) / 4 : 65535);
  const cudaError_t e = launch_dependent(gemm_fp4_few_kernel<4>, grid, kFewThreads, 0, s, a);
  return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

}  // extern "C"
