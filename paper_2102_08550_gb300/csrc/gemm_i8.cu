// The product of a dense layer kept in 8 bits, and the rows' quantisation.
//
//   C[m][n] = act(sa[m] sb[n] sum_k A[m][k] B[n][k] + bias[n]),  the sum in int32
//   scale[i] = max_j |x[i][j]| / 127,  q[i][j] = rint(x[i][j] / scale[i])
#include "../../include/oscars.h"
#include "common.cuh"
#include "internal.h"

namespace oscars {

namespace {

constexpr int kMaxK = 131071;   // 2^14 (2^17 - 1) < 2^31

// ------------------------------------------------------------------ quantisation
// one block a row: the maximum (NaN wins), then the codes
template <typename T>
__global__ void __launch_bounds__(256) quantize_i8_kernel(const T* __restrict__ x, int64_t ldx, int cols, int8_t* __restrict__ q,
                                                          int64_t ldq, float* __restrict__ scale) {
  __shared__ float part[8];
  const T* row = x + blockIdx.x * ldx;
  int8_t* out = q + blockIdx.x * ldq;
  float mx = 0.f;
  for (int j = threadIdx.x; j < cols; j += 256) {
    const float v = fabsf(static_cast<float>(row[j]));
    mx = v > mx || v != v ? v : mx;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float v = __shfl_xor_sync(0xffffffffu, mx, o);
    mx = v > mx || v != v ? v : mx;
  }
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = mx;
  __syncthreads();
  mx = part[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) mx = part[i] > mx || part[i] != part[i] ? part[i] : mx;
  const float s = mx / 127.f;
  if (threadIdx.x == 0) scale[blockIdx.x] = s;
  const bool codes = s > 0.f && s <= 3.4e38f;
  for (int j = threadIdx.x; j < cols; j += 256) {
    const float v = codes ? fminf(fmaxf(rintf(static_cast<float>(row[j]) / s), -127.f), 127.f) : 0.f;
    out[j] = static_cast<int8_t>(v);
  }
}

// ------------------------------------------------------------------ product
struct I8Args {
  const int8_t *A, *B;
  const float *sa, *sb, *bias;
  void* C;
  int64_t lda, ldb, ldc;
  int M, N, K, relu;
};

// four codes of a row from column k on, zero past column K
__device__ __forceinline__ int codes4(const int8_t* row, int k, int K) {
  const int v = *reinterpret_cast<const int*>(row + k);
  return K - k >= 4 ? v : v & ((1 << (8 * (K - k))) - 1);
}

// 64 x 64 a block, 4 x 4 a thread
template <typename T>
__global__ void __launch_bounds__(256) gemm_i8_kernel(const __grid_constant__ I8Args p) {
  __shared__ int sa[16][65], sb[16][65];
  const int m0 = blockIdx.x * 64, n0 = blockIdx.y * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  int acc[4][4] = {};
  for (int k0 = 0; k0 < p.K; k0 += 64) {
    for (int e = threadIdx.x; e < 64 * 16; e += 256) {
      const int kq = e & 15, i = e >> 4, k = k0 + 4 * kq;
      sa[kq][i] = k < p.K && m0 + i < p.M ? codes4(p.A + (m0 + i) * p.lda, k, p.K) : 0;
      sb[kq][i] = k < p.K && n0 + i < p.N ? codes4(p.B + (n0 + i) * p.ldb, k, p.K) : 0;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(sa[k][ty + 16 * i], sb[k][tx + 16 * j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
      if (m >= p.M || n >= p.N) continue;
      float v = static_cast<float>(acc[i][j]) * p.sa[m] * p.sb[n];
      if (p.bias) v += p.bias[n];
      if (p.relu) v = v < 0.f ? 0.f : v;
      static_cast<T*>(p.C)[m * p.ldc + n] = static_cast<T>(v);
    }
}

}  // namespace
}  // namespace oscars

using namespace oscars;

extern "C" {

oscars_status oscars_quantize_i8(const void* x, int64_t ldx, int32_t dtype, int32_t rows, int32_t cols, int8_t* q,
                                 int64_t ldq, float* scale, void* stream) {
  if (rows < 0 || cols < 1 || ldx < cols || ldq < cols || (dtype != OSCARS_F32 && dtype != OSCARS_BF16))
    return OSCARS_EINVAL;
  if (rows == 0) return OSCARS_OK;
  if (!x || !q || !scale || (reinterpret_cast<uintptr_t>(scale) & 3) ||
      (reinterpret_cast<uintptr_t>(x) & (dtype == OSCARS_F32 ? 3 : 1)))
    return OSCARS_EINVAL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == OSCARS_F32)
    quantize_i8_kernel<float><<<rows, 256, 0, s>>>(static_cast<const float*>(x), ldx, cols, q, ldq, scale);
  else
    quantize_i8_kernel<__nv_bfloat16><<<rows, 256, 0, s>>>(static_cast<const __nv_bfloat16*>(x), ldx, cols, q, ldq, scale);
  return cudaGetLastError() == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

oscars_status oscars_gemm_i8_nt(const int8_t* A, int64_t lda, const float* scale_a, const int8_t* B, int64_t ldb,
                                const float* scale_b, const float* bias, int32_t relu, void* C, int64_t ldc,
                                int32_t dtype, int32_t M, int32_t N, int32_t K, void* stream) {
  if (M < 0 || N < 1 || K < 1 || K > kMaxK || lda < K || ldb < K || lda % 16 || ldb % 16 || ldc < N ||
      (dtype != OSCARS_F32 && dtype != OSCARS_BF16))
    return OSCARS_EINVAL;
  if (M == 0) return OSCARS_OK;
  if (!A || !B || !C || !scale_a || !scale_b) return OSCARS_EINVAL;
  if ((reinterpret_cast<uintptr_t>(A) | reinterpret_cast<uintptr_t>(B)) & 15) return OSCARS_EINVAL;
  if ((reinterpret_cast<uintptr_t>(scale_a) | reinterpret_cast<uintptr_t>(scale_b) | reinterpret_cast<uintptr_t>(bias)) & 3)
    return OSCARS_EINVAL;
  if (reinterpret_cast<uintptr_t>(C) & (dtype == OSCARS_F32 ? 3 : 1)) return OSCARS_EINVAL;
  const I8Args p{A, B, scale_a, scale_b, bias, C, lda, ldb, ldc, M, N, K, relu};
  const dim3 grid((M + 63) / 64, (N + 63) / 64);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == OSCARS_F32) gemm_i8_kernel<float><<<grid, 256, 0, s>>>(p);
  else gemm_i8_kernel<__nv_bfloat16><<<grid, 256, 0, s>>>(p);
  return cudaGetLastError() == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

}  // extern "C"
