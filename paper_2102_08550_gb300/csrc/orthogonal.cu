// Orthogonalised updates: Newton-Schulz steps on weight matrices, and the
// server step that merges pushed deltas, orthogonalises the result and applies
// it (the update rule of the Muon optimiser in place of the average of Eq. 4).
//
//   X = G / (|G|_F + eps);  steps times:  A = X X^T,  B = a I + b A + c A A,
//   X <- B X;  O = scale X.
//
// With s = min(rows, cols) the Gram matrix is taken on the shorter side: A = X
// X^T [rows][rows] of a wide matrix, A = X^T X [cols][cols] of a tall one, where
// X <- X B (B is a polynomial in A, so both are the same step).  No transposed
// copy is made of either.
//
// Launches: the sum of squares (with the merge of the deltas in the same pass),
// X = G / norm, then three products a step.
#include <cmath>

#include "../../include/oscars.h"
#include "common.cuh"
#include "internal.h"

namespace oscars {

namespace {

constexpr int kPasses = 256;        // threads of the streaming passes
constexpr int kMaxParts = 304;      // partial sums of squares of one matrix
constexpr int kMaxDim = 65536, kMaxBatch = 65535, kMaxSteps = 64;
constexpr float kMaxCoeff = 8.f;

struct Shape {
  int batch, rows, cols, s;         // s: the shorter side
  int64_t ldx, lds;                 // rows of X and of A, B in the workspace, in elements
  int parts;                        // partial sums a matrix
  int64_t off_part, off_u, off_x[2], off_a, off_b, bytes;
};

int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

Shape make_shape(int batch, int rows, int cols, bool with_u) {
  Shape p;
  p.batch = batch;
  p.rows = rows;
  p.cols = cols;
  p.s = rows < cols ? rows : cols;
  p.ldx = up(cols, 8);
  p.lds = up(p.s, 8);
  const int64_t elems = static_cast<int64_t>(rows) * cols;
  const int64_t parts = (elems + 8 * kPasses - 1) / (8 * kPasses);
  p.parts = static_cast<int>(parts < kMaxParts ? parts : kMaxParts);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at = up(at + bytes, 256);
    return o;
  };
  p.off_part = take(static_cast<int64_t>(batch) * p.parts * 8);
  p.off_u = with_u ? take(elems * 4) : 0;
  for (int i = 0; i < 2; ++i) p.off_x[i] = take(static_cast<int64_t>(batch) * rows * p.ldx * 4);
  p.off_a = take(static_cast<int64_t>(batch) * p.s * p.lds * 4);
  p.off_b = take(static_cast<int64_t>(batch) * p.s * p.lds * 4);
  p.bytes = at;
  return p;
}

// ------------------------------------------------------------------ streaming passes

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// 8 elements of a row; `vec`: 16-byte loads, all 8 inside
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, bool vec, float (&v)[8]) {
  if (vec && n >= 8) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(p);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}

// Sum of 8 squares.  In fp32 where neither it nor a term that counts can leave
// the range, else (magnitudes below 1e-10 or above 1e15) in fp64, so that no
// update is too small or too large for its norm.
template <int N>
__device__ __forceinline__ double squares(const float (&v)[N]) {
  float s = 0.f;
  bool any = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    s = fmaf(v[i], v[i], s);
    any |= v[i] != 0.f;
  }
  if (any && !(s > 1e-20f && s < 1e30f)) {
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) d += static_cast<double>(v[i]) * static_cast<double>(v[i]);
    return d;
  }
  return s;
}

// Sum over the block in a fixed order; the result is thread 0's.
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double part[kPasses / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
  __syncthreads();
  double s = 0.0;
  if (threadIdx.x == 0)
    for (int i = 0; i < kPasses / 32; ++i) s += part[i];
  return s;
}

// part[z][block] = sum of squares of the block's share of matrix z
template <typename T>
__global__ void __launch_bounds__(kPasses) orth_norm_kernel(const T* __restrict__ G, int64_t ldg, int64_t bsg, int rows,
                                                            int cols, int vec, double* __restrict__ part) {
  const T* g = G + blockIdx.y * bsg;
  const int per_row = (cols + 7) / 8;
  const int64_t n = static_cast<int64_t>(rows) * per_row, step = static_cast<int64_t>(gridDim.x) * kPasses;
  double sum = 0.0;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kPasses + threadIdx.x; i < n; i += step) {
    const int r = static_cast<int>(i / per_row), c = static_cast<int>(i - static_cast<int64_t>(r) * per_row) * 8;
    float v[8];
    load8(g + r * ldg + c, cols - c, vec, v);
    sum += squares(v);
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) part[blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// v <- mu v + sum_k w_k delta_k, u and the sums of squares of u
template <int V>
__global__ void __launch_bounds__(kPasses) orth_merge_kernel(const __grid_constant__ MergeArgs a, float* __restrict__ mom,
                                                             float mu, int nesterov, float* __restrict__ u, int64_t n,
                                                             double* __restrict__ part) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kPasses * V;
  double sum = 0.0;
  for (int64_t i = (static_cast<int64_t>(blockIdx.x) * kPasses + threadIdx.x) * V; i < n; i += step) {
    const bool full = i + V <= n;
    float d[V], x[V];
    auto load = [&](const float* p, float (&to)[V]) {
      if (V == 4 && full) {
        const float4 t = __ldcs(reinterpret_cast<const float4*>(p + i));
        to[0] = t.x, to[V > 1 ? 1 : 0] = t.y, to[V > 2 ? 2 : 0] = t.z, to[V > 3 ? 3 : 0] = t.w;
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) to[j] = i + j < n ? __ldcs(p + i + j) : 0.f;
      }
    };
#pragma unroll
    for (int j = 0; j < V; ++j) d[j] = 0.f;
    int k = 0;
    for (; k + 8 <= a.W; k += 8) {   // 8 loads in flight, summed in worker order
      float t[8][V];
#pragma unroll
      for (int g = 0; g < 8; ++g) load(a.src[k + g], t[g]);
#pragma unroll
      for (int g = 0; g < 8; ++g)
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] = fmaf(a.w[k + g], t[g][j], d[j]);
    }
    for (; k < a.W; ++k) {
      float t[V];
      load(a.src[k], t);
#pragma unroll
      for (int j = 0; j < V; ++j) d[j] = fmaf(a.w[k], t[j], d[j]);
    }
    if (mom) {
      load(mom, x);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float m = fmaf(mu, x[j], d[j]);
        x[j] = m;
        d[j] = nesterov ? fmaf(mu, m, d[j]) : m;
      }
      if (V == 4 && full) {
        *reinterpret_cast<float4*>(mom + i) = make_float4(x[0], x[V > 1 ? 1 : 0], x[V > 2 ? 2 : 0], x[V > 3 ? 3 : 0]);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (i + j < n) mom[i + j] = x[j];
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (i + j < n) u[i + j] = d[j];
    sum += squares(d);
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// X = G / (norm + eps), the row padding of X zero
template <typename T>
__global__ void __launch_bounds__(kPasses) orth_scale_kernel(const T* __restrict__ G, int64_t ldg, int64_t bsg, int rows,
                                                             int cols, int vec, const double* __restrict__ part, int parts,
                                                             float eps, float* __restrict__ X, int64_t ldx) {
  __shared__ float inv_s[2];
  double t = 0.0;
  for (int i = threadIdx.x; i < parts; i += kPasses) t += part[blockIdx.y * static_cast<int64_t>(parts) + i];
  t = block_sum(t);
  if (threadIdx.x == 0) {
    // 1 / (norm + eps) = power x factor, each a normal fp32 number
    int e;
    const double m = frexp(sqrt(t) + static_cast<double>(eps), &e);
    inv_s[0] = static_cast<float>(1.0 / m);
    inv_s[1] = isinf(t) ? 0.f : ldexpf(1.f, -e);
  }
  __syncthreads();
  const float f = inv_s[0], pw = inv_s[1];
  const T* g = G + blockIdx.y * bsg;
  float* x = X + blockIdx.y * rows * ldx;
  const int per_row = static_cast<int>(ldx / 8);
  const int64_t n = static_cast<int64_t>(rows) * per_row, step = static_cast<int64_t>(gridDim.x) * kPasses;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kPasses + threadIdx.x; i < n; i += step) {
    const int r = static_cast<int>(i / per_row), c = static_cast<int>(i - static_cast<int64_t>(r) * per_row) * 8;
    float v[8];
    load8(g + r * ldg + c, cols - c, vec, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[r * ldx + c + j] = (v[j] * pw) * f;
  }
}

// ------------------------------------------------------------------ products
// D[i][j] = sum_k A(i, k) B(k, j), 64 x 64 a block, 4 x 4 a thread
enum { kGram, kSquare, kStep, kLastF32, kLastBf16, kApply };
struct ProdArgs {
  const float *A, *B, *Y;            // Y: kSquare reads b Y[i][j]
  void* D;
  int64_t ai, ak, bk, bj, za, zb, zy, zd, ldy, ldd;
  int M, N, K;
  float a, b, c;                     // kSquare's coefficients; a: the scale of the last step
};

template <int EPI>
__global__ void __launch_bounds__(256) orth_product_kernel(const __grid_constant__ ProdArgs p) {
  __shared__ float sa[16][65], sb[16][65];
  const float* A = p.A + blockIdx.z * p.za;
  const float* B = p.B + blockIdx.z * p.zb;
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < p.K; k0 += 16) {
    for (int e = threadIdx.x; e < 64 * 16; e += 256) {
      // the contiguous index of each operand runs along the threads
      const int ka = p.ak == 1 ? e & 15 : e >> 6, ia = p.ak == 1 ? e >> 4 : e & 63;
      const int kb = p.bk == 1 ? e & 15 : e >> 6, jb = p.bk == 1 ? e >> 4 : e & 63;
      sa[ka][ia] = k0 + ka < p.K && m0 + ia < p.M ? A[(m0 + ia) * p.ai + (k0 + ka) * p.ak] : 0.f;
      sb[kb][jb] = k0 + kb < p.K && n0 + jb < p.N ? B[(k0 + kb) * p.bk + (n0 + jb) * p.bj] : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      float x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = sa[k][ty + 16 * i], y[i] = sb[k][tx + 16 * i];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = m0 + ty + 16 * i, c = n0 + tx + 16 * j;
      if (r >= p.M || c >= p.N) continue;
      const int64_t at = blockIdx.z * p.zd + r * p.ldd + c;
      const float v = acc[i][j];
      if (EPI == kGram || EPI == kStep) static_cast<float*>(p.D)[at] = v;
      if (EPI == kSquare)
        static_cast<float*>(p.D)[at] = fmaf(p.c, v, fmaf(p.b, p.Y[blockIdx.z * p.zy + r * p.ldy + c], r == c ? p.a : 0.f));
      if (EPI == kLastF32) static_cast<float*>(p.D)[at] = p.a * v;
      if (EPI == kLastBf16) static_cast<__nv_bfloat16*>(p.D)[at] = __float2bfloat16_rn(p.a * v);
      if (EPI == kApply) static_cast<float*>(p.D)[at] = fmaf(p.a, v, static_cast<float*>(p.D)[at]);
    }
}

template <int EPI>
cudaError_t product(const ProdArgs& p, int batch, cudaStream_t s) {
  orth_product_kernel<EPI><<<dim3((p.N + 63) / 64, (p.M + 63) / 64, batch), 256, 0, s>>>(p);
  return cudaGetLastError();
}

// where the last step's result goes
struct Target {
  void* D;
  int64_t ldd, zd;
  int epi;
  float scale;
};

int pass_blocks(int64_t units, int most) {
  const int64_t b = (units + kPasses - 1) / kPasses;
  return static_cast<int>(b < most ? b : most);
}

template <typename T>
cudaError_t steps_from(const Shape& p, uint8_t* ws, const T* G, int64_t ldg, int64_t bsg, float eps, int steps,
                       const float (&co)[3], const Target& to, cudaStream_t s) {
  float* X[2] = {reinterpret_cast<float*>(ws + p.off_x[0]), reinterpret_cast<float*>(ws + p.off_x[1])};
  float *A = reinterpret_cast<float*>(ws + p.off_a), *B = reinterpret_cast<float*>(ws + p.off_b);
  const int vec = (reinterpret_cast<uintptr_t>(G) | (ldg * sizeof(T)) | (bsg * sizeof(T))) % 16 == 0;
  orth_scale_kernel<T><<<dim3(pass_blocks(p.rows * (p.ldx / 8), 1024), p.batch), kPasses, 0, s>>>(
      G, ldg, bsg, p.rows, p.cols, vec, reinterpret_cast<const double*>(ws + p.off_part), p.parts, eps, X[0], p.ldx);
  cudaError_t e = cudaGetLastError();
  const bool tall = p.rows > p.cols;
  const int64_t zx = p.rows * p.ldx, zs = p.s * p.lds;
  for (int k = 0; k < steps && e == cudaSuccess; ++k) {
    const float* x = X[k & 1];
    ProdArgs g{};   // A = X X^T or X^T X
    g.A = g.B = x;
    g.za = g.zb = zx;
    g.D = A;
    g.zd = zs;
    g.ldd = p.lds;
    g.M = g.N = p.s;
    g.K = tall ? p.rows : p.cols;
    g.ai = g.bj = tall ? 1 : p.ldx;
    g.ak = g.bk = tall ? p.ldx : 1;
    if ((e = product<kGram>(g, p.batch, s)) != cudaSuccess) break;
    ProdArgs q{};   // B = a I + b A + c A A
    q.A = q.B = q.Y = A;
    q.za = q.zb = q.zy = q.zd = zs;
    q.D = B;
    q.ldy = q.ldd = q.ai = q.bj = p.lds;
    q.ak = q.bk = 1;
    q.M = q.N = q.K = p.s;
    q.a = co[0], q.b = co[1], q.c = co[2];
    if ((e = product<kSquare>(q, p.batch, s)) != cudaSuccess) break;
    ProdArgs u{};   // X <- B X or X B
    u.A = tall ? x : B;
    u.B = tall ? B : x;
    u.za = tall ? zx : zs;
    u.zb = tall ? zs : zx;
    u.ai = tall ? p.ldx : p.lds;
    u.ak = 1;
    u.bk = tall ? 1 : p.ldx;
    u.bj = tall ? p.lds : 1;
    u.M = p.rows;
    u.N = p.cols;
    u.K = p.s;
    if (k + 1 < steps) {
      u.D = X[(k + 1) & 1];
      u.ldd = p.ldx;
      u.zd = zx;
      e = product<kStep>(u, p.batch, s);
    } else {
      u.D = to.D;
      u.ldd = to.ldd;
      u.zd = to.zd;
      u.a = to.scale;
      e = to.epi == kApply ? product<kApply>(u, p.batch, s)
          : to.epi == kLastBf16 ? product<kLastBf16>(u, p.batch, s) : product<kLastF32>(u, p.batch, s);
    }
  }
  return e;
}

bool sizes_ok(int32_t batch, int32_t rows, int32_t cols) {
  return batch >= 0 && batch <= kMaxBatch && rows >= 1 && rows <= kMaxDim && cols >= 1 && cols <= kMaxDim;
}

bool settings_ok(int32_t steps, const float* coeff, float eps, float scale, float (&co)[3]) {
  const float muon[3] = {3.4445f, -4.7750f, 2.0315f};
  for (int i = 0; i < 3; ++i) {
    co[i] = coeff ? coeff[i] : muon[i];
    if (!(std::fabs(co[i]) <= kMaxCoeff)) return false;
  }
  return steps >= 1 && steps <= kMaxSteps && eps > 0.f && std::isfinite(eps) && std::isfinite(scale);
}

bool workspace_ok(const void* ws, int64_t have, int64_t need) {
  return ws && (reinterpret_cast<uintptr_t>(ws) & 255) == 0 && have >= need;
}

template <typename T>
oscars_status orthogonalize(const Shape& p, const void* G, int64_t ldg, int64_t bsg, uint8_t* ws, int steps,
                            const float (&co)[3], float eps, const Target& to, cudaStream_t s) {
  const T* g = static_cast<const T*>(G);
  const int vec = (reinterpret_cast<uintptr_t>(g) | (ldg * sizeof(T)) | (bsg * sizeof(T))) % 16 == 0;
  orth_norm_kernel<T><<<dim3(p.parts, p.batch), kPasses, 0, s>>>(g, ldg, bsg, p.rows, p.cols, vec,
                                                                 reinterpret_cast<double*>(ws + p.off_part));
  if (cudaGetLastError() != cudaSuccess) return OSCARS_ECUDA;
  return steps_from(p, ws, g, ldg, bsg, eps, steps, co, to, s) == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

}  // namespace
}  // namespace oscars

using namespace oscars;

extern "C" {

oscars_status oscars_orthogonalize_workspace(int32_t batch, int32_t rows, int32_t cols, int32_t dtype,
                                             int64_t* bytes) {
  if (!bytes || !sizes_ok(batch, rows, cols) || (dtype != OSCARS_F32 && dtype != OSCARS_BF16)) return OSCARS_EINVAL;
  *bytes = make_shape(batch, rows, cols, false).bytes;
  return OSCARS_OK;
}

oscars_status oscars_orthogonalize(const void* G, int64_t ldg, int64_t batch_stride_g, void* O, int64_t ldo,
                                   int64_t batch_stride_o, int32_t batch, int32_t rows, int32_t cols, int32_t dtype,
                                   int32_t steps, const float* coeff, float eps, float scale, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
  float co[3];
  if (!sizes_ok(batch, rows, cols) || !settings_ok(steps, coeff, eps, scale, co)) return OSCARS_EINVAL;
  if (dtype != OSCARS_F32 && dtype != OSCARS_BF16) return OSCARS_EINVAL;
  if (ldg < cols || ldo < cols || batch_stride_g < 0) return OSCARS_EINVAL;
  if (batch > 1 && batch_stride_o < (rows - 1) * ldo + cols) return OSCARS_EINVAL;
  if (batch == 0) return OSCARS_OK;
  const uintptr_t size = dtype == OSCARS_F32 ? 4 : 2;
  if (!G || !O || (reinterpret_cast<uintptr_t>(G) | reinterpret_cast<uintptr_t>(O)) % size) return OSCARS_EINVAL;
  const Shape p = make_shape(batch, rows, cols, false);
  if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return OSCARS_EINVAL;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const Target to{O, ldo, batch_stride_o, dtype == OSCARS_F32 ? kLastF32 : kLastBf16, scale};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == OSCARS_F32)
    return orthogonalize<float>(p, G, ldg, batch_stride_g, ws, steps, co, eps, to, s);
  return orthogonalize<__nv_bfloat16>(p, G, ldg, batch_stride_g, ws, steps, co, eps, to, s);
}

oscars_status oscars_merge_orthogonal_workspace(int32_t rows, int32_t cols, int64_t* bytes) {
  if (!bytes || !sizes_ok(1, rows, cols)) return OSCARS_EINVAL;
  *bytes = make_shape(1, rows, cols, true).bytes;
  return OSCARS_OK;
}

oscars_status oscars_merge_orthogonal(float* x_g, const float* const* deltas, const float* w, int32_t W, int32_t rows,
                                      int32_t cols, float* momentum, float mu, int32_t nesterov, float server_lr,
                                      int32_t steps, const float* coeff, float eps, void* workspace,
                                      int64_t workspace_bytes, void* stream) {
  float co[3];
  if (!sizes_ok(1, rows, cols) || !settings_ok(steps, coeff, eps, server_lr, co)) return OSCARS_EINVAL;
  if (!x_g || !deltas || !w || W < 1 || W > kMaxMergeWorkers) return OSCARS_EINVAL;
  if (momentum ? !std::isfinite(mu) : nesterov != 0) return OSCARS_EINVAL;
  MergeArgs a;
  a.W = W;
  uintptr_t bits = reinterpret_cast<uintptr_t>(momentum);
  for (int k = 0; k < W; ++k) {
    if (!deltas[k]) return OSCARS_EINVAL;
    a.src[k] = deltas[k];
    a.w[k] = w[k];
    bits |= reinterpret_cast<uintptr_t>(deltas[k]);
  }
  if ((bits | reinterpret_cast<uintptr_t>(x_g)) & 3) return OSCARS_EINVAL;
  const Shape p = make_shape(1, rows, cols, true);
  if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return OSCARS_EINVAL;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  float* u = reinterpret_cast<float*>(ws + p.off_u);
  double* part = reinterpret_cast<double*>(ws + p.off_part);
  const int64_t n = static_cast<int64_t>(rows) * cols;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((bits & 15) == 0) orth_merge_kernel<4><<<p.parts, kPasses, 0, s>>>(a, momentum, mu, nesterov != 0, u, n, part);
  else orth_merge_kernel<1><<<p.parts, kPasses, 0, s>>>(a, momentum, mu, nesterov != 0, u, n, part);
  if (cudaGetLastError() != cudaSuccess) return OSCARS_ECUDA;
  const Target to{x_g, cols, 0, kApply, server_lr};
  return steps_from(p, ws, static_cast<const float*>(u), cols, 0, eps, steps, co, to, s) == cudaSuccess ? OSCARS_OK
                                                                                                       : OSCARS_ECUDA;
}

}  // extern "C"
