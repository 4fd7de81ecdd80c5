// Orthogonalised updates: Newton-Schulz steps on weight matrices, and the
// server step that merges pushed deltas, orthogonalises the result and applies
// it (the update rule of the Muon optimiser in place of the average of Eq. 4).
//
//   X = G / (|G|_F + eps);  steps times:  A = X X^T,  B = a I + b A + c A A
//   (as c (A + beta I)^2 + gamma I, or a I + b A where c = 0),
//   X <- B X;  O = scale X.
//
// With s = min(rows, cols) the Gram matrix is taken on the shorter side: A = X
// X^T [rows][rows] of a wide matrix, A = X^T X [cols][cols] of a tall one, where
// X <- X B (B is a polynomial in A, so both are the same step).  No transposed
// copy is made of either.
//
// Small matrices: one launch (orth_small.cu).  Others: the sum of squares (with the merge of the deltas in the same pass),
// X = G / norm, then three products a step, two where c = 0 (orth_product.cu, where the precision
// of X, A and B is explained).
#include <cmath>

#include "../../include/oscars.h"
#include "common.cuh"
#include "internal.h"
#include "rows.cuh"

namespace oscars {

namespace {

constexpr int kPasses = 256;        // threads of the streaming passes
constexpr int kMaxParts = 608;      // partial sums of squares of one matrix
constexpr int kAhead = 4;           // groups of eight elements that a thread of a pass requests together
constexpr int kMaxDim = 65536, kMaxBatch = 65535, kMaxSteps = 64;
constexpr int kFewSteps = 5, kCoarse = 3;   // a bf16 result's steps that take one half of A and B (orth_product.cu)
constexpr float kMaxCoeff = 8.f;

struct Shape {
  int batch, rows, cols, s;         // s: the shorter side
  int small;                        // CTAs a matrix of the one launch, or 0: products on the tensor cores
  int64_t ldx, lds;                 // rows of X and of A, B in the workspace, in elements
  int parts;                        // partial sums a matrix
  int64_t off_status, off_part, off_u, off_cut, off_x[2], off_a, off_b, bytes;
};

int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

Shape make_shape(int batch, int rows, int cols, int dtype, bool with_u) {
  Shape p{};
  p.batch = batch;
  p.rows = rows;
  p.cols = cols;
  p.s = rows < cols ? rows : cols;
  p.small = ns_small_cluster(batch, rows, cols, dtype == OSCARS_F32);
  // rows on 128-byte lines: a box's row of 128 bytes is one line then, not two (server step on 1537 x 385: 156 -> 146 us)
  p.ldx = up(cols, 64);
  p.lds = up(p.s, 64);
  const int64_t elems = static_cast<int64_t>(rows) * cols;
  const int64_t each = (with_u ? 4 : 8 * kAhead) * kPasses, parts = (elems + each - 1) / each;   // a block's share, at least
  p.parts = static_cast<int>(parts < kMaxParts ? parts : kMaxParts);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at = up(at + bytes, 256);
    return o;
  };
  p.off_status = take(sizeof(int));   // first, where the caller finds it
  if (!p.small || with_u) p.off_part = take(static_cast<int64_t>(batch) * p.parts * sizeof(Squares));
  p.off_u = with_u ? take(elems * 4) : 0;
  if (!p.small) {   // one launch keeps a matrix in shared memory
    // X, A and B in two fp16 halves each
    for (int i = 0; i < 2; ++i) p.off_x[i] = take(static_cast<int64_t>(batch) * rows * p.ldx * 4);
    if (dtype != OSCARS_F32) p.off_cut = take(static_cast<int64_t>(batch) * p.s * sizeof(float));
    p.off_a = take(static_cast<int64_t>(batch) * p.s * p.lds * 4);
    p.off_b = take(static_cast<int64_t>(batch) * p.s * p.lds * 4);
  }
  p.bytes = at;
  return p;
}

// ------------------------------------------------------------------ streaming passes

// part[z][block] = sum of squares of the block's share of matrix z
template <typename T>
__global__ void __launch_bounds__(kPasses) orth_norm_kernel(const T* __restrict__ G, int64_t ldg, int64_t bsg, int rows,
                                                            int cols, int vec, Squares* __restrict__ part, int* __restrict__ status) {
  __shared__ Squares warps[kPasses / 32];
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *status = kDevOk;
  const T* g = G + blockIdx.y * bsg;
  // groups of eight: at most 2^29 (a 64-bit division for each took longer than its bytes)
  const uint32_t per_row = (cols + 7) / 8, n = rows * per_row, step = gridDim.x * kPasses;
  Squares sum;
  for (uint32_t i0 = blockIdx.x * kPasses + threadIdx.x; i0 < n; i0 += kAhead * step) {
    Held8<T> h[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const uint32_t i = i0 + e * step, r = i / per_row, c = (i - r * per_row) * 8;
      h[e].load(g + static_cast<int64_t>(r) * ldg + c, i < n ? cols - static_cast<int>(c) : 0, vec);
    }
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      float v[8];
      h[e].get(v);
      sum.add(v);
    }
  }
  sum.block_sum(warps);
  if (threadIdx.x == 0) part[blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// v <- mu v + sum_k w_k delta_k, u and the sums of squares of u
template <int V>
__global__ void __launch_bounds__(kPasses) orth_merge_kernel(const __grid_constant__ MergeArgs a, float* __restrict__ mom,
                                                             float mu, int nesterov, float* __restrict__ u, int64_t n,
                                                             Squares* __restrict__ part, int* __restrict__ status) {
  __shared__ Squares warps[kPasses / 32];
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = kDevOk;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kPasses * V;
  Squares sum;
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
    sum.add(d);
  }
  sum.block_sum(warps);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// X = G / (norm + eps) as two fp16 halves, [half][z][rows][ldx], the row padding zero
template <typename T>
__global__ void __launch_bounds__(kPasses) orth_scale_kernel(const T* __restrict__ G, int64_t ldg, int64_t bsg, int rows,
                                                             int cols, int vec, const Squares* __restrict__ part, int parts,
                                                             float eps, float second_scale, __half* __restrict__ X, int64_t ldx) {
  __shared__ float inv_s[2];
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x < 32) {   // one warp adds up the parts: blocks' sums may leave fp32's range together, so in fp64
    double t = 0.0;
    for (int i = threadIdx.x; i < parts; i += 32) t += part[blockIdx.y * static_cast<int64_t>(parts) + i].total();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if (threadIdx.x == 0) inverse_norm(t, eps, inv_s[1], inv_s[0]);
  }
  __syncthreads();
  const float f = inv_s[0], pw = inv_s[1];
  const T* g = G + blockIdx.y * bsg;
  __half* x = X + blockIdx.y * rows * ldx;
  const int64_t second = static_cast<int64_t>(gridDim.y) * rows * ldx;
  const uint32_t per_row = static_cast<uint32_t>(ldx / 8), n = rows * per_row, step = gridDim.x * kPasses;
  for (uint32_t i0 = blockIdx.x * kPasses + threadIdx.x; i0 < n; i0 += kAhead * step) {
    Held8<T> held[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const uint32_t i = i0 + e * step, r = i / per_row, c = (i - r * per_row) * 8;
      held[e].load(g + static_cast<int64_t>(r) * ldg + c, i < n ? cols - static_cast<int>(c) : 0, vec);
    }
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const uint32_t i = i0 + e * step;
      if (i >= n) break;
      float v[8];
      held[e].get(v);
      __align__(16) __half hi[8], lo[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = ((v[j] * pw) * f) * kNsScaleX;
        hi[j] = __float2half_rn(y);
        lo[j] = __float2half_rn((y - __half2float(hi[j])) * second_scale);
      }
      // rows of X are as long as their groups, so group i lies at 8 i
      *reinterpret_cast<uint4*>(x + 8 * static_cast<int64_t>(i)) = *reinterpret_cast<const uint4*>(hi);
      *reinterpret_cast<uint4*>(x + second + 8 * static_cast<int64_t>(i)) = *reinterpret_cast<const uint4*>(lo);
    }
  }
}

// where the last step's result goes
struct Target {
  void* D;
  int64_t ldd, zd;
  int type;                         // NsOut
  float scale;
};

// fp16 [halves][batch][rows][ld]
bool half_maps(NsMaps* m, const void* base, int64_t ld, int cols, int rows, int batch, int halves) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows),
                              static_cast<cuuint64_t>(batch) * halves};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(ld) * rows * 2};
  const cuuint32_t b64[3] = {64, 64, 1}, b128[3] = {64, 128, 1}, out[3] = {32, 32, 1};
  const CUtensorMapDataType t = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return encode_map(&m->load64, t, 3, base, dims, strides, b64, CU_TENSOR_MAP_SWIZZLE_128B) &&
         encode_map(&m->load128, t, 3, base, dims, strides, b128, CU_TENSOR_MAP_SWIZZLE_128B) &&
         encode_map(&m->store, t, 3, base, dims, strides, out, CU_TENSOR_MAP_SWIZZLE_64B);
}

int pass_blocks(int64_t units, int most) {
  const int64_t b = (units + kPasses - 1) / kPasses;
  return static_cast<int>(b < most ? b : most);
}

template <typename T>
cudaError_t steps_from(const Shape& p, uint8_t* ws, const T* G, int64_t ldg, int64_t bsg, float eps, int steps,
                       const float (&co)[3], const Target& to, cudaStream_t s) {
  __half* X[2] = {reinterpret_cast<__half*>(ws + p.off_x[0]), reinterpret_cast<__half*>(ws + p.off_x[1])};
  __half *A = reinterpret_cast<__half*>(ws + p.off_a), *B = reinterpret_cast<__half*>(ws + p.off_b);
  NsMaps mX[2], mA, mB;
  for (int i = 0; i < 2; ++i)
    if (!half_maps(&mX[i], X[i], p.ldx, p.cols, p.rows, p.batch, 2)) return cudaErrorInvalidValue;
  if (!half_maps(&mA, A, p.lds, p.s, p.s, p.batch, 2) || !half_maps(&mB, B, p.lds, p.s, p.s, p.batch, 2))
    return cudaErrorInvalidValue;
  const int vec = (reinterpret_cast<uintptr_t>(G) | (ldg * sizeof(T)) | (bsg * sizeof(T))) % 16 == 0;
  constexpr bool kF32 = sizeof(T) == 4;
  auto halves = [&](int k) { return kF32 || (steps > kFewSteps && steps - k > kCoarse) ? 2 : 1; };   // of A and B in step k
  auto second = [&](int k) { return halves(k) == 2 ? static_cast<float>(1 << kNsShift) : 1.f; };
  cudaError_t e = launch_dependent(orth_scale_kernel<T>, dim3(pass_blocks((p.rows * (p.ldx / 8) + kAhead - 1) / kAhead, 608), p.batch), kPasses, 0, s,
                                   G, ldg, bsg, p.rows, p.cols, vec, reinterpret_cast<const Squares*>(ws + p.off_part), p.parts,
                                   eps, second(0), X[0], p.ldx);
  const bool tall = p.rows > p.cols;
  const bool cubic = co[2] == 0.f;
  NsArgs g{};   // A + beta I, or B itself where c = 0
  g.status = reinterpret_cast<int*>(ws + p.off_status);
  g.batch = p.batch;
  g.M = g.N = p.s;
  g.K = tall ? p.rows : p.cols;
  g.a_halves = g.b_halves = kF32 ? 2 : 1;
  g.a_mn = g.b_mn = tall;
  g.factor = (kF32 ? kNsWhole : 1.f) * (kNsScaleA / (kNsScaleX * kNsScaleX)) * (cubic ? co[1] : 1.f);
  g.diag = (cubic ? co[0] : static_cast<float>(0.5 * co[1] / co[2])) * kNsScaleA;
  NsArgs q = g;   // B = c (A + beta I)^2 + gamma I
  q.K = p.s;
  q.a_mn = q.b_mn = 0;
  q.diag = static_cast<float>(co[0] - 0.25 * co[1] * co[1] / co[2]) * kNsScaleA;
  NsArgs u{};   // X <- B X or X B
  u.status = g.status;
  u.batch = p.batch;
  u.M = p.rows;
  u.N = p.cols;
  u.K = p.s;
  u.b_mn = !tall;
  u.scale = to.scale;
  u.out = to.D;
  u.ldo = to.ldd;
  u.zo = to.zd;
  u.out_type = to.type;
  for (int k = 0; k < steps && e == cudaSuccess; ++k) {
    const NsMaps& x = mX[k & 1];
    const bool end = k + 1 == steps;
    const int h = halves(k);
    const float whole = h == 2 ? kNsWhole : 1.f;   // what the accumulator cuts off (orth_product.cu)
    g.d_halves = q.d_halves = q.a_halves = q.b_halves = h;
    g.cut = h == 1 && !cubic ? reinterpret_cast<float*>(ws + p.off_cut) : nullptr;
    q.add = g.cut;
    q.factor = whole * (co[2] / kNsScaleA);
    // The step before a bf16 result's last one leaves X in one half, and the last step takes that: its rounding is multiplied
    // by a once (3.4 x 2^-12), where an earlier one would be by a to the number of steps left.
    const int xh = end && !kF32 ? 1 : 2;
    u.a_halves = tall ? xh : h;
    u.b_halves = tall ? h : xh;
    u.d_halves = k + 2 == steps && !kF32 ? 1 : 2;
    u.d_second = second(k + 1);
    u.factor = whole / kNsScaleA * (end ? 1.f / kNsScaleX : 1.f);
    e = launch_ns_product(kNsSym, x, x, cubic ? mB : mA, g, s);
    if (e == cudaSuccess && !cubic) e = launch_ns_product(kNsSym, mA, mA, mB, q, s);
    if (e == cudaSuccess) e = launch_ns_product(end ? kNsLast : kNsStep, tall ? x : mB, tall ? mB : x, mX[(k + 1) & 1], u, s);
  }
  return e;
}

bool sizes_ok(int32_t batch, int32_t rows, int32_t cols) {
  if (batch < 0 || batch > kMaxBatch || rows < 1 || rows > kMaxDim || cols < 1 || cols > kMaxDim) return false;
  // tiles of 128 x 64 (the smallest) in clusters of four are counted in 32 bits; more take some 2^44 bytes of workspace
  return static_cast<int64_t>(batch) * ((rows + 127) / 128) * ((cols + 63) / 64) <= INT32_MAX / 4;
}

bool settings_ok(int32_t steps, const float* coeff, float eps, float scale, float (&co)[3]) {
  const float muon[3] = {3.4445f, -4.7750f, 2.0315f};
  for (int i = 0; i < 3; ++i) {
    co[i] = coeff ? coeff[i] : muon[i];
    if (!(std::fabs(co[i]) <= kMaxCoeff)) return false;
  }
  // (A + beta I)^2 must not lose what it adds up to: c beta^2 = b^2 / 4c
  if (co[2] != 0.f && !(co[1] * co[1] <= 32.f * std::fabs(co[2]) && std::fabs(co[1]) <= 64.f * std::fabs(co[2]))) return false;
  return steps >= 1 && steps <= kMaxSteps && eps > 0.f && std::isfinite(eps) && std::isfinite(scale);
}

bool workspace_ok(const void* ws, int64_t have, int64_t need) {
  return ws && (reinterpret_cast<uintptr_t>(ws) & 255) == 0 && have >= need;
}

template <typename T>
oscars_status orthogonalize(const Shape& p, const void* G, int64_t ldg, int64_t bsg, uint8_t* ws, int steps,
                            const float (&co)[3], float eps, const Target& to, cudaStream_t s) {
  const T* g = static_cast<const T*>(G);
  if (p.small)
    return launch_ns_small(G, ldg, bsg, sizeof(T) == 2, to.D, to.ldd, to.zd, to.type, p.batch, p.rows, p.cols, p.small, steps, co, eps,
                           to.scale, reinterpret_cast<int*>(ws + p.off_status), s) == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
  const int vec = (reinterpret_cast<uintptr_t>(g) | (ldg * sizeof(T)) | (bsg * sizeof(T))) % 16 == 0;
  if (launch_dependent(orth_norm_kernel<T>, dim3(p.parts, p.batch), kPasses, 0, s, g, ldg, bsg, p.rows, p.cols, vec,
                       reinterpret_cast<Squares*>(ws + p.off_part), reinterpret_cast<int*>(ws + p.off_status)) != cudaSuccess)
    return OSCARS_ECUDA;
  return steps_from(p, ws, g, ldg, bsg, eps, steps, co, to, s) == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

}  // namespace
}  // namespace oscars

using namespace oscars;

extern "C" {

oscars_status oscars_orthogonalize_workspace(int32_t batch, int32_t rows, int32_t cols, int32_t dtype,
                                             int64_t* bytes) {
  if (!bytes || !sizes_ok(batch, rows, cols) || (dtype != OSCARS_F32 && dtype != OSCARS_BF16)) return OSCARS_EINVAL;
  *bytes = make_shape(batch, rows, cols, dtype, false).bytes;
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
  const Shape p = make_shape(batch, rows, cols, dtype, false);
  if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return OSCARS_EINVAL;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const Target to{O, ldo, batch_stride_o, dtype == OSCARS_F32 ? kNsF32 : kNsBf16, scale};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == OSCARS_F32)
    return orthogonalize<float>(p, G, ldg, batch_stride_g, ws, steps, co, eps, to, s);
  return orthogonalize<__nv_bfloat16>(p, G, ldg, batch_stride_g, ws, steps, co, eps, to, s);
}

oscars_status oscars_merge_orthogonal_workspace(int32_t rows, int32_t cols, int64_t* bytes) {
  if (!bytes || !sizes_ok(1, rows, cols)) return OSCARS_EINVAL;
  *bytes = make_shape(1, rows, cols, OSCARS_F32, true).bytes;
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
  const Shape p = make_shape(1, rows, cols, OSCARS_F32, true);
  if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return OSCARS_EINVAL;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  float* u = reinterpret_cast<float*>(ws + p.off_u);
  Squares* part = reinterpret_cast<Squares*>(ws + p.off_part);
  const int64_t n = static_cast<int64_t>(rows) * cols;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_dependent((bits & 15) == 0 ? orth_merge_kernel<4> : orth_merge_kernel<1>, dim3(p.parts), kPasses, 0, s, a, momentum,
                       mu, nesterov != 0 ? 1 : 0, u, n, part, reinterpret_cast<int*>(ws + p.off_status)) != cudaSuccess)
    return OSCARS_ECUDA;
  const Target to{x_g, cols, 0, kNsAdd, server_lr};
  if (p.small)
    return launch_ns_small(u, cols, 0, false, to.D, to.ldd, to.zd, to.type, 1, rows, cols, p.small, steps, co, eps, to.scale, nullptr,
                           s) == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
  return steps_from(p, ws, static_cast<const float*>(u), cols, 0, eps, steps, co, to, s) == cudaSuccess ? OSCARS_OK
                                                                                                       : OSCARS_ECUDA;
}

}  // extern "C"
