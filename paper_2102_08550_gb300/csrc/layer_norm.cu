// Layer norm, forward and backward, of groups of rows with parameters of their own.
//
//   y = (x - mean) rstd gamma + beta,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   dx = rstd (h - mean(h) - xh mean(h xh)),  h = dy gamma,  xh = (x - mean) rstd
//   dgamma = sum over the group's rows of dy xh,  dbeta = sum of dy
//
// Bound by memory: forward reads x and writes y, backward reads dy and x and writes dx.
#include "../../include/oscars.h"
#include "common.cuh"
#include "internal.h"
#include "rows.cuh"

namespace oscars {

namespace {

constexpr int kMaxSide = 1 << 30, kMaxGroups = 65535;
constexpr int kThreads = 256, kKeep = 4;

// the sum of a value over the TPR threads of a row, in each of them, in a fixed order (a barrier of the row's threads
// alone: rows of one block may differ in how many sums they take)
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (TPR > 32) {
    const int r = threadIdx.x / TPR;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    bar_named(1 + r, TPR);
    v = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) v += part[r * (TPR / 32) + i];
    bar_named(1 + r, TPR);
  }
  return v;
}

// 8 of a row's parameters, or ones (or zeros) if there are none
__device__ __forceinline__ void params8(const float* p, int at, int cols, bool vec, float none, float (&v)[8]) {
  if (p) {
    load8(p + at, cols - at, vec, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = none;
  }
}

// ------------------------------------------------------------------ forward
struct FwdArgs {
  const void* x;
  void* y;
  const float *gamma, *beta;
  float *mean, *rstd;
  int64_t ldx, ldy, pstride, total;   // total: rows of all groups
  int rows, cols;
  float eps;
  int xvec, yvec, pvec;
};

// Sum of squares in the whole range of fp32 only where the plain one left it.
__device__ __forceinline__ float inverse_std(const Squares& s, int cols, float eps) {
  if (s.big == 0.f && s.small == 0.f) return 1.f / sqrtf(s.mid / cols + eps);
  return static_cast<float>(1.0 / sqrt(s.total() / cols + eps));
}

template <typename T, int TPR>
__global__ void __launch_bounds__(kThreads) layer_norm_kernel(const __grid_constant__ FwdArgs a) {
  __shared__ float part[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / TPR) + threadIdx.x / TPR;
  const int t = threadIdx.x % TPR, turns = (a.cols + TPR * 8 - 1) / (TPR * 8);
  if (TPR == 32 && row >= a.total) return;
  const bool live = row < a.total;
  const T* x = static_cast<const T*>(a.x) + (live ? row : 0) * a.ldx;
  Held8<T> held[kKeep];
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kKeep; ++i) held[i].load(x + (i * TPR + t) * 8, a.cols - (i * TPR + t) * 8, a.xvec);
  auto each = [&](auto&& f) {   // f(first column, its 8 values), zeros behind the row's end
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
      if ((i * TPR + t) * 8 < a.cols) {
        float v[8];
        held[i].get(v);
        f((i * TPR + t) * 8, v);
      }
    for (int i = kKeep; i < turns; ++i) {
      const int at = (i * TPR + t) * 8;
      if (at >= a.cols) break;
      float v[8];
      load8(x + at, a.cols - at, a.xvec, v);
      f(at, v);
    }
  };
  each([&](int, float (&v)[8]) { sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); });
  sum = row_sum<TPR>(sum, part);
  float mean = sum / a.cols;
  if (!(fabsf(sum) < INFINITY)) {   // the sum may have left fp32 where the mean does not
    sum = 0.f;
    each([&](int, float (&v)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += v[e] * 0x1p-32f;
    });
    sum = row_sum<TPR>(sum, part);
    mean = sum / a.cols * 0x1p32f;
  }
  Squares sq;
  each([&](int at, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = at + e < a.cols ? v[e] - mean : 0.f;
    sq.add(v);
  });
  sq.mid = row_sum<TPR>(sq.mid, part);
  sq.big = row_sum<TPR>(sq.big, part);
  sq.small = row_sum<TPR>(sq.small, part);
  if (!live) return;
  const float rstd = inverse_std(sq, a.cols, a.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  const int64_t group = row / a.rows;
  const float *gamma = a.gamma ? a.gamma + group * a.pstride : nullptr, *beta = a.beta ? a.beta + group * a.pstride : nullptr;
  T* y = static_cast<T*>(a.y) + row * a.ldy;
  each([&](int at, float (&v)[8]) {
    float g[8], b[8];
    params8(gamma, at, a.cols, a.pvec, 1.f, g);
    params8(beta, at, a.cols, a.pvec, 0.f, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf((v[e] - mean) * rstd, g[e], b[e]);
    store8(y + at, a.cols - at, a.yvec, v);
  });
}

template <typename T>
cudaError_t forward(const FwdArgs& a, cudaStream_t s) {
  if (a.cols <= 32 * 8 * kKeep)
    return launch_dependent(layer_norm_kernel<T, 32>, dim3(static_cast<unsigned>((a.total + 7) / 8)), kThreads, 0, s, a);
  if (a.cols <= 128 * 8 * kKeep)
    return launch_dependent(layer_norm_kernel<T, 128>, dim3(static_cast<unsigned>((a.total + 1) / 2)), kThreads, 0, s, a);
  return launch_dependent(layer_norm_kernel<T, kThreads>, dim3(static_cast<unsigned>(a.total)), kThreads, 0, s, a);
}

// ------------------------------------------------------------------ backward
struct BwdArgs {
  const void *dy, *x;
  void* dx;
  const float *gamma, *mean, *rstd;
  float *dgamma, *dbeta, *part;       // part: [group][chunk][2][cols]
  int64_t lddy, ldx, lddx, pstride, dstride, total;
  int groups, rows, cols, chunks, per;   // per: rows of a chunk
  int dyvec, xvec, dxvec, pvec;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) norm_dx_kernel(const __grid_constant__ BwdArgs a) {
  __shared__ float part[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int64_t row = blockIdx.x;
  const T *dy = static_cast<const T*>(a.dy) + row * a.lddy, *x = static_cast<const T*>(a.x) + row * a.ldx;
  T* dx = static_cast<T*>(a.dx) + row * a.lddx;
  const float* gamma = a.gamma ? a.gamma + row / a.rows * a.pstride : nullptr;
  const float mean = a.mean[row], rstd = a.rstd[row];
  auto each = [&](auto&& f) {
    for (int64_t at = threadIdx.x * 8; at < a.cols; at += kThreads * 8) {
      float h[8], xh[8], g[8];
      load8(dy + at, a.cols - static_cast<int>(at), a.dyvec, h);
      load8(x + at, a.cols - static_cast<int>(at), a.xvec, xh);
      params8(gamma, static_cast<int>(at), a.cols, a.pvec, 1.f, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[e] *= g[e];
        xh[e] = (xh[e] - mean) * rstd;
      }
      f(static_cast<int>(at), h, xh);
    }
  };
  float sh = 0.f, shx = 0.f;
  each([&](int at, float (&h)[8], float (&xh)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at + e < a.cols) {
        sh += h[e];
        shx = fmaf(h[e], xh[e], shx);
      }
  });
  sh = row_sum<kThreads>(sh, part) / a.cols;
  shx = row_sum<kThreads>(shx, part) / a.cols;
  each([&](int at, float (&h)[8], float (&xh)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = rstd * (h[e] - sh - xh[e] * shx);
    store8(dx + at, a.cols - at, a.dxvec, h);
  });
}

// Sums over a chunk's rows, a column a thread and eight rows at a time.
constexpr int kColTile = 32, kRowLanes = kThreads / kColTile;

template <typename T>
__global__ void __launch_bounds__(kThreads) norm_columns_kernel(const __grid_constant__ BwdArgs a) {
  __shared__ float sums[2][kRowLanes][kColTile];
  pdl_wait();
  pdl_trigger();
  const int c = threadIdx.x % kColTile, lane = threadIdx.x / kColTile;
  const int64_t col = static_cast<int64_t>(blockIdx.x) * kColTile + c;
  const int group = blockIdx.z, chunk = blockIdx.y;
  const int r0 = chunk * a.per, r1 = r0 + a.per < a.rows ? r0 + a.per : a.rows;
  float dg = 0.f, db = 0.f;
  if (col < a.cols)
    for (int r = r0 + lane; r < r1; r += kRowLanes) {
      const int64_t row = static_cast<int64_t>(group) * a.rows + r;
      const float dy = to_f32(static_cast<const T*>(a.dy)[row * a.lddy + col]);
      const float xh = (to_f32(static_cast<const T*>(a.x)[row * a.ldx + col]) - a.mean[row]) * a.rstd[row];
      dg = fmaf(dy, xh, dg);
      db += dy;
    }
  sums[0][lane][c] = dg;
  sums[1][lane][c] = db;
  __syncthreads();
  if (lane < 2 && col < a.cols) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kRowLanes; ++i) s += sums[lane][i][c];
    float* to = a.chunks > 1 ? a.part + ((static_cast<int64_t>(group) * a.chunks + chunk) * 2 + lane) * a.cols
                             : (lane == 0 ? a.dgamma : a.dbeta);
    if (to) to[(a.chunks > 1 ? 0 : group * a.dstride) + col] = s;
  }
}

__global__ void __launch_bounds__(kThreads) norm_join_kernel(const __grid_constant__ BwdArgs a) {
  pdl_wait();
  pdl_trigger();
  const int64_t col = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (col >= a.cols) return;
  const int group = blockIdx.z, which = blockIdx.y;
  float* to = which == 0 ? a.dgamma : a.dbeta;
  if (!to) return;
  const float* from = a.part + (static_cast<int64_t>(group) * a.chunks * 2 + which) * a.cols + col;
  float s = 0.f;
  for (int i = 0; i < a.chunks; ++i) s += from[static_cast<int64_t>(i) * 2 * a.cols];
  to[group * a.dstride + col] = s;
}

// Rows of a chunk: chunks enough to fill the card, each of 64 rows or more.
void split_rows(int groups, int rows, int cols, int& chunks, int& per) {
  const int64_t tiles = (static_cast<int64_t>(cols) + kColTile - 1) / kColTile * groups;
  int64_t want = (1216 + tiles - 1) / tiles;
  const int64_t most = (static_cast<int64_t>(rows) + 63) / 64;
  want = want < most ? want : most;
  if (want < 1) want = 1;
  per = static_cast<int>((rows + want - 1) / want);
  if (per < 1) per = 1;
  chunks = rows > 0 ? (rows + per - 1) / per : 1;
}

int64_t workspace_bytes_of(int groups, int rows, int cols) {
  int chunks, per;
  split_rows(groups, rows, cols, chunks, per);
  return chunks > 1 ? static_cast<int64_t>(groups) * chunks * 2 * cols * 4 : 0;
}

template <typename T>
cudaError_t backward(BwdArgs a, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (a.dgamma || a.dbeta) {
    split_rows(a.groups, a.rows, a.cols, a.chunks, a.per);
    const dim3 grid((a.cols + kColTile - 1) / kColTile, a.chunks, a.groups);
    e = launch_dependent(norm_columns_kernel<T>, grid, kThreads, 0, s, a);
    if (e == cudaSuccess && a.chunks > 1)
      e = launch_dependent(norm_join_kernel, dim3((a.cols + kThreads - 1) / kThreads, 2, a.groups), kThreads, 0, s, a);
  }
  if (e == cudaSuccess && a.dx && a.total > 0)
    e = launch_dependent(norm_dx_kernel<T>, dim3(static_cast<unsigned>(a.total)), kThreads, 0, s, a);
  return e;
}

bool sizes_ok(int groups, int rows, int cols, int dtype) {
  return groups >= 0 && groups <= kMaxGroups && rows >= 0 && rows <= kMaxSide && static_cast<int64_t>(groups) * rows <= kMaxSide &&
         cols >= 1 && cols <= kMaxSide && (dtype == OSCARS_F32 || dtype == OSCARS_BF16);
}
bool at_bytes(const void* p, int n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int rows_16(const void* p, int64_t ld, int size) { return at_bytes(p, 16) && ld * size % 16 == 0; }

}  // namespace
}  // namespace oscars

using namespace oscars;

extern "C" {

oscars_status oscars_layer_norm(const void* x, int64_t ldx, const float* gamma, const float* beta, int64_t param_stride, void* y,
                                int64_t ldy, float* mean, float* rstd, int32_t dtype, int32_t groups, int32_t rows, int32_t cols,
                                float eps, void* stream) {
  if (!sizes_ok(groups, rows, cols, dtype) || ldx < cols || ldy < cols || param_stride < 0 || !(eps > 0.f) || !(eps < INFINITY))
    return OSCARS_EINVAL;
  if (groups == 0 || rows == 0) return OSCARS_OK;
  const int size = dtype == OSCARS_F32 ? 4 : 2;
  if (!x || !y || !at_bytes(x, size) || !at_bytes(y, size) || !at_bytes(gamma, 4) || !at_bytes(beta, 4) || !at_bytes(mean, 4) ||
      !at_bytes(rstd, 4) || (x == y && ldx != ldy))
    return OSCARS_EINVAL;
  FwdArgs a{x, y, gamma, beta, mean, rstd, ldx, ldy, param_stride, static_cast<int64_t>(groups) * rows, rows, cols, eps,
            rows_16(x, ldx, size), rows_16(y, ldy, size), rows_16(gamma, param_stride, 4) && at_bytes(beta, 16)};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == OSCARS_F32 ? forward<float>(a, s) : forward<__nv_bfloat16>(a, s);
  return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

oscars_status oscars_layer_norm_backward_workspace(int32_t groups, int32_t rows, int32_t cols, int64_t* bytes) {
  if (!bytes || !sizes_ok(groups, rows, cols, OSCARS_F32)) return OSCARS_EINVAL;
  *bytes = workspace_bytes_of(groups > 0 ? groups : 1, rows, cols);
  return OSCARS_OK;
}

oscars_status oscars_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* gamma,
                                         int64_t param_stride, const float* mean, const float* rstd, void* dx, int64_t lddx,
                                         float* dgamma, float* dbeta, int64_t dparam_stride, int32_t dtype, int32_t groups,
                                         int32_t rows, int32_t cols, void* workspace, int64_t workspace_bytes, void* stream) {
  if (!sizes_ok(groups, rows, cols, dtype) || lddy < cols || ldx < cols || param_stride < 0) return OSCARS_EINVAL;
  if (groups == 0) return OSCARS_OK;
  const int size = dtype == OSCARS_F32 ? 4 : 2;
  if (rows > 0 && (!dy || !x || !mean || !rstd || !at_bytes(dy, size) || !at_bytes(x, size))) return OSCARS_EINVAL;
  if (!at_bytes(gamma, 4) || !at_bytes(mean, 4) || !at_bytes(rstd, 4) || !at_bytes(dx, size) || !at_bytes(dgamma, 4) || !at_bytes(dbeta, 4))
    return OSCARS_EINVAL;
  if (dx && (lddx < cols || (dx == dy && lddx != lddy) || (dx == x && lddx != ldx))) return OSCARS_EINVAL;
  const bool params = dgamma || dbeta;
  if (params && groups > 1 && dparam_stride < cols) return OSCARS_EINVAL;
  const int64_t need = params ? workspace_bytes_of(groups, rows, cols) : 0;
  if (workspace_bytes < need || (need > 0 && !workspace) || !at_bytes(workspace, 16)) return OSCARS_EINVAL;
  BwdArgs a{};
  a.dy = dy, a.x = x, a.dx = dx, a.gamma = gamma, a.mean = mean, a.rstd = rstd, a.dgamma = dgamma, a.dbeta = dbeta;
  a.part = static_cast<float*>(workspace);
  a.lddy = lddy, a.ldx = ldx, a.lddx = lddx, a.pstride = param_stride, a.dstride = dparam_stride;
  a.total = static_cast<int64_t>(groups) * rows, a.groups = groups, a.rows = rows, a.cols = cols;
  a.dyvec = rows_16(dy, lddy, size), a.xvec = rows_16(x, ldx, size), a.dxvec = rows_16(dx, lddx, size);
  a.pvec = rows_16(gamma, param_stride, 4);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == OSCARS_F32 ? backward<float>(a, s) : backward<__nv_bfloat16>(a, s);
  return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

}  // extern "C"
