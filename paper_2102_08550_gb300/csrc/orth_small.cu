// Newton-Schulz steps of small matrices in one launch (see orthogonal.cu for the method).
//
// Where the shorter side s is at most 64, a launch for each of a step's products takes longer than its products: 15
// launches of a 10 x 512 matrix took 68 us, their products less than one.  Here a matrix stays in shared memory for all
// steps, the longer side over a cluster of up to 8 CTAs.  A step: each CTA's share of the Gram matrix (fp32, tiles of 4 x 4
// a thread, the long sum over groups of threads); the shares are added in rank order, each CTA a part of the entries, and
// the sums stored to every CTA; B = a I + b A + c A A in every CTA; X <- B X on its columns.  Everything in fp32.
#include <atomic>

#include "../../include/oscars.h"
#include "common.cuh"
#include "internal.h"
#include "rows.cuh"

namespace oscars {

namespace {

constexpr int kThreads = 512;
constexpr int kMaxS = 64, kMaxCluster = 8;
constexpr size_t kMaxSmem = 200 * 1024;
constexpr int kMaxGroups = 32;                   // of threads that share a tile's long sum

struct SmallArgs {
  const void* G;
  int64_t ldg, zg;
  void* out;
  int64_t ldo, zo;
  int out_type;                                  // NsOut
  int rows, cols, s, len, share, cluster, steps; // share: columns (of the longer side) of a CTA, a multiple of 4
  float a, b, c, eps, scale;
  int* status;                                   // set to zero (no wait of this kernel can run out), or NULL
};

int up4(int x) { return (x + 3) / 4 * 4; }
// floats of a row of X: 16-byte aligned, rows on different banks
__host__ __device__ inline int row_floats(int share) { return share % 8 == 4 ? share : share + 4; }
size_t smem_floats(int s, int share) {
  const int s4 = up4(s);
  return static_cast<size_t>(2) * s4 * row_floats(share) + 3 * static_cast<size_t>(s4) * (s4 + 4) + kThreads * 16;
}

__device__ __forceinline__ void st_peer(const void* local, int rank, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr(local, rank)), "f"(v) : "memory");
}
template <typename T>
__global__ void __launch_bounds__(kThreads) orth_small_kernel(const __grid_constant__ SmallArgs p) {
  extern __shared__ __align__(16) float sm[];
  __shared__ Squares norm_part[kThreads / 32], norm_peer[kMaxCluster];
  __shared__ float scale_s[2];
  const int s4 = (p.s + 3) / 4 * 4, lda = s4 + 4, ldx = row_floats(p.share), tid = threadIdx.x;
  float* X = sm;                                 // [2][s4][ldx]
  float* A = X + 2 * s4 * ldx;                   // [s4][lda]
  float* B = A + s4 * lda;                       // [s4][lda]
  float* P = B + s4 * lda;                       // [s4][lda]: this CTA's share of A
  float* red = P + s4 * lda;                     // [groups][tiles][16]
  const int rank = p.cluster > 1 ? static_cast<int>(cluster_ctarank()) : 0, z = blockIdx.x / p.cluster;
  const int l0 = rank * p.share, n = p.len - l0 < p.share ? (p.len - l0 > 0 ? p.len - l0 : 0) : p.share;
  const bool tall = p.rows > p.cols;
  pdl_wait();
  pdl_trigger();
  if (p.status && blockIdx.x == 0 && tid == 0) *p.status = kDevOk;

  // ---- X as it comes, and its norm.  Of a wide matrix a CTA holds columns, of a tall one rows (as columns)
  const T* g = static_cast<const T*>(p.G) + z * p.zg;
  for (int i = tid * 4; i < s4 * ldx; i += kThreads * 4) *reinterpret_cast<float4*>(X + i) = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();
  Squares sum;
  const uint32_t fast = tall ? p.s : n, count = static_cast<uint32_t>(p.s) * n;   // fast: consecutive in memory
  for (uint32_t i0 = tid; i0 < count; i0 += kThreads * 8) {
    float v[8];
    int at[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {   // eight loads in flight
      const uint32_t i = i0 + e * kThreads;
      at[e] = -1;
      v[e] = 0.f;
      if (i < count) {
        const uint32_t outer = i / fast, inner = i - outer * fast;
        const int r = tall ? inner : outer, l = tall ? outer : inner;
        v[e] = to_f32(tall ? g[(l0 + l) * p.ldg + r] : g[r * p.ldg + l0 + l]);
        at[e] = r * ldx + l;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at[e] >= 0) X[at[e]] = v[e];
    sum.add(v);
  }
  sum.block_sum(norm_part);
  if (p.cluster > 1) {
    cluster_sync();                              // every CTA runs
    if (tid == 0)
      for (int q = 0; q < p.cluster; ++q) {
        st_peer(&norm_peer[rank].mid, q, sum.mid);
        st_peer(&norm_peer[rank].big, q, sum.big);
        st_peer(&norm_peer[rank].small, q, sum.small);
      }
    cluster_sync();
    if (tid == 0) {
      sum = norm_peer[0];
      for (int q = 1; q < p.cluster; ++q) sum.add(norm_peer[q]);
    }
  }
  if (tid == 0) inverse_norm(sum.total(), p.eps, scale_s[0], scale_s[1]);   // fp64: one thread's, not 512
  __syncthreads();
  const float power = scale_s[0], factor = scale_s[1];
  for (int i = tid * 4; i < s4 * ldx; i += kThreads * 4) {
    float4 v = *reinterpret_cast<const float4*>(X + i);
    v.x = (v.x * power) * factor, v.y = (v.y * power) * factor, v.z = (v.z * power) * factor, v.w = (v.w * power) * factor;
    *reinterpret_cast<float4*>(X + i) = v;
  }
  __syncthreads();

  // a thread's tile: rows tr, tr + side, ... and columns tc, tc + side, ... (neighbours read neighbouring rows, which
  // lie on different banks); the tiles' long sums over groups of threads
  const int side = s4 / 4, tiles = side * side;  // at most 256
  int groups = 1;
  while (groups < kMaxGroups && groups * 2 * tiles <= kThreads) groups *= 2;
  const int tile = tid % tiles, group = tid / tiles, tr = tile / side, tc = tile % side;
  const int across = p.share / 4;
  int cur = 0;
  for (int step = 0; step < p.steps; ++step) {
    const float* x = X + cur * s4 * ldx;
    float* y = X + (cur ^ 1) * s4 * ldx;
    // ---- this CTA's share of A = X X^T
    if (group < groups) {
      float acc[4][4] = {};
      for (int l = group * 4; l < p.share; l += groups * 4) {
        float4 u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[i] = *reinterpret_cast<const float4*>(x + (tr + i * side) * ldx + l);
          v[i] = *reinterpret_cast<const float4*>(x + (tc + i * side) * ldx + l);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[i][j] = fmaf(u[i].x, v[j].x, fmaf(u[i].y, v[j].y, fmaf(u[i].z, v[j].z, fmaf(u[i].w, v[j].w, acc[i][j]))));
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) red[(group * 16 + e) * tiles + tile] = acc[e / 4][e % 4];
    }
    __syncthreads();
    // entry e of a tile is group e's, e + groups', ... thread of that tile
    if (group < groups)
      for (int e = group; e < 16; e += groups) {
        float v = 0.f;
#pragma unroll 8
        for (int q = 0; q < groups; ++q) v += red[(q * 16 + e) * tiles + tile];
        P[(tr + e / 4 * side) * lda + tc + e % 4 * side] = v;
      }
    // ---- A in every CTA
    const float* full = P;
    if (p.cluster > 1) {
      cluster_sync();                            // the shares are there, and no peer reads the last step's A any more
      const int all = s4 * s4, per = (all + p.cluster - 1) / p.cluster;
      for (int i = rank * per + tid; i < (rank + 1) * per && i < all; i += kThreads) {
        const int at = i / s4 * lda + i % s4;
        float v[kMaxCluster];
#pragma unroll
        for (int q = 0; q < kMaxCluster; ++q) v[q] = q < p.cluster ? ld_dsmem_f32(P + at, q) : 0.f;
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < kMaxCluster; ++q) t += v[q];
        for (int q = 0; q < p.cluster; ++q) st_peer(A + at, q, t);
      }
      cluster_sync();
      full = A;
    } else {
      __syncthreads();
    }
    // ---- B = a I + b A + c A A: an entry a thread, or of more than 16 rows a tile
    if (s4 <= 16) {
      for (int i = tid; i < s4 * s4; i += kThreads) {
        const int r = i / s4, c = i - r * s4;
        float acc = 0.f;
        for (int k = 0; k < s4; k += 4) {
          const float4 u = *reinterpret_cast<const float4*>(full + r * lda + k), v = *reinterpret_cast<const float4*>(full + c * lda + k);
          acc = fmaf(u.x, v.x, fmaf(u.y, v.y, fmaf(u.z, v.z, fmaf(u.w, v.w, acc))));   // A is symmetric
        }
        B[r * lda + c] = fmaf(p.c, acc, fmaf(p.b, full[r * lda + c], r == c ? p.a : 0.f));
      }
    } else if (tid < tiles) {
      float acc[4][4] = {};
      for (int k = 0; k < s4; k += 4) {
        float4 u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[i] = *reinterpret_cast<const float4*>(full + (tr + i * side) * lda + k);
          v[i] = *reinterpret_cast<const float4*>(full + (tc + i * side) * lda + k);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[i][j] = fmaf(u[i].x, v[j].x, fmaf(u[i].y, v[j].y, fmaf(u[i].z, v[j].z, fmaf(u[i].w, v[j].w, acc[i][j]))));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = tr + i * side, c = tc + j * side;
          B[r * lda + c] = fmaf(p.c, acc[i][j], fmaf(p.b, full[r * lda + c], r == c ? p.a : 0.f));
        }
    }
    __syncthreads();
    // ---- X <- B X, four rows and columns a thread
    for (int t = tid; t < side * across; t += kThreads) {
      const int i0 = t / across * 4, l = t % across * 4;
      float4 acc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < s4; k += 4) {
        float4 u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[i] = *reinterpret_cast<const float4*>(B + (i0 + i) * lda + k);
          v[i] = *reinterpret_cast<const float4*>(x + (k + i) * ldx + l);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            acc[i].x = fmaf(w[j], v[j].x, acc[i].x);
            acc[i].y = fmaf(w[j], v[j].y, acc[i].y);
            acc[i].z = fmaf(w[j], v[j].z, acc[i].z);
            acc[i].w = fmaf(w[j], v[j].w, acc[i].w);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(y + (i0 + i) * ldx + l) = acc[i];
    }
    cur ^= 1;
    __syncthreads();
  }
  // ---- the result
  const float* x = X + cur * s4 * ldx;
  for (uint32_t i0 = tid; i0 < count; i0 += kThreads * 8) {
    float v[8];
    int64_t at[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t i = i0 + e * kThreads;
      at[e] = -1;
      if (i < count) {
        const uint32_t outer = i / fast, inner = i - outer * fast;
        const int r = tall ? inner : outer, l = tall ? outer : inner;
        at[e] = z * p.zo + (tall ? (l0 + l) * p.ldo + r : r * p.ldo + l0 + l);
        v[e] = x[r * ldx + l] * p.scale;
        if (p.out_type == kNsAdd) v[e] += static_cast<const float*>(p.out)[at[e]];
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (at[e] < 0) continue;
      if (p.out_type == kNsBf16) static_cast<__nv_bfloat16*>(p.out)[at[e]] = __float2bfloat16_rn(v[e]);
      else static_cast<float*>(p.out)[at[e]] = v[e];
    }
  }
  if (p.cluster > 1) cluster_sync();             // no CTA ends while a peer may read its share
}

}  // namespace

// CTAs a matrix, or 0 where the products run on the tensor cores: the shorter of two estimates of five steps in us, each
// fitted to measurements (s x len x batch, fp32: this kernel / the tensor cores: 10 x 512 x 1 21 / 66, 32 x 1000 x 1 34 / 76,
// 32 x 1000 x 16 67 / 90, 48 x 800 x 1 55 / 78, 64 x 784 x 1 74 / 78, 64 x 784 x 16 146 / 90; bf16: 24 x 1000 x 64 140 / 98).
// A CTA takes 15 us for its barriers and the load, more for longer sides of A and for its share; one CTA runs on an SM.
// The fit is of up to 64 matrices and five steps: the tensor cores' estimate has no waves of its own, so a batch of some hundreds
// goes there sooner than it should (10 x 512 fp32 from 433 matrices on), and other numbers of steps choose as five do.
int ns_small_cluster(int batch, int rows, int cols, bool f32) {
  const int s = rows < cols ? rows : cols, len = rows < cols ? cols : rows;
  if (s > kMaxS) return 0;
  const double per_len = batch <= 8 ? 0.01 : batch <= 32 ? 0.02 : 0.04;   // the tensor cores' Gram products
  double best = 0.9 * ((f32 ? 55.0 : 43.0) + per_len * len);
  int most = 0;
  for (int c = 1; c <= kMaxCluster; c *= 2) {
    const int share = up4((len + c - 1) / c);
    if (smem_floats(s, share) * 4 > kMaxSmem) continue;
    const int room = c == 8 ? 15 * 8 : 144;      // CTAs at once: a GPC's SMs are no multiple of 8
    const double waves = static_cast<double>((static_cast<int64_t>(batch) * c + room - 1) / room);
    const double cost = waves * (15.0 + 0.35 * s + 8e-5 * s * s * share + (c > 1 ? 4.0 : 0.0));
    if (cost < best) {
      best = cost;
      most = c;
    }
  }
  return most;
}

cudaError_t launch_ns_small(const void* G, int64_t ldg, int64_t zg, bool bf16, void* out, int64_t ldo, int64_t zo, int out_type,
                            int batch, int rows, int cols, int cluster, int steps, const float (&co)[3], float eps,
                            float scale, int* status, cudaStream_t s) {
  SmallArgs a{};
  a.G = G, a.ldg = ldg, a.zg = zg;
  a.out = out, a.ldo = ldo, a.zo = zo, a.out_type = out_type;
  a.rows = rows, a.cols = cols;
  a.s = rows < cols ? rows : cols;
  a.len = rows < cols ? cols : rows;
  a.cluster = cluster;
  a.share = up4((a.len + a.cluster - 1) / a.cluster);
  a.steps = steps;
  a.a = co[0], a.b = co[1], a.c = co[2];
  a.eps = eps, a.scale = scale;
  a.status = status;
  const size_t smem = smem_floats(a.s, a.share) * 4;
  void (*kernel)(SmallArgs) = bf16 ? orth_small_kernel<__nv_bfloat16> : orth_small_kernel<float>;
  cudaError_t e = allow_smem(kernel, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(batch * a.cluster, 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = a.cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace oscars
