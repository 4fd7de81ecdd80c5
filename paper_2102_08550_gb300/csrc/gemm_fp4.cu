// The product of a dense layer kept in 4 bits.
//
//   C[m][n] = act(ra[m] rb[n] sum_k A[m][k] B[n][k] + bias[n]),  A and B codes times their blocks' scales
//
// A product of two codes is a multiple of 1/4 up to 36, so a block's sum is exact in fp32.
//
// Which operand gives the accumulator's rows (its lanes, 128 a CTA) and which its columns is chosen for each call.  With channels
// as rows, the lanes run along a row of C, so that a store of a token's 32 channels is coalesced as it leaves the registers,
// whatever C's alignment.  With tokens as rows, a thread holds a piece of a row of C, which goes through shared memory and leaves by
// TMA: a third of the instructions, with which the warp that issues the products has to share its scheduler.
//
// gemm_fp4_kernel: tcgen05 (kind::mxf4nvf4), persistent, one CTA per SM or a pair (cta_group::2), 20 warps:
//   0       TMA of codes (128 channels and BN tokens, 256 of K) and of their scales into a ring
//   1       copies a stage's scales to tensor memory and issues its products
//   4-19    accumulators -> C, under the products of the next tile
// What bounds a large product is the tensor pipe (69% busy; a pair's K-block of 256 x 256 x 256 is 512 clocks of products) and, while
// results leave, the loads' latency: five stages of 38 KB cover 2500 clocks of it (four 47.3 us, three 54.9).  8192 x 4096 x
// 4096 NV takes 43.5 us in a burst (6.3 PFLOP/s), 48 to 50 back to back for seconds under the power cap; without its results'
// stores 4.5 us less.
// gemm_fp4_few_kernel for one token, or up to three of few channels.
#include <atomic>

#include "../../include/oscars.h"
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

// sum x ra x rb, in this order.  The first product may leave fp32's normal numbers where the result does not: then all of it is
// taken in 64 bits, of this element alone, so that a row knows nothing of its neighbours.  (A call, so that it stays behind a
// branch: 40 x 4096 x 4096 MX takes 9.1 us for 6.8 with both sides computed.)
__device__ __noinline__ float scaled_64(float sum, float ra, float rb) { return static_cast<float>(static_cast<double>(sum) * ra * rb); }
__device__ __forceinline__ float scaled(float sum, float ra, float rb) {
  const float t = sum * ra, m = fabsf(t);   // (a sum of 0 takes the other way to the same 0)
  return m >= 0x1p-126f && m < INFINITY ? t * rb : scaled_64(sum, ra, rb);
}
// Whether it may do so, asked once for many elements (a call without row_a or row_b has one product alone): sums between 2^-20 and
// 2^62, or 0, by scales in [2^-96, 2^64], or 0, stay in [2^-116, 2^126].  NV's sums are all of this kind: multiples of 2^-20,
// and up to 2^30 x 2688^2.
__device__ __forceinline__ bool far_scale(float s) { return s != 0.f && !(fabsf(s) >= 0x1p-96f && fabsf(s) <= 0x1p64f); }
__device__ __forceinline__ bool far_sums(const float (&s)[16]) {   // by their bits without the sign, 0 behind all others in `least`
  uint32_t least = ~0u, most = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const uint32_t u = __float_as_uint(s[e]) << 1;
    least = min(least, u - 1);
    most = max(most, u);
  }
  return least < ((127u - 20) << 24) - 1 || most > (127u + 62) << 24;
}

// N channels' results of a token
template <bool kMx, int N>
__device__ __forceinline__ void finish(const Fp4Args& a, float (&v)[N], float ra, const float (&rb)[N], const float (&bias)[N]) {
  if (__builtin_expect(a.ra && a.rb && (kMx || far_scale(ra)), 0)) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = scaled(v[j], ra, rb[j]);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = v[j] * ra * rb[j];
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (a.bias) v[j] += bias[j];
    if (a.relu && v[j] < 0.f) v[j] = 0.f;
  }
}

// ------------------------------------------------------------------ few tokens
// A warp takes one channel, a lane 32 codes of a row a turn.  Eight products of codes are at most 288, in quarters, which fp16
// holds exactly: a block's sum is two or four such sums, exact in fp32, and is added up times its scales.
// Neither the tensor core's set-up nor its exchange pays here.  Measured (us, this kernel / the one below): 1 x 64 x 100 1.6 / 2.6;
// 1 x 512 x 784 1.8 / 3.5; 1 x 4096 x 1024 3.2 / 3.5; 1 x 4096 x 4096 5.1 / 5.3; 2 x 1024 x 1024 2.5 / 3.4; 3 x 1024 x 1024 3.0 /
// 3.4; beyond the rule 1 x 8192 x 512 3.6 / 3.0, 1 x 8192 x 8192 12 / 8.1, 2 x 4096 x 1024 5.2 / 3.4, 4 x 1024 x 1024 3.4 / 3.4.
constexpr int kFewThreads = 256;
bool few_tokens(int M, int N, int K) {
  const int64_t codes = static_cast<int64_t>(N) * K;
  return M == 1 ? N <= 4096 && codes <= 1 << 24 : M <= 3 && K <= 2048 && codes <= 1 << 20;
}

// codes' products over 16 columns, exact
__device__ __forceinline__ float dot16(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
  uint32_t p[4], q[4];
  eight_values(a0, p);
  eight_values(b0, q);
  __half2 s = __hmul2(*reinterpret_cast<const __half2*>(&p[0]), *reinterpret_cast<const __half2*>(&q[0]));
#pragma unroll
  for (int i = 1; i < 4; ++i) s = __hfma2(*reinterpret_cast<const __half2*>(&p[i]), *reinterpret_cast<const __half2*>(&q[i]), s);
  eight_values(a1, p);
  eight_values(b1, q);
#pragma unroll
  for (int i = 0; i < 4; ++i) s = __hfma2(*reinterpret_cast<const __half2*>(&p[i]), *reinterpret_cast<const __half2*>(&q[i]), s);
  const float2 f = __half22float2(s);
  return f.x + f.y;
}

template <int MT, bool kMx>
__global__ void __launch_bounds__(kFewThreads) gemm_fp4_few_kernel(const __grid_constant__ Fp4Args a) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_trigger();
  const int n = blockIdx.x * (kFewThreads / 32) + warp;
  if (n >= a.N) return;
  const int groups = (a.K + 31) / 32;   // of 32 codes: a block, or two
  auto scales = [&](const uint8_t* s, int64_t row, int g) -> uint32_t {
    if constexpr (kMx) return s[fp4_scale_at(row, g >> 2, a.tiles) + (g & 3)];
    else return *reinterpret_cast<const uint16_t*>(s + fp4_scale_at(row, g >> 1, a.tiles) + 2 * (g & 1));
  };
  float sum[MT] = {};
  constexpr int kAhead = 4;             // turns whose codes are requested together
  for (int g0 = lane; g0 < groups; g0 += 32 * kAhead) {
    uint4 w[kAhead];
    uint32_t sw[kAhead];
#pragma unroll
    for (int h = 0; h < kAhead; ++h) {
      const int g = g0 + 32 * h < groups ? g0 + 32 * h : g0;
      w[h] = *reinterpret_cast<const uint4*>(a.B + n * a.ldb + g * 16);
      sw[h] = scales(a.sb, n, g);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      uint4 x[kAhead];
      uint32_t sx[kAhead];
#pragma unroll
      for (int h = 0; h < kAhead; ++h) {
        const int g = g0 + 32 * h < groups ? g0 + 32 * h : g0;
        x[h] = *reinterpret_cast<const uint4*>(a.A + m * a.lda + g * 16);
        sx[h] = scales(a.sa, m, g);
      }
#pragma unroll
      for (int h = 0; h < kAhead; ++h) {
        if (g0 + 32 * h >= groups) break;
        const float lo = dot16(w[h].x, w[h].y, x[h].x, x[h].y), hi = dot16(w[h].z, w[h].w, x[h].z, x[h].w);
        if constexpr (kMx) {
          sum[m] = fmaf(lo + hi, e8m0_value(sw[h]) * e8m0_value(sx[h]), sum[m]);
        } else {
          const float2 f = __half22float2(e4m3_pair(sw[h])), g = __half22float2(e4m3_pair(sx[h]));
          sum[m] = fmaf(hi, f.y * g.y, fmaf(lo, f.x * g.x, sum[m]));
        }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    float s = sum[m];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == m) {
      float y[1] = {s};
      const float rb[1] = {a.rb ? a.rb[n] : 1.f}, bias[1] = {a.bias ? a.bias[n] : 0.f};
      finish<kMx>(a, y, a.ra ? a.ra[m] : 1.f, rb, bias);
      if (a.bf16) static_cast<__nv_bfloat16*>(a.C)[m * a.ldc + n] = __float2bfloat16_rn(y[0]);
      else static_cast<float*>(a.C)[m * a.ldc + n] = y[0];
    }
  }
}

template <bool kMx>
cudaError_t launch_few(const Fp4Args& a, cudaStream_t s) {
  const dim3 grid((a.N + kFewThreads / 32 - 1) / (kFewThreads / 32));
  switch (a.M) {
    case 1: return launch_dependent(gemm_fp4_few_kernel<1, kMx>, grid, kFewThreads, 0, s, a);
    case 2: return launch_dependent(gemm_fp4_few_kernel<2, kMx>, grid, kFewThreads, 0, s, a);
    default: return launch_dependent(gemm_fp4_few_kernel<3, kMx>, grid, kFewThreads, 0, s, a);
  }
}

// ------------------------------------------------------------------ tensor cores
constexpr int kThreads = 640, kMaxBN = 256, kMaxStages = 8, kEpiWarps = 16, kSpan = kMaxBN / 4;
constexpr int kK = 256;                          // K-block: 128 bytes of a row
constexpr int kBarBytes = 512, kSmem = 227 * 1024;
constexpr size_t kLeast = 164 * 1024;            // one CTA an SM, and no other kernel's cluster beside it (tensor memory)
static_assert(no_cluster_beside(kLeast), "no other cluster's CTA beside this kernel's");
constexpr int kScaleCol = 256;                   // tensor memory: accumulators in front of it, scales of the stages behind

constexpr int kBox = 32 * 64, kTokenBytes = kEpiWarps * kBox + (4 * 2 + 1) * kSpan * 4;   // of the epilogue, with tokens as rows

struct Tile {
  int BN, nt, mt, units, split, stages, accs, tokens;   // accs: accumulators; tokens: they are the rows
};

struct Bars {
  uint64_t full[kMaxStages], empty[kMaxStages], accf[2], acce[2], parts;   // parts: kSplit, all parts' sums are here
  uint32_t tmem;
};
static_assert(sizeof(Bars) <= kBarBytes, "barriers fit");

constexpr uint32_t kLeaderMask = 0xFEFFFFFFu;    // a pair's barrier of the leader at the same offset
__device__ __forceinline__ void tma_load_3d_pair(void* smem_dst, const CUtensorMap* map, int c0, int c1, int c2, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(smem_dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar) & kLeaderMask)
      : "memory");
}
// D (+)= A B^T of codes with block scales in tensor memory, 64 of K
template <int CL, bool kMx>
__device__ __forceinline__ void umma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
#define OSCARS_UMMA_FP4(group, vec)                                                                                       \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"                                                          \
               "tcgen05.mma.cta_group::" group ".kind::mxf4nvf4.block_scale.scale_vec::" vec " [%0], %1, %2, %3, [%4], [%5], p;\n\t}" \
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)                                      \
               : "memory")
  if constexpr (CL == 2 && kMx) OSCARS_UMMA_FP4("2", "2X");
  else if constexpr (CL == 2) OSCARS_UMMA_FP4("2", "4X");
  else if constexpr (kMx) OSCARS_UMMA_FP4("1", "2X");
  else OSCARS_UMMA_FP4("1", "4X");
#undef OSCARS_UMMA_FP4
}
// 512 bytes of scales (a tile of 128 rows x 4 blocks) to four columns of tensor memory
template <int CL>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  if constexpr (CL == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// such a tile in shared memory: 32 rows of 16 bytes, groups of 8 rows 128 bytes apart, no swizzle
__device__ __forceinline__ uint64_t scale_desc(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | static_cast<uint64_t>(128 >> 4) << 32 | static_cast<uint64_t>(1) << 46;
}
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          smem_u32(bar)),
      "h"(static_cast<uint16_t>(0x3))
      : "memory");
}
// An arrival on a barrier of the pair's leader, released at CTA scope: all that it has to come after are reads of this SM's
// tensor memory, which tcgen05.wait::ld has seen finished (gemm_i8.cu).
__device__ __forceinline__ void mbar_arrive_at(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}

// e2m1 operands (1), both K-major; scales e8m0 or e4m3
__host__ __device__ constexpr uint32_t idesc_fp4(int M, int N, bool mx) {
  return (1u << 7) | (1u << 10) | (static_cast<uint32_t>(N >> 3) << 17) | (mx ? 1u << 23 : 0u) | (static_cast<uint32_t>(M >> 7) << 27);
}
// which of a tile's four scales a product takes (0, 2), of both operands
__host__ __device__ constexpr uint32_t scale_id(int id) { return static_cast<uint32_t>(id) << 4 | static_cast<uint32_t>(id) << 29; }

// A thread's channel n of tokens m0 ... m0 + span
template <typename T>
__device__ __forceinline__ void store_tokens(const Fp4Args& a, T* C, int m0, int n, int span, const float (&sum)[kSpan / 16][16],
                                             const float (&ra)[kSpan / 32], float rb, float bias) {
  T* at = C + m0 * a.ldc + n;
  const int rows = n < a.N ? a.M - m0 : 0;
#pragma unroll
  for (int g = 0; g < kSpan / 16; ++g)
    if (16 * g < span) {
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = sum[g][e] * __shfl_sync(0xffffffffu, ra[g / 2], (g & 1) * 16 + e) * rb;
      if (a.bias) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] += bias;
      }
      if (a.relu) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (16 * g + e < rows) *at = static_cast<T>(v[e]);
        at += a.ldc;
      }
    }
}

// 8 values of shared memory, in pairs, read here and not earlier (all of a tile's at once do not fit the registers)
__device__ __forceinline__ void lds8(const float* from, float2 (&v)[4]) {
  const uint32_t at = smem_u32(from);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v[2 * i].x), "=f"(v[2 * i].y), "=f"(v[2 * i + 1].x), "=f"(v[2 * i + 1].y)
                 : "r"(at + 16 * i)
                 : "memory");
}
// A warp's 32 tokens from row on, channels n0 ... n0 + span: 64 bytes of each token at a time go to the warp's box in shared
// memory (64-byte swizzle) and by TMA to C, which clips them at its edges.  `scale`, `bias`: the channels' [kSpan]
template <typename T>
__device__ __forceinline__ void store_channels(const Fp4Args& a, const CUtensorMap* mapC, uint8_t* box, int row, int n0, int span,
                                               const float (&sum)[kSpan / 16][16], const float* scale, const float* bias, float ra) {
  constexpr int kCols = 64 / sizeof(T);
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int c0 = 0; c0 < kSpan; c0 += kCols)
    if (c0 < span && n0 + c0 < a.N) {
      if (lane == 0) bulk_wait_read_all();   // the box is free
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kCols; i += 8) {
        const int at = c0 + i;
        float2 v[4], c[4];
        lds8(scale + at, c);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = __fmul2_rn(__fmul2_rn(make_float2(sum[at / 16][at % 16 + 2 * e], sum[at / 16][at % 16 + 2 * e + 1]), make_float2(ra, ra)), c[e]);
        if (a.bias) {
          lds8(bias + at, c);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = __fadd2_rn(v[e], c[e]);
        }
        if (a.relu) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = make_float2(v[e].x < 0.f ? 0.f : v[e].x, v[e].y < 0.f ? 0.f : v[e].y);
        }
        auto put = [&](int chunk, uint4 w) { *reinterpret_cast<uint4*>(box + lane * 64 + ((chunk ^ ((lane >> 1) & 3)) << 4)) = w; };
        if constexpr (sizeof(T) == 2) {
          put(i / 8, make_uint4(pack_bf16x2(v[0].x, v[0].y), pack_bf16x2(v[1].x, v[1].y), pack_bf16x2(v[2].x, v[2].y), pack_bf16x2(v[3].x, v[3].y)));
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            put(i / 4 + h, make_uint4(__float_as_uint(v[2 * h].x), __float_as_uint(v[2 * h].y), __float_as_uint(v[2 * h + 1].x), __float_as_uint(v[2 * h + 1].y)));
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        tma_store_3d(mapC, box, n0 + c0, row, 0);
        bulk_commit_group();
      }
    }
}

// Tile u of mu x nt: rows fastest, in groups of kGroup of them, so that the tiles under way at once share both operands and a
// wave asks memory for little that is new (8192 x 4096 x 4096 with operands in memory: rows alone 47.1 us, groups of eight 45.8,
// of four 45.0, of two 46.2).
constexpr int kGroup = 4;
__device__ __forceinline__ void tile_at(int u, int mu, int nt, int& row, int& col) {
  const int group = u / (kGroup * nt), in = u - group * kGroup * nt, rows = min(kGroup, mu - group * kGroup);
  col = in / rows;
  row = group * kGroup + in - col * rows;
}

// Rows (W): channels, or, with kTokens, tokens; columns (X): the other.
template <int CL, bool kSplit, bool kMx, bool kTokens>
__global__ void __launch_bounds__(kThreads, 1) gemm_fp4_kernel(const __grid_constant__ CUtensorMap mapW, const __grid_constant__ CUtensorMap mapX,
                                                               const __grid_constant__ CUtensorMap mapSW, const __grid_constant__ CUtensorMap mapSX,
                                                               const __grid_constant__ CUtensorMap mapC,
                                                               const __grid_constant__ Fp4Args a, const __grid_constant__ Tile p) {
  extern __shared__ uint8_t fp4_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(fp4_raw) + 1023) & ~uintptr_t(1023));
  constexpr int kTk = kMx ? 2 : 4;                 // scale tiles of a row tile in a K-block
  const int bn = p.BN / CL, xt = p.BN > 128 ? 2 : 1;   // this CTA's rows of X in a tile; row tiles of their scales
  const int x_at = 128 * 128, sw_at = x_at + bn * 128, sx_at = sw_at + kTk * 512, stage_bytes = (sx_at + xt * kTk * 512 + 1023) & ~1023;
  const int copied = sx_at + xt * kTk * 512;
  uint8_t* ring = smem;
  uint8_t* recv = smem + p.stages * stage_bytes;   // kSplit: the parts' sums of this CTA's tokens [part][BN / split][128]
  uint8_t* boxes = recv;                           // kTokens: a box for each warp of the epilogue, four quarters' scales and biases, ones
  float* ones = reinterpret_cast<float*>(boxes + kEpiWarps * kBox) + 4 * 2 * kSpan;
  Bars* bars = reinterpret_cast<Bars*>(recv + (kSplit ? p.BN * 512 : kTokens ? kTokenBytes : 0));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int part = kSplit ? static_cast<int>(cluster_ctarank()) : 0;
  const int rank = CL > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int nk = (a.K + kK - 1) / kK;
  const int k0 = kSplit ? static_cast<int>(static_cast<int64_t>(nk) * part / p.split) : 0;
  const int k1 = kSplit ? static_cast<int>(static_cast<int64_t>(nk) * (part + 1) / p.split) : nk;
  const int per = kSplit ? p.split : CL;           // CTAs of a tile
  const int u0 = blockIdx.x / per, ustep = gridDim.x / per;
  const int mu = p.mt / CL;                        // row tiles

  if (threadIdx.x == 0) {
    prefetch_tmap(&mapW);
    prefetch_tmap(&mapX);
    prefetch_tmap(&mapSW);
    prefetch_tmap(&mapSX);
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(&bars->full[i], 1);
      mbar_init(&bars->empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->accf[i], 1);
      mbar_init(&bars->acce[i], kEpiWarps * CL);
    }
    mbar_init(&bars->parts, 1);
    if (kSplit) mbar_arrive_expect_tx(&bars->parts, p.BN * 512);
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (kTokens && threadIdx.x >= 128 && threadIdx.x < 128 + kSpan) ones[threadIdx.x - 128] = 1.f;
  if (warp == 2) {
    if (CL == 1) {
      tmem_alloc(&bars->tmem, 512);
      tmem_relinquish();
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem)), "r"(512)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  if (CL > 1 || kSplit) cluster_sync();   // the peers run, and their barriers are initialised
  else __syncthreads();
  tc_fence_after();
  // all of tensor memory is this CTA's, so its columns start at 0: written so, addresses stay in uniform registers and an
  // instruction takes its issue slot instead of 40 clocks (8192 x 4096 x 4096 51.6 -> 44.6 us)
  constexpr uint32_t tmem = 0;
  pdl_wait();
  pdl_trigger();

  bool ok = true;   // of the epilogue's warps: no wait has run out
  if (warp == 0) {
    // ---- TMA
    int it = 0, s = 0, ph = 1;
    uint32_t limit = kSpinLimit;
    for (int u = u0; u < p.units; u += ustep) {
      int tr, tc;
      tile_at(u, mu, p.nt, tr, tc);
      const int r0 = (tr * CL + rank) * 128, c0 = tc * p.BN;
      for (int kb = k0; kb < k1; ++kb, ++it) {
        if (it >= p.stages) mbar_wait_keep(limit, &bars->empty[s], ph, nullptr, kDevTimeoutEmpty);
        if (elect_one() && limit > 1) {
          uint8_t* at = ring + s * stage_bytes;
          uint64_t* bar = &bars->full[s];
          if (rank == 0) mbar_arrive_expect_tx(bar, CL * copied);   // a pair's bytes count on the leader's
          auto load = [&](int to, const CUtensorMap* map, int x, int y, int z) {
            if (CL > 1) tma_load_3d_pair(at + to, map, x, y, z, bar);
            else tma_load_3d(at + to, map, x, y, z, bar);
          };
          load(0, &mapW, kb * 128, r0, 0);
          load(x_at, &mapX, kb * 128, c0 + rank * bn, 0);
          load(sw_at, &mapSW, 0, kb * kTk, r0 >> 7);
          load(sx_at, &mapSX, 0, kb * kTk, c0 >> 7);
        }
        __syncwarp();
        if (++s == p.stages) {
          s = 0;
          ph ^= 1;
        }
      }
    }
    // no copy and no commit of the leader may still be on its way to this CTA when it ends
    for (int i = it > p.stages ? it - p.stages : 0; i < it; ++i)
      mbar_wait_keep(limit, &bars->empty[i % p.stages], (i / p.stages) & 1, nullptr, kDevTimeoutEmpty);
  } else if (warp == 1 && rank == 0) {
    // ---- scales to tensor memory, products (the leader's, of a pair); the warp stays converged and one elected lane issues
    const uint32_t idesc = idesc_fp4(128 * CL, p.BN, kMx), ring0 = smem_u32(ring);
    const int cols = (1 + xt) * kTk * 4;           // of a stage's scales
    int s = 0, ph = 0, t = 0;                      // t: tiles begun
    uint32_t limit = kSpinLimit;
    for (int u = u0; u < p.units; u += ustep, ++t) {
      const int b = t % p.accs;
      const uint32_t acc = tmem + b * 128;
      for (int kb = k0; kb < k1; ++kb) {
        mbar_wait_keep(limit, &bars->full[s], ph, nullptr, kDevTimeoutFull);
        tc_fence_after();
        const uint32_t at = ring0 + s * stage_bytes, sw = tmem + kScaleCol + s * cols, sx = sw + 4 * kTk;
        if (elect_one() && limit > 1) {
          const uint64_t swd = scale_desc(at + sw_at), sxd = scale_desc(at + sx_at);
          // a stage's columns were last read by products that have ended: its copies have been waited for.  Tiles behind the
          // last are zeros that no product takes
          if (xt == 2) {
#pragma unroll
            for (int j = 0; j < kTk; ++j) {
              copy_scales<CL>(sw + 4 * j, swd + j * 32);
              copy_scales<CL>(sx + 8 * j, sxd + j * 32);
              copy_scales<CL>(sx + 8 * j + 4, sxd + (kTk + j) * 32);
            }
          } else {
#pragma unroll
            for (int j = 0; j < kTk; ++j) {
              copy_scales<CL>(sw + 4 * j, swd + j * 32);
              copy_scales<CL>(sx + 4 * j, sxd + j * 32);
            }
          }
        }
        __syncwarp();
        if (kb == k0) {   // the accumulator is free
          if (t >= p.accs) mbar_wait_keep(limit, &bars->acce[b], (t / p.accs + 1) & 1, nullptr, kDevTimeoutAccum);
          tc_fence_after();
        }
        if (elect_one() && limit > 1) {
          const uint64_t wd = smem_desc_k128(at), xd = smem_desc_k128(at + x_at);
          const int left = a.K - kb * kK;
          auto product = [&](int j) {
            const int tile = kMx ? j / 2 : j;
            umma_fp4<CL, kMx>(acc, wd + 2 * j, xd + 2 * j, idesc | (kMx ? scale_id(j % 2 * 2) : 0), sw + 4 * tile, sx + 4 * tile * xt,
                              (kb > k0) | (j > 0));
          };
          if (left >= kK) {
#pragma unroll
            for (int j = 0; j < 4; ++j) product(j);
          } else {
            for (int j = 0; j * 64 < left; ++j) product(j);
          }
          if (CL > 1) umma_commit_pair(&bars->empty[s]);
          else umma_commit(&bars->empty[s]);
        }
        __syncwarp();
        if (++s == p.stages) {
          s = 0;
          ph ^= 1;
        }
      }
      if (elect_one() && limit > 1) {
        if (CL > 1) umma_commit_pair(&bars->accf[b]);
        else umma_commit(&bars->accf[b]);
      }
      __syncwarp();
    }
  } else if (warp >= 4) {
    // ---- C: thread = one row and a quarter of the tile's columns (16 of fewer than 64)
    const int quarter = warp & 3, span = p.BN > 64 ? p.BN / 4 : 16, cb = (warp / 4 - 1) * span;
    const bool works = cb < p.BN;
    int t = 0;
    for (int u = u0; (kTokens || ok) && u < p.units; u += ustep) {
      int tr, tc;
      tile_at(u, mu, p.nt, tr, tc);
      const int row = (tr * CL + rank) * 128 + 32 * quarter + lane, col0 = tc * p.BN + cb;
      const uint32_t row0 = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + cb;
      // of the row; of the columns, lane l those of l, 32 + l, ...
      float mine = 1.f, bias = 0.f, theirs[kSpan / 32];
      const int group = warp / 4 - 1;   // the four warps that have the same columns
      float* scale = reinterpret_cast<float*>(boxes + kEpiWarps * kBox) + group * 2 * kSpan;
      if constexpr (kTokens) {
        if (a.ra && row < a.M) mine = __ldg(a.ra + row);
        // They are done with the tile before.  A wait may have run out in one of them alone, which then comes here once more, and
        // all four leave together: none waits for one that has gone.
        if (!bar_and(1 + group, 128, ok)) break;
        const int i = threadIdx.x & 127, n = col0 + (i & (kSpan - 1));
        if (i < kSpan) scale[i] = a.rb && n < a.N ? __ldg(a.rb + n) : 1.f;
        else scale[i] = a.bias && n < a.N ? __ldg(a.bias + n) : 0.f;
        bar_named(1 + group, 128);
      } else if (!kSplit) {
        if (a.rb && row < a.N) mine = __ldg(a.rb + row);
        if (a.bias && row < a.N) bias = __ldg(a.bias + row);
#pragma unroll
        for (int i = 0; i < kSpan / 32; ++i) theirs[i] = a.ra && col0 + 32 * i + lane < a.M && 32 * i < span ? __ldg(a.ra + col0 + 32 * i + lane) : 1.f;
      }
      float sum[kSpan / 16][16];
      const int b = t % p.accs;
      ok = mbar_wait_warp(&bars->accf[b], (t / p.accs) & 1, nullptr, kDevTimeoutAccum);
      tc_fence_after();
      if (ok) {
        const uint32_t from = row0 + b * 128;
        if (span == kSpan) {
#pragma unroll
          for (int g = 0; g < kSpan / 16; g += 2) tmem_ld_32x32b_x16_pair(from + 16 * g, sum[g], from + 16 * (g + 1), sum[g + 1]);
        } else if (works) {
#pragma unroll
          for (int g = 0; g < kSpan / 32; ++g)
            if (16 * g < span) tmem_ld_32x32b_x16(from + 16 * g, sum[g]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (CL > 1) mbar_arrive_at(cluster_addr(&bars->acce[b], 0));
          else mbar_arrive(&bars->acce[b]);
        }
      }
      ++t;
      if (!ok) {   // every wait that runs out in this CTA ends in one of the accumulator's
        if constexpr (kTokens) continue;
        else break;
      }
      if (!works) continue;
      if constexpr (kSplit) {   // the part's sums [token][channel], where the ring was: its products have ended
#pragma unroll
        for (int g = 0; g < kSpan / 16; ++g)
          if (16 * g < span) {
#pragma unroll
            for (int e = 0; e < 16; ++e) *reinterpret_cast<float*>(ring + ((cb + 16 * g + e) * 128 + 32 * quarter + lane) * 4) = sum[g][e];
          }
      } else {
        bool apart = false;
        if (a.ra && a.rb) {   // the same for all
          if constexpr (kTokens) {
            apart = far_scale(mine);
          } else {
#pragma unroll
            for (int i = 0; i < kSpan / 32; ++i) apart |= far_scale(theirs[i]);
          }
          if constexpr (kMx) {
#pragma unroll
            for (int g = 0; g < kSpan / 16; ++g)
              if (16 * g < span) apart |= far_sums(sum[g]);
          }
          apart = __any_sync(0xffffffffu, apart);
        }
        if (__builtin_expect(apart, 0)) {   // the scales are taken here, and ones below
#pragma unroll
          for (int g = 0; g < kSpan / 16; ++g)
            if (16 * g < span) {
#pragma unroll
              for (int e = 0; e < 16; ++e)
                sum[g][e] = kTokens ? scaled(sum[g][e], mine, scale[16 * g + e])
                                    : scaled(sum[g][e], __shfl_sync(0xffffffffu, theirs[g / 2], (g & 1) * 16 + e), mine);
            }
          mine = 1.f;
#pragma unroll
          for (int i = 0; i < kSpan / 32; ++i) theirs[i] = 1.f;
        }
        if constexpr (kTokens) {
          uint8_t* box = boxes + (warp - 4) * kBox;
          const float* rb = apart ? ones : scale;
          if (row - lane < a.M) {
            if (a.bf16) store_channels<__nv_bfloat16>(a, &mapC, box, row - lane, col0, span, sum, rb, scale + kSpan, mine);
            else store_channels<float>(a, &mapC, box, row - lane, col0, span, sum, rb, scale + kSpan, mine);
          }
        } else {
          if (a.bf16) store_tokens(a, static_cast<__nv_bfloat16*>(a.C), col0, row, span, sum, theirs, mine, bias);
          else store_tokens(a, static_cast<float*>(a.C), col0, row, span, sum, theirs, mine, bias);
        }
      }
    }
    if (kTokens && lane == 0) bulk_wait_all();
  }
  if constexpr (kSplit) {
    // each token's sums go to the CTA that adds up its parts, 128 channels of all of its tokens at once
    const int tokens = p.BN / p.split, bytes = tokens * 512;
    if (warp >= 4) {
      fence_proxy_async_smem();
      if (bar_and(1, kEpiWarps * 32, ok) && threadIdx.x == 128)   // no part is sent that is not whole
        for (int i = 0; i < p.split; ++i) {   // each begins with another one: all at one CTA are received one after the other
          const int r = (part + i) % p.split;
          bulk_copy_to_peer(recv + part * bytes, ring + r * bytes, bytes, &bars->parts, r);
        }
      // a warp adds up a token, four channels a lane
      int tr, tc;
      tile_at(u0, mu, p.nt, tr, tc);
      const int n0 = tr * 128 + lane, m0 = tc * p.BN + part * tokens, end = a.M - m0 < tokens ? a.M - m0 : tokens;
      float rb[4], bias[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        rb[j] = a.rb && n0 + 32 * j < a.N ? __ldg(a.rb + n0 + 32 * j) : 1.f;
        bias[j] = a.bias && n0 + 32 * j < a.N ? __ldg(a.bias + n0 + 32 * j) : 0.f;
      }
      const float* sums = reinterpret_cast<const float*>(recv) + lane;
      if (mbar_wait_warp(&bars->parts, 0, nullptr, kDevTimeoutAccum)) {   // and none is added up that is not there
        for (int i = warp - 4; i < end; i += kEpiWarps) {
          const float ra = a.ra ? __ldg(a.ra + m0 + i) : 1.f;
          float t[4] = {};
          for (int q = 0; q < p.split; ++q)
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] += sums[(q * tokens + i) * 128 + 32 * j];
          finish<kMx>(a, t, ra, rb, bias);
          const int64_t at = (m0 + i) * a.ldc + n0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (n0 + 32 * j >= a.N) continue;
            if (a.bf16) static_cast<__nv_bfloat16*>(a.C)[at + 32 * j] = __float2bfloat16_rn(t[j]);
            else static_cast<float*>(a.C)[at + 32 * j] = t[j];
          }
        }
      }
    }
  }
  tc_fence_before();
  if (CL > 1 || kSplit) cluster_sync();   // the pair's products and arrivals are done in both CTAs; every part's sums have been read
  else __syncthreads();
  if (warp == 2) {
    tc_fence_after();
    if (CL == 1) tmem_dealloc(bars->tmem, 512);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(bars->tmem), "r"(512) : "memory");
  }
}

constexpr int kMaxDevices = 64;
struct DevInfo {
  std::atomic<int> sms{0}, pairs{0};
};
DevInfo g_dev[kMaxDevices];

cudaLaunchConfig_t config(cudaLaunchAttribute* attr, int cluster, int grid, size_t smem, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 0;
  if (cluster > 1) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.numAttrs = 1;
  }
  return cfg;
}

// {SMs, resident clusters of two} of the current device, queried once
void device_room(int& sms, int& pairs) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  sms = g_dev[dev].sms.load(std::memory_order_relaxed);
  pairs = g_dev[dev].pairs.load(std::memory_order_relaxed);
  if (sms > 0 && pairs > 0) return;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) sms = 1;
  cudaLaunchAttribute attr[1];
  pairs = 0;
  if (allow_smem(gemm_fp4_kernel<2, false, false, false>, kSmem) == cudaSuccess) {
    cudaLaunchConfig_t cfg = config(attr, 2, 2, kSmem, nullptr);
    if (cudaOccupancyMaxActiveClusters(&pairs, gemm_fp4_kernel<2, false, false, false>, &cfg) != cudaSuccess) pairs = 0;
  }
  cudaGetLastError();
  if (pairs < 1) pairs = 1;
  g_dev[dev].sms.store(sms, std::memory_order_relaxed);
  g_dev[dev].pairs.store(pairs, std::memory_order_relaxed);
}

template <int CL, bool kSplit, bool kMx, bool kTokens>
cudaError_t launch_fp4(const CUtensorMap (&m)[5], const Fp4Args& a, Tile p, int grid, cudaStream_t s) {
  const int tk = kMx ? 2 : 4, xt = p.BN > 128 ? 2 : 1;
  const int stage = (128 * 128 + p.BN / CL * 128 + (1 + xt) * tk * 512 + 1023) & ~1023, sums = kSplit ? p.BN * 512 : kTokens ? kTokenBytes : 0;
  p.stages = (kSmem - 1024 - kBarBytes - sums) / stage;
  if (p.stages > kMaxStages) p.stages = kMaxStages;
  const int cols = (1 + xt) * tk * 4;
  if (p.stages > (512 - kScaleCol) / cols) p.stages = (512 - kScaleCol) / cols;
  size_t smem = 1024 + static_cast<size_t>(p.stages) * stage + sums + kBarBytes;
  if (smem < kLeast) smem = kLeast;
  cudaError_t e = allow_smem(gemm_fp4_kernel<CL, kSplit, kMx, kTokens>, kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = config(attr, kSplit ? p.split : CL, grid, smem, s);
  attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
  ++cfg.numAttrs;
  return cudaLaunchKernelEx(&cfg, gemm_fp4_kernel<CL, kSplit, kMx, kTokens>, m[0], m[1], m[2], m[3], m[4], a, p);
}

bool code_map(CUtensorMap* m, const uint8_t* base, int64_t ld, int K, int rows, int box_rows) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(fp4_row_bytes(K)), static_cast<cuuint64_t>(rows), 1};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld), static_cast<cuuint64_t>(ld)};   // the third dimension has one entry
  const cuuint32_t box[3] = {128, static_cast<cuuint32_t>(box_rows), 1};
  return encode_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
// scale tiles, 128 words each; tiles past the last are zeros
bool scale_map(CUtensorMap* m, const uint8_t* base, int tiles, int rows, int box_tiles, int box_rows) {
  const cuuint64_t dims[3] = {128, static_cast<cuuint64_t>(tiles), static_cast<cuuint64_t>((static_cast<int64_t>(rows) + 127) / 128)};
  const cuuint64_t strides[2] = {512, static_cast<cuuint64_t>(tiles) * 512};
  const cuuint32_t box[3] = {128, static_cast<cuuint32_t>(box_tiles), static_cast<cuuint32_t>(box_rows)};
  return encode_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE);
}

// C in boxes of 32 rows of 64 bytes
bool result_map(CUtensorMap* m, void* C, int64_t ldc, int M, int N, bool bf16) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(N), static_cast<cuuint64_t>(M), 1};
  const cuuint64_t stride = static_cast<cuuint64_t>(ldc) * (bf16 ? 2 : 4), strides[2] = {stride, stride};
  const cuuint32_t box[3] = {bf16 ? 32u : 16u, 32, 1};
  return encode_map(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, C, dims, strides, box,
                    CU_TENSOR_MAP_SWIZZLE_64B);
}

// The shape with the least estimated time, in clocks, as fitted to 31 sizes in all of their shapes (the choice is within 10% of
// the best of them, one within 15%).  A wave of tiles takes its K-blocks (issue, or loads at 60 bytes a clock, 80 while
// few tiles load) and what lies between two accumulations, or its results' way to memory if that is longer; the last one's
// comes on top, and a split's exchange.
void choose(const Fp4Args& a, bool boxes, int sms, int pairs, Tile& p, int& cl) {
  const int nk = (a.K + kK - 1) / kK;
  double best = 0.0;
  for (int tokens = 0; tokens <= (boxes ? 1 : 0); ++tokens) {
    const int64_t rows = tokens ? a.M : a.N, cols = tokens ? a.N : a.M;
    for (int c = 1; c <= (rows > 128 ? 2 : 1); ++c) {
      const int64_t mt = ((rows + 127) / 128 + c - 1) / c * c;
      for (int bn = c == 1 ? 16 : 64; bn <= kMaxBN; bn *= 2) {
        // a product takes a scale tile from its first row on, and a warp's columns are whole boxes
        if (bn < 128 && (cols > bn || tokens)) continue;
        const int64_t nt = (cols + bn - 1) / bn, units = mt / c * nt;
        const int room = c == 2 ? pairs : sms;
        const double waves = static_cast<double>((units + room - 1) / room);
        const double bytes = (128 + bn / c) * 128 + 512 * (a.mx ? 2 : 4) * (bn > 128 ? 3 : 2);
        const double issue = (c == 2 ? 340.0 : 420.0) + bn, loads = bytes / (waves > 2.0 ? 60.0 : 80.0), kb = issue > loads ? issue : loads;
        const double wide = a.bf16 ? 1.0 : 1.6;
        const double store = tokens ? 1200.0 + 9.4 * wide * bn : (c == 2 ? 400.0 : 2200.0) + 25.0 * bn, last = (tokens ? 12.0 * wide : 26.0) * bn;
        for (int split = 1; split <= (c == 1 && !tokens ? 8 : 1); split *= 2) {
          if (split > 1 && (units * split > sms * 7 / 8 || nk < 2 * split || bn < 2 * split || bn > 128)) break;
          const double main = (nk + split - 1) / split * kb + (bn > 128 ? 900.0 : 300.0);
          const double cost = (split > 1 ? main + 1500.0 + 29.0 * bn : waves * (main > store || waves == 1.0 ? main : store)) + last + (c == 2 ? 900.0 : 0.0);
          if (best == 0.0 || cost < best) {
            best = cost;
            cl = c;
            p.BN = bn;
            p.mt = static_cast<int>(mt);
            p.nt = static_cast<int>(nt);
            p.split = split;
            p.tokens = tokens;
          }
        }
      }
    }
  }
  p.accs = p.BN > 128 ? 1 : 2;
}

template <bool kMx>
cudaError_t launch_tile(const CUtensorMap (&m)[5], const Fp4Args& a, const Tile& p, int cl, int room, cudaStream_t s) {
  const int grid = (p.units < room ? p.units : room) * cl;
  if (p.tokens) return cl == 2 ? launch_fp4<2, false, kMx, true>(m, a, p, grid, s) : launch_fp4<1, false, kMx, true>(m, a, p, grid, s);
  return p.split > 1 ? launch_fp4<1, true, kMx, false>(m, a, p, p.units * p.split, s)
         : cl == 2   ? launch_fp4<2, false, kMx, false>(m, a, p, grid, s)
                     : launch_fp4<1, false, kMx, false>(m, a, p, grid, s);
}

constexpr int64_t kMaxStride = int64_t(1) << 40;   // of a tensor map
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
  if (lda >= kMaxStride || ldb >= kMaxStride) return OSCARS_EINVAL;
  if (M == 0) return OSCARS_OK;
  if (!A || !B || !C || !scales_a || !scales_b || !at_bytes(A, 16) || !at_bytes(B, 16) || !at_bytes(scales_a, 16) || !at_bytes(scales_b, 16) ||
      !at_bytes(row_a, 4) || !at_bytes(row_b, 4) || !at_bytes(bias, 4) || !at_bytes(C, dtype == OSCARS_F32 ? 4 : 2))
    return OSCARS_EINVAL;
  Fp4Args a{A, scales_a, B, scales_b, row_a, row_b, bias, C, lda, ldb, ldc, M, N, K, format == OSCARS_MXFP4, fp4_tiles(K, format), relu,
            dtype == OSCARS_BF16};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (few_tokens(M, N, K)) {
    const cudaError_t e = a.mx ? launch_few<true>(a, s) : launch_few<false>(a, s);
    return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
  }
  int sms, pairs, cl = 1;
  device_room(sms, pairs);
  Tile p{};
  const int size = dtype == OSCARS_F32 ? 4 : 2;
  // TMA stores rows of 16 bytes' alignment
  choose(a, at_bytes(C, 16) && ldc * size % 16 == 0 && ldc < kMaxStride / 8, sms, pairs, p, cl);
  const int64_t units = static_cast<int64_t>(p.mt / cl) * p.nt;
  if (units > INT32_MAX / 2) return OSCARS_EINVAL;
  p.units = static_cast<int>(units);
  const int tk = a.mx ? 2 : 4;
  CUtensorMap m[5] = {};
  const int boxes[2] = {128, p.BN / cl}, tiles[2] = {1, p.BN > 128 ? 2 : 1};   // of the rows' operand, of the columns'
  const int of_a = p.tokens ? 0 : 1, of_b = 1 - of_a;
  if (!code_map(&m[of_a], A, lda, K, M, boxes[of_a]) || !code_map(&m[of_b], B, ldb, K, N, boxes[of_b]) ||
      !scale_map(&m[2 + of_a], scales_a, a.tiles, M, tk, tiles[of_a]) || !scale_map(&m[2 + of_b], scales_b, a.tiles, N, tk, tiles[of_b]) ||
      (p.tokens && !result_map(&m[4], C, ldc, M, N, dtype == OSCARS_BF16)))
    return OSCARS_ECUDA;
  const int room = cl == 2 ? pairs : sms;
  const cudaError_t e = a.mx ? launch_tile<true>(m, a, p, cl, room, s) : launch_tile<false>(m, a, p, cl, room, s);
  return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

}  // extern "C"
