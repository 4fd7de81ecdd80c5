// The product of a dense layer kept in 8 bits, and the rows' quantisation.
//
//   C[m][n] = act(sa[m] sb[n] sum_k A[m][k] B[n][k] + bias[n]),  the sum exact
//   scale[i] = max_j |x[i][j]| / 127,  q[i][j] = rint(x[i][j] / scale[i])
//
// sm_103a's tensor cores have no 8-bit integer kind.  An 8-bit integer is exact in
// fp16, a product of two is at most 2^14, and fp32 holds sums of 1024 such products
// exactly.  So warps turn tiles of codes into fp16 in shared memory, tcgen05
// (kind::f16) multiplies them, and every kChunk K-blocks (1024 of K) the
// epilogue moves the accumulator, an exact integer, to a sum in int32.
//
// The product is computed as rows = channels (B), columns = tokens (A): the
// accumulator's lanes then run along a row of C, so that a store of a token's 32
// channels is coalesced as it leaves the registers, whatever C's alignment.
//
// gemm_i8_kernel: persistent, one CTA per SM or a cluster of two (cta_group::2),
// 20 warps:
//   0       TMA of code tiles (128 channels and BN tokens, 128 of K) into a ring
//   1       issues the products from the operand ring into one of two accumulators
//   4-11    codes -> fp16, into the operand ring (K-major, 128-byte swizzle)
//   12-19   accumulators -> int32 sums -> C, under the products of the next tile
// What bounds a large product is shared memory: a pair's K-block (256 x 256 x 64)
// brings 16 KB of codes into an SM, which are written, read, written as 32 KB and read
// by the tensor core: 96 KB, 768 clocks at 128 bytes a clock, to 512 of products.
// 8192 x 4096 x 4096 takes 171 us (1.6 PFLOP/s).
//
// gemm_i8_narrow_kernel (up to 32 tokens) and gemm_i8_few_kernel (one or two) below.
#include <atomic>

#include "../../include/oscars.h"
#include "common.cuh"
#include "internal.h"
#include "rows.cuh"

namespace oscars {

namespace {

constexpr int kMaxK = 131071;   // 2^14 (2^17 - 1) < 2^31
constexpr int kMaxSide = 1 << 30;   // rows, columns, tokens, channels: what is counted beyond them by a tile stays an int

// ------------------------------------------------------------------ quantisation
// A row on TPR threads, eight elements a thread and turn; up to kKeep turns stay in registers between the maximum and
// the codes (a longer row is read again, from L2).  Bound by memory: a row is read and its codes are written once.
constexpr int kQThreads = 256, kKeep = 4;

// Four codes.  The quotient's integer is that of x times the reciprocal wherever the product, which is within 3e-5 of the
// quotient, is further than that from a half; the division (about 20 instructions, and most of the kernel's time when every
// value took one: 8192 x 4096 fp32 48 us) is left for the others.  Adding 1.5 x 2^23 rounds to an integer in the low byte.
__device__ __forceinline__ uint32_t four_codes(const float (&w)[8], int at, float s, float r) {
  uint32_t bits[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float q = w[at + e] * r, t = q + 12582912.f;
    bits[e] = __float_as_uint(t);
    if (!(fabsf(q - (t - 12582912.f)) < 0.4999f && fabsf(q) < 127.4f))
      bits[e] = __float_as_uint(fminf(fmaxf(w[at + e] / s, -127.f), 127.f) + 12582912.f);
  }
  return __byte_perm(__byte_perm(bits[0], bits[1], 0x0040), __byte_perm(bits[2], bits[3], 0x0040), 0x5410);
}

template <typename T, int TPR>
__global__ void __launch_bounds__(kQThreads, sizeof(T) == 2 ? 6 : 4) quantize_i8_kernel(const T* __restrict__ x, int64_t ldx, int rows, int cols, int vec,
                                                                int8_t* __restrict__ q, int64_t ldq, int qvec,
                                                                float* __restrict__ scale) {
  constexpr int kRows = kQThreads / TPR;
  __shared__ uint32_t part[kQThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / TPR;
  const int t = threadIdx.x % TPR, turns = (cols + TPR * 8 - 1) / (TPR * 8);
  if (TPR == 32 && row >= rows) return;          // a whole warp
  const bool live = row < rows;
  const T* src = x + (live ? row : 0) * ldx;
  // magnitudes as integers: in order, infinity above every number and NaN above it
  Held8<T> v[kKeep];
  uint32_t mx = 0;
  auto take = [&](const float (&w)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) mx = max(mx, __float_as_uint(w[e]) & 0x7FFFFFFFu);
  };
#pragma unroll
  for (int i = 0; i < kKeep; ++i)
    v[i].load(src + (i * TPR + t) * 8, cols - (i * TPR + t) * 8, vec != 0);
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    float w[8];
    v[i].get(w);
    take(w);
  }
  for (int i = kKeep; i < turns; ++i) {
    float w[8];
    load8(src + (i * TPR + t) * 8, cols - (i * TPR + t) * 8, vec != 0, w);
    take(w);
  }
  mx = __reduce_max_sync(0xffffffffu, mx);
  if (TPR > 32) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = mx;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) mx = max(mx, part[threadIdx.x / TPR * (TPR / 32) + i]);
    if (!live) return;
  }
  const float s = __uint_as_float(mx) / 127.f, r = 1.f / s;
  if (t == 0) scale[row] = s;
  const bool codes = s > 0.f && s < INFINITY;   // neither a row of zeros nor one with an infinity or NaN
  int8_t* out = q + row * ldq;
  auto store = [&](int at, const float (&w)[8]) {
    const uint32_t word[2] = {codes ? four_codes(w, 0, s, r) : 0u, codes ? four_codes(w, 4, s, r) : 0u};
    if (qvec && at + 8 <= cols) {
      *reinterpret_cast<uint2*>(out + at) = make_uint2(word[0], word[1]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < cols) out[at + e] = static_cast<int8_t>(word[e >> 2] >> (8 * (e & 3)));
    }
  };
#pragma unroll
  for (int i = 0; i < kKeep; ++i)
    if ((i * TPR + t) * 8 < cols) {
      float w[8];
      v[i].get(w);
      store((i * TPR + t) * 8, w);
    }
  for (int i = kKeep; i < turns; ++i) {
    float w[8];
    load8(src + (i * TPR + t) * 8, cols - (i * TPR + t) * 8, vec != 0, w);
    if ((i * TPR + t) * 8 < cols) store((i * TPR + t) * 8, w);
  }
}

// Rows up to 1024 long on a warp each, up to 4096 on four, longer ones on a block: as few threads as keep the row in
// registers, so that more rows' loads are in flight (8192 x 4096 bf16 on a block each 40 us).
template <typename T>
cudaError_t quantize(const void* x, int64_t ldx, int rows, int cols, int8_t* q, int64_t ldq, float* scale, cudaStream_t s) {
  const T* src = static_cast<const T*>(x);
  const int vec = (reinterpret_cast<uintptr_t>(x) | static_cast<uintptr_t>(ldx) * sizeof(T)) % 16 == 0;
  const int qvec = (reinterpret_cast<uintptr_t>(q) | static_cast<uintptr_t>(ldq)) % 8 == 0;
  if (cols <= 32 * 8 * kKeep)
    return launch_dependent(quantize_i8_kernel<T, 32>, dim3((rows + 7) / 8), kQThreads, 0, s, src, ldx, rows, cols, vec, q, ldq,
                            qvec, scale);
  if (cols <= 128 * 8 * kKeep)
    return launch_dependent(quantize_i8_kernel<T, 128>, dim3((rows + 1) / 2), kQThreads, 0, s, src, ldx, rows, cols, vec, q, ldq,
                            qvec, scale);
  return launch_dependent(quantize_i8_kernel<T, kQThreads>, dim3(rows), kQThreads, 0, s, src, ldx, rows, cols, vec, q, ldq, qvec,
                          scale);
}

// ------------------------------------------------------------------ product
struct I8Args {
  const float *sa, *sb, *bias;
  void* C;
  int64_t ldc;
  int M, N, K, relu, bf16;
  int BN, nt, mt, units, split, raw_stages, op_stages;   // set by the launcher
};

constexpr int kK = 64, kThreads = 640, kMaxBN = 256;
constexpr int kChunk = 16;                       // K-blocks whose sums fp32 holds exactly
constexpr int kMaxStages = 8, kConvWarps = 8, kEpiWarps = 8;
constexpr int kBarBytes = 512;
constexpr int kSmem = 227 * 1024;
// at least: one CTA an SM, and no other kernel's cluster beside it (tensor memory)
constexpr size_t kLeast = 164 * 1024;
static_assert(no_cluster_beside(kLeast), "no other cluster's CTA beside this kernel's");
static_assert(kChunk * kK * 128 * 128 <= 1 << 24, "a chunk's sums are exact in fp32");

struct Bars {
  uint64_t raw_full[kMaxStages], raw_empty[kMaxStages], op_full[kMaxStages], op_empty[kMaxStages], accf[2], acce[2];
  uint32_t tmem;
  int failed;   // kSplit: a part's sums are not all there
};
static_assert(sizeof(Bars) <= kBarBytes, "barriers fit");

__device__ __forceinline__ void umma_f16_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                              uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          smem_u32(bar)),
      "h"(static_cast<uint16_t>(0x3))
      : "memory");
}
// An arrival on a barrier of the pair's leader, released at CTA scope (the default).  By PTX's memory model that does not
// synchronise with the leader, a thread of another CTA; this relies on the hardware instead: all that the arrival has to come
// after has happened in this SM before it is issued.  That is operands in its own shared memory, which its own tensor core
// reads and a fence.proxy.async of each writing lane has shown to it (the lanes then meet in __syncwarp), or reads of its tensor
// memory, which tcgen05.wait::ld has seen finished.  At cluster scope an arrival took 1000 clocks (8192 x 4096 x 4096: a K-block
// 1200 clocks).
__device__ __forceinline__ void mbar_arrive_at(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
template <int N>
__device__ __forceinline__ void regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
// registers: 640 threads at 96; the warps that keep sums take what the others leave
constexpr int kLowRegs = 48, kHighRegs = 168;
static_assert(kThreads / 128 * 96 == 3 * kLowRegs + 2 * kHighRegs, "the shares add up to the launch's registers");

// four codes as fp16: a code plus 128 in the mantissa of 1024, less 1152
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const uint32_t u = w ^ 0x80808080u;
  const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
  const __half2 off = __half2half2(__ushort_as_half(0x6480));   // 1152
  const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), off), y = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
  lo = *reinterpret_cast<const uint32_t*>(&x);
  hi = *reinterpret_cast<const uint32_t*>(&y);
}

// fp16 operands (format 0), K-major, fp32 accumulator
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N) {
  return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// sum x sa x sb for any scales.  The sum is below 2^31, so its product with a scale in [2^-126, 2^96], or with zero, stays
// among fp32's normal numbers, and only the result can leave them.  With other scales it may where the result does not
// (tokens of 1e37 against channels of 1e-3); then sa is taken 2^64 nearer to 1, and the result times `back` afterwards.
__device__ __forceinline__ float near_one(float s) { return fabsf(s) > 0x1p96f ? s * 0x1p-64f : fabsf(s) < 0x1p-126f ? s * 0x1p64f : s; }
__device__ __forceinline__ float back(float s) { return fabsf(s) > 0x1p96f ? 0x1p64f : fabsf(s) < 0x1p-126f ? 0x1p-64f : 1.f; }

__device__ __forceinline__ float finish(const I8Args& a, int sum, float sa, float sb, float bias) {
  float v = static_cast<float>(sum) * near_one(sa) * sb * back(sa);
  if (a.bias) v += bias;
  return a.relu && v < 0.f ? 0.f : v;
}

// A thread's channel n of tokens m0 ... m0 + span: 16 values at a time without a branch between them (with the type and
// the edges tested at each, a token took a warp 120 clocks, and a tile of 256 x 256 longer than its products)
// (kFar: some of sa are near_one's, a copy of its own, since a branch more a group took 8192 x 512 x 784 from 24.7 to 25.4 us)
template <bool kFar, typename T>
__device__ __forceinline__ void store_tokens(const I8Args& a, T* C, int m0, int n, int span, const int (&sum)[kMaxBN / 32][16],
                                             const float (&sa)[kMaxBN / 64], float sb, float bias) {
  T* at = C + m0 * a.ldc + n;
  const int rows = n < a.N ? a.M - m0 : 0;
#pragma unroll
  for (int g = 0; g < kMaxBN / 32; ++g)
    if (16 * g < span) {
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e)
        v[e] = static_cast<float>(sum[g][e]) * __shfl_sync(0xffffffffu, sa[g / 2], (g & 1) * 16 + e) * sb;
      if constexpr (kFar) {
        const int m = m0 + 16 * g + (threadIdx.x & 15);
        const float to = m < a.M ? back(__ldg(a.sa + m)) : 1.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] *= __shfl_sync(0xffffffffu, to, e);
      }
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

// four bytes into a peer's shared memory
__device__ __forceinline__ void st_peer(const void* local, int rank, int v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(local, rank)), "r"(v) : "memory");
}

template <int CL, bool kSplit>
__global__ void __launch_bounds__(kThreads, 1) gemm_i8_kernel(const __grid_constant__ CUtensorMap mapW,
                                                              const __grid_constant__ CUtensorMap mapX,
                                                              const __grid_constant__ I8Args a) {
  extern __shared__ uint8_t i8_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(i8_raw) + 1023) & ~uintptr_t(1023));
  const int bn = a.BN / CL, rows = 128 + bn;       // this CTA's tokens of a tile; rows of codes of a K-block
  const int raw_bytes = rows * 128, op_bytes = rows * 128;   // 128 codes, or 64 in fp16
  uint8_t* op = smem;                              // [op stages][128 channels | bn tokens][128 bytes]
  uint8_t* raw = smem + a.op_stages * op_bytes;    // [raw stages][128 channels | bn tokens][128 bytes]
  uint8_t* recv = raw + a.raw_stages * raw_bytes;  // kSplit: the parts' sums of this CTA's tokens [part][BN / split][128]
  Bars* bars = reinterpret_cast<Bars*>(recv + (kSplit ? a.BN * 512 : 0));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int part = kSplit ? static_cast<int>(cluster_ctarank()) : 0;
  const int rank = CL > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int nk = (a.K + kK - 1) / kK;
  // this CTA's pairs of K-blocks (a code tile each); the last one's second half may lie behind nk: it takes its
  // turn in the operand ring, but nothing is multiplied
  const int np = (nk + 1) / 2, p0 = kSplit ? np * part / a.split : 0, p1 = kSplit ? np * (part + 1) / a.split : np;
  const int per = kSplit ? a.split : CL;           // CTAs of a tile
  const int u0 = blockIdx.x / per, ustep = gridDim.x / per;
  const int mu = a.mt / CL;                        // row tiles (of channels); rows fastest

  if (threadIdx.x == 0) {
    prefetch_tmap(&mapW);
    prefetch_tmap(&mapX);
    for (int i = 0; i < a.raw_stages; ++i) {
      mbar_init(&bars->raw_full[i], 1);
      mbar_init(&bars->raw_empty[i], kConvWarps);
    }
    for (int i = 0; i < a.op_stages; ++i) {
      mbar_init(&bars->op_full[i], kConvWarps / 2 * CL);
      mbar_init(&bars->op_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->accf[i], 1);
      mbar_init(&bars->acce[i], kEpiWarps * CL);
    }
    bars->failed = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
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
  const uint32_t tmem = bars->tmem;
  pdl_wait();
  pdl_trigger();

  if (warp < 4) {
    regs_down<kLowRegs>();
    if (warp == 0 && lane == 0) {
      // ---- TMA of codes
      int it = 0, s = 0, ph = 1;
      bool ok = true;
      for (int u = u0; ok && u < a.units; u += ustep) {
        const int n0 = ((u % mu) * CL + rank) * 128, m0 = (u / mu) * a.BN + rank * bn;
        for (int p = p0; p < p1; ++p, ++it) {
          if (it >= a.raw_stages && !(ok = mbar_wait(&bars->raw_empty[s], ph, nullptr, kDevTimeoutEmpty))) break;
          uint8_t* at = raw + s * raw_bytes;
          mbar_arrive_expect_tx(&bars->raw_full[s], raw_bytes);
          tma_load_3d(at, &mapW, p * 2 * kK, n0, 0, &bars->raw_full[s]);
          tma_load_3d(at + 128 * 128, &mapX, p * 2 * kK, m0, 0, &bars->raw_full[s]);
          if (++s == a.raw_stages) {
            s = 0;
            ph ^= 1;
          }
        }
      }
      // the copies have landed before this CTA ends: the converting warps wait for each of them, and after a
      // timeout of theirs this thread's waits on the freed slots run out later than any copy takes
      for (int i = it > a.raw_stages ? it - a.raw_stages : 0; i < it; ++i) {
        if (!mbar_wait(&bars->raw_full[i % a.raw_stages], (i / a.raw_stages) & 1, nullptr, kDevTimeoutFull)) break;
      }
    } else if (warp == 1 && rank == 0) {
      // ---- MMA issuer (the leader's, of a pair); the warp stays converged and one elected lane issues
      const uint32_t idesc = idesc_f16(128 * CL, a.BN);
      const uint32_t op0 = smem_u32(op);
      int s = 0, ph = 0, t = 0;   // t: accumulations begun
      uint32_t limit = kSpinLimit;
      for (int u = u0; u < a.units; u += ustep) {
        for (int k0 = 2 * p0; k0 < 2 * p1; k0 += kChunk, ++t) {
          const int b = t & 1, k1 = k0 + kChunk < 2 * p1 ? k0 + kChunk : 2 * p1;
          if (t >= 2) mbar_wait_keep(limit, &bars->acce[b], ((t >> 1) + 1) & 1, nullptr, kDevTimeoutAccum);
          tc_fence_after();
          const uint32_t acc = tmem + static_cast<uint32_t>(b * kMaxBN);
          for (int kb = k0; kb < k1; ++kb) {
            mbar_wait_keep(limit, &bars->op_full[s], ph, nullptr, kDevTimeoutFull);
            tc_fence_after();
            const uint64_t wd = smem_desc_k128(op0 + s * op_bytes), xd = smem_desc_k128(op0 + s * op_bytes + 128 * 128);
            if (elect_one() && limit > 1) {
              for (int j = 0; kb < nk && j < kK / 16; ++j) {
                if (CL > 1) umma_f16_pair(acc, wd + 2 * j, xd + 2 * j, idesc, (kb - k0) | j ? 1u : 0u);
                else umma_bf16(acc, wd + 2 * j, xd + 2 * j, idesc, (kb - k0) | j ? 1u : 0u);
              }
              if (CL > 1) umma_commit_pair(&bars->op_empty[s]);
              else umma_commit(&bars->op_empty[s]);
            }
            __syncwarp();
            if (++s == a.op_stages) {
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
      }
    }
  } else if (warp < 4 + kConvWarps) {
    // ---- codes to fp16: two groups of four warps take the two K-blocks of a code tile, so that one's waits and
    // stores run under the other's; 16 codes of a row a thread and turn, a row's 64 in four neighbouring lanes.
    // Eight lanes, which move 16 bytes each at once, take rows p and p ^ 5 of eight: with the 128-byte swizzle
    // their reads (half a row each) and writes (every second chunk of a row) fall on different banks
    regs_down<kLowRegs>();
    const int th = threadIdx.x & 127, c = th & 3, group = (warp >> 2) - 1;
    const int p8 = lane >> 3, r8 = lane & 4 ? p8 ^ 5 : p8, row = (th >> 5) * 8 + r8;   // rows row, row + 32, ...
    const int from = row * 128 + (((4 * group + c) ^ r8) << 4);
    const int to0 = row * 128 + (((2 * c) ^ r8) << 4), to1 = row * 128 + (((2 * c + 1) ^ r8) << 4);
    int it = 0, rs = 0, rph = 0, os = group, oph = 1;
    bool ok = true;
    for (int u = u0; ok && u < a.units; u += ustep) {
      for (int p = p0; p < p1; ++p, ++it) {
        ok = mbar_wait_warp(&bars->raw_full[rs], rph, nullptr, kDevTimeoutFull);
        if (ok && 2 * it >= a.op_stages) ok = mbar_wait_warp(&bars->op_empty[os], oph, nullptr, kDevTimeoutEmpty);
        if (!ok) break;
        const uint8_t* src = raw + rs * raw_bytes + from;
        uint8_t* dst = op + os * op_bytes;
        if (2 * p + group < nk) {
          for (int r = row; r < rows; r += 128, src += 128 * 128, dst += 128 * 128) {
            uint4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (r + 32 * i < rows) w[i] = *reinterpret_cast<const uint4*>(src + 32 * 128 * i);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (r + 32 * i >= rows) break;
              uint4 x, y;
              codes_to_half(w[i].x, x.x, x.y);
              codes_to_half(w[i].y, x.z, x.w);
              codes_to_half(w[i].z, y.x, y.y);
              codes_to_half(w[i].w, y.z, y.w);
              *reinterpret_cast<uint4*>(dst + to0 + 32 * 128 * i) = x;
              *reinterpret_cast<uint4*>(dst + to1 + 32 * 128 * i) = y;
            }
          }
          fence_proxy_async_smem();
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&bars->raw_empty[rs]);
          if (CL > 1) mbar_arrive_at(cluster_addr(&bars->op_full[os], 0));
          else mbar_arrive(&bars->op_full[os]);
        }
        if (++rs == a.raw_stages) {
          rs = 0;
          rph ^= 1;
        }
        os += 2;
        if (os >= a.op_stages) {
          os = group;
          oph ^= 1;
        }
      }
    }
    it *= 2;
    // no commit of the leader may still be on its way to this CTA when it ends
    for (int i = it > a.op_stages ? it - a.op_stages : 0; ok && i < it; ++i)
      ok = mbar_wait_warp(&bars->op_empty[i % a.op_stages], (i / a.op_stages) & 1, nullptr, kDevTimeoutEmpty);
  } else {
    // ---- sums and C: thread = one channel and half of the tile's tokens
    regs_up<kHighRegs>();
    const int quarter = warp & 3, span = a.BN / 2, cb = warp < 16 ? 0 : span;
    int t = 0;
    bool ok = true;
    for (int u = u0; ok && u < a.units; u += ustep) {
      const int n = ((u % mu) * CL + rank) * 128 + 32 * quarter + lane, m0 = (u / mu) * a.BN + cb;
      const uint32_t row0 = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + cb;
      const float sb = n < a.N ? __ldg(a.sb + n) : 0.f, bias = a.bias && n < a.N ? __ldg(a.bias + n) : 0.f;
      float sa[kMaxBN / 64];   // lane l: tokens l, 32 + l, ...
#pragma unroll
      for (int i = 0; i < kMaxBN / 64; ++i) sa[i] = m0 + 32 * i + lane < a.M && 32 * i < span ? __ldg(a.sa + m0 + 32 * i + lane) : 0.f;
      bool far = false;        // of any of the tile's tokens
      if (!kSplit) {
#pragma unroll
        for (int i = 0; i < kMaxBN / 64; ++i) {
          far |= sa[i] != 0.f && back(sa[i]) != 1.f;
          sa[i] = near_one(sa[i]);
        }
        far = __any_sync(0xffffffffu, far);
      }
      int sum[kMaxBN / 32][16];
#pragma unroll
      for (int g = 0; g < kMaxBN / 32; ++g)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[g][e] = 0;
      for (int k0 = 2 * p0; k0 < 2 * p1; k0 += kChunk, ++t) {
        const int b = t & 1;
        if (!(ok = mbar_wait_warp(&bars->accf[b], (t >> 1) & 1, nullptr, kDevTimeoutAccum))) break;
        tc_fence_after();
#pragma unroll
        for (int g = 0; g < kMaxBN / 32; ++g)
          if (16 * g < span) {
            float v[16];
            tmem_ld_32x32b_x16(row0 + b * kMaxBN + 16 * g, v);
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[g][e] += __float2int_rn(v[e]);
          }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (CL > 1) mbar_arrive_at(cluster_addr(&bars->acce[b], 0));
          else mbar_arrive(&bars->acce[b]);
        }
      }
      if (!ok) {   // every wait that runs out in this CTA ends in one of the accumulator's; its peers then leave the tile alone too
        if (kSplit && lane < a.split) st_peer(&bars->failed, lane, 1);
        break;
      }
      if constexpr (kSplit) {   // a part's sums [token][channel] go to the CTA that adds up the token
        const int owned = a.BN / a.split;
#pragma unroll
        for (int g = 0; g < kMaxBN / 32; ++g)
          if (16 * g < span) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int tok = cb + 16 * g + e;
              st_peer(recv + ((part * owned + tok % owned) * 128 + 32 * quarter + lane) * 4, tok / owned, sum[g][e]);
            }
          }
      } else if (far) {
        if (a.bf16) store_tokens<true>(a, static_cast<__nv_bfloat16*>(a.C), m0, n, span, sum, sa, sb, bias);
        else store_tokens<true>(a, static_cast<float*>(a.C), m0, n, span, sum, sa, sb, bias);
      } else if (a.bf16) {
        store_tokens<false>(a, static_cast<__nv_bfloat16*>(a.C), m0, n, span, sum, sa, sb, bias);
      } else {
        store_tokens<false>(a, static_cast<float*>(a.C), m0, n, span, sum, sa, sb, bias);
      }
    }
  }
  tc_fence_before();
  if (CL > 1 || kSplit) cluster_sync();   // the pair's products and arrivals are done in both CTAs; every part's sums are there
  else __syncthreads();
  if constexpr (kSplit) {
    // each CTA adds up its tokens of the tile over the parts
    const int missing = bars->failed;
    const int n0 = (u0 % mu) * 128, tokens = a.BN / a.split, m0 = (u0 / mu) * a.BN + part * tokens;
    const int* sums = reinterpret_cast<const int*>(recv);
    for (int i = threadIdx.x; missing == 0 && i < tokens * 128; i += kThreads) {
      const int m = m0 + i / 128, n = n0 + i % 128;
      if (m >= a.M || n >= a.N) continue;
      int t = 0;
      for (int p = 0; p < a.split; ++p) t += sums[p * tokens * 128 + i];
      const float y = finish(a, t, __ldg(a.sa + m), __ldg(a.sb + n), a.bias ? __ldg(a.bias + n) : 0.f);
      if (a.bf16) static_cast<__nv_bfloat16*>(a.C)[m * a.ldc + n] = __float2bfloat16_rn(y);
      else static_cast<float*>(a.C)[m * a.ldc + n] = y;
    }
  }
  if (warp == 2) {
    tc_fence_after();
    if (CL == 1) tmem_dealloc(tmem, 512);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// ------------------------------------------------------------------ few tokens
// One token, or two of few channels: bound by the channels' bytes and by latency, so neither the tensor core's set-up nor a
// conversion pays.  A warp takes one channel, each lane 16 codes of a row a turn; the tokens are multiplied with them by dp4a
// as they come, and the lanes' sums meet in log2(32) exchanges that halve the number of values a lane holds.  Measured (us,
// this kernel / the one for up to 32 tokens): 1 x 512 x 784 1.7 / 2.3; 1 x 4096 x 4096 4.3 / 5.6 (3.9 TB/s of codes); 2 x 300 x
// 8192 8.0 / 8.9; 2 x 1024 x 1024 2.3 / 2.4; beyond the rule 2 x 4096 x 4096 6.5 / 5.9, 4 x 512 x 784 2.9 / 2.4.
constexpr int kFewThreads = 256;
bool few_tokens(int M, int N) { return M == 1 || (M == 2 && N <= 1024); }

// the sums over the lanes of V (a power of two) values: lane l ends with that of value l V / 32
template <int V>
__device__ __forceinline__ void lanes_sum(int (&v)[V], int lane) {
#pragma unroll
  for (int o = 16, n = V; o > 0; o >>= 1) {
    if (n > 1) {
      n >>= 1;
      const bool up = lane & o;
#pragma unroll
      for (int i = 0; i < V / 2; ++i)
        if (i < n) {
          const int mine = up ? v[i + n] : v[i], other = up ? v[i] : v[i + n];
          v[i] = mine + __shfl_xor_sync(0xffffffffu, other, o);
        }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
  }
}

// 16 codes from column k on, zero from column K on
__device__ __forceinline__ int4 codes16(const int8_t* p, int left) {
  int4 w = *reinterpret_cast<const int4*>(p);
  if (left < 16) {
    auto cut = [&](int v, int n) { return n >= 4 ? v : n <= 0 ? 0 : v & ((1 << (8 * n)) - 1); };
    w.x = cut(w.x, left), w.y = cut(w.y, left - 4), w.z = cut(w.z, left - 8), w.w = cut(w.w, left - 12);
  }
  return w;
}

template <int MT>
__global__ void __launch_bounds__(kFewThreads) gemm_i8_few_kernel(const int8_t* __restrict__ A, int64_t lda, const int8_t* __restrict__ B,
                                                                  int64_t ldb, const __grid_constant__ I8Args a) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = blockIdx.x * (kFewThreads / 32) + warp;
  pdl_wait();
  pdl_trigger();
  if (n >= a.N) return;
  int sum[MT] = {};
  const int8_t* w = B + n * ldb;
  constexpr int kAhead = 4;   // turns whose codes are requested together
  for (int k0 = lane * 16; k0 < a.K; k0 += 512 * kAhead) {
    int4 b[kAhead];
#pragma unroll
    for (int h = 0; h < kAhead; ++h)
      b[h] = k0 + 512 * h < a.K ? *reinterpret_cast<const int4*>(w + k0 + 512 * h) : make_int4(0, 0, 0, 0);
#pragma unroll
    for (int h = 0; h < kAhead; ++h) {
      const int k = k0 + 512 * h;
      if (k >= a.K) break;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int4 x = codes16(A + m * lda + k, a.K - k);   // what lies behind column K of B meets zeros
        sum[m] = __dp4a(b[h].x, x.x, sum[m]);
        sum[m] = __dp4a(b[h].y, x.y, sum[m]);
        sum[m] = __dp4a(b[h].z, x.z, sum[m]);
        sum[m] = __dp4a(b[h].w, x.w, sum[m]);
      }
    }
  }
  lanes_sum<MT>(sum, lane);
  if (lane % (32 / MT) != 0) return;
  const int m = lane / (32 / MT);
  const float v = finish(a, sum[0], __ldg(a.sa + m), __ldg(a.sb + n), a.bias ? __ldg(a.bias + n) : 0.f);
  if (a.bf16) static_cast<__nv_bfloat16*>(a.C)[m * a.ldc + n] = __float2bfloat16_rn(v);
  else static_cast<float*>(a.C)[m * a.ldc + n] = v;
}

template <int MT>
cudaError_t launch_few(const int8_t* A, int64_t lda, const int8_t* B, int64_t ldb, const I8Args& a, cudaStream_t s) {
  constexpr int kPer = kFewThreads / 32;
  return launch_dependent(gemm_i8_few_kernel<MT>, dim3((a.N + kPer - 1) / kPer), kFewThreads, 0, s, A, lda, B, ldb, a);
}

// ------------------------------------------------------------------ up to 32 tokens
// Bound by the channels' bytes: they go from global memory to registers, become fp16 there and meet the tokens in mma.sync
// (m16n8k16), whose operands need no shared memory; in the tcgen05 kernel a K-block's 128 channels pass it four times.  The
// order of K within a lane's 16 codes is the same for both operands, so a lane's 16-byte load holds its share of four
// products as it comes.  A CTA takes 32 channels, its warps K-blocks of 128 in turn; sums move to int32 every 1024 of
// K, and the warps' sums meet in shared memory.
constexpr int kNarrowK = 128, kNarrowCh = 32;

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int NT, int kWarps>   // groups of 8 tokens
__global__ void __launch_bounds__(32 * kWarps, NT == 4 ? 1 : 16 / kWarps) gemm_i8_narrow_kernel(const int8_t* __restrict__ A, int64_t lda,
                                                                        const int8_t* __restrict__ B, int64_t ldb,
                                                                        const __grid_constant__ I8Args a) {
  __shared__ int sums[kWarps][NT * 8][kNarrowCh];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * kNarrowCh;
  pdl_wait();
  pdl_trigger();
  const int8_t* w[4];        // rows g, g + 8, g + 16, g + 24 of the channels; the last one again past the end
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = B + static_cast<int64_t>(n0 + g + 8 * i < a.N ? n0 + g + 8 * i : a.N - 1) * ldb + 16 * t;
  float acc[2][NT][4] = {};
  int sum[2][NT][4] = {};
  int turn = 0;
  for (int k0 = warp * kNarrowK; k0 < a.K; k0 += kWarps * kNarrowK) {
    int4 c[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        c[h][i] = k0 + 64 * h + 16 * t < a.K ? __ldcs(reinterpret_cast<const int4*>(w[i] + k0 + 64 * h)) : make_int4(0, 0, 0, 0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = k0 + 64 * h + 16 * t;
      int4 x[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j)   // codes behind column K, and tokens behind the last, are zeros
        x[j] = k < a.K && 8 * j + g < a.M ? codes16(A + (8 * j + g) * lda + k, a.K - k) : make_int4(0, 0, 0, 0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) codes_to_half(q == 0 ? c[h][i].x : q == 1 ? c[h][i].y : q == 2 ? c[h][i].z : c[h][i].w, lo[i], hi[i]);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          uint32_t b0, b1;
          codes_to_half(q == 0 ? x[j].x : q == 1 ? x[j].y : q == 2 ? x[j].z : x[j].w, b0, b1);
          mma_f16(acc[0][j], lo[0], lo[1], hi[0], hi[1], b0, b1);
          mma_f16(acc[1][j], lo[2], lo[3], hi[2], hi[3], b0, b1);
        }
      }
    }
    if (++turn == 1024 / kNarrowK) {
      turn = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sum[i][j][e] += __float2int_rn(acc[i][j][e]);
            acc[i][j][e] = 0.f;
          }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)   // channel 16 i + g (+ 8), token 8 j + 2 t (+ 1)
        sums[warp][8 * j + 2 * t + (e & 1)][16 * i + g + 8 * (e >> 1)] = sum[i][j][e] + __float2int_rn(acc[i][j][e]);
  __syncthreads();
  const int n = n0 + lane;
  if (n >= a.N) return;
  const float sb = __ldg(a.sb + n), bias = a.bias ? __ldg(a.bias + n) : 0.f;
  for (int m = warp; m < a.M; m += kWarps) {
    int v = 0;
#pragma unroll
    for (int p = 0; p < kWarps; ++p) v += sums[p][m][lane];
    const float y = finish(a, v, __ldg(a.sa + m), sb, bias);
    if (a.bf16) static_cast<__nv_bfloat16*>(a.C)[m * a.ldc + n] = __float2bfloat16_rn(y);
    else static_cast<float*>(a.C)[m * a.ldc + n] = y;
  }
}

// Measured (us, this kernel / the tcgen05 kernel): 8 x 512 x 784 2.3 / 7.5, 16 x 512 x 784 3.2 / 7.5, 32 x 1024 x 1024 4.7 / 6.4,
// 8 x 4096 x 4096 4.7 / 10.4 (3.6 TB/s of codes), 16 x 4096 x 4096 6.5 / 10.3; 16 x 300 x 8192 9.2 / 9.4; beyond the rule 32 x 4096
// x 4096 13.2 / 10.6, 32 x 16384 x 512 11.8 / 6.4.
bool narrow(int M, int N, int K) {
  return M <= 16 || (M <= 32 && static_cast<int64_t>(N) * K <= (2 << 20));
}

template <int NT, int kWarps>
cudaError_t launch_narrow(const int8_t* A, int64_t lda, const int8_t* B, int64_t ldb, const I8Args& a, cudaStream_t s) {
  return launch_dependent(gemm_i8_narrow_kernel<NT, kWarps>, dim3((a.N + kNarrowCh - 1) / kNarrowCh), 32 * kWarps, 0, s, A, lda, B,
                          ldb, a);
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
  if (allow_smem(gemm_i8_kernel<2, false>, kSmem) == cudaSuccess) {
    cudaLaunchConfig_t cfg = config(attr, 2, 2, kSmem, nullptr);
    if (cudaOccupancyMaxActiveClusters(&pairs, gemm_i8_kernel<2, false>, &cfg) != cudaSuccess) pairs = 0;
  }
  cudaGetLastError();
  if (pairs < 1) pairs = 1;
  g_dev[dev].sms.store(sms, std::memory_order_relaxed);
  g_dev[dev].pairs.store(pairs, std::memory_order_relaxed);
}

template <int CL, bool kSplit>
cudaError_t launch_i8(const CUtensorMap& mW, const CUtensorMap& mX, I8Args a, int grid, cudaStream_t s) {
  const int tile = (128 + a.BN / CL) * 128, sums = kSplit ? a.BN * 512 : 0, room = kSmem - 1024 - kBarBytes - sums;
  // an even number of operand stages: a slot belongs to one of the two converting groups, which sees each of its phases
  a.op_stages = 6 * tile > room ? 2 : 4;
  a.raw_stages = room / tile - a.op_stages;
  if (a.raw_stages > kMaxStages) a.raw_stages = kMaxStages;
  size_t smem = 1024 + static_cast<size_t>(a.op_stages + a.raw_stages) * tile + sums + kBarBytes;
  if (smem < kLeast) smem = kLeast;
  cudaError_t e = allow_smem(gemm_i8_kernel<CL, kSplit>, kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = config(attr, kSplit ? a.split : CL, grid, smem, s);
  attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
  ++cfg.numAttrs;
  return cudaLaunchKernelEx(&cfg, gemm_i8_kernel<CL, kSplit>, mW, mX, a);
}

bool code_map(CUtensorMap* m, const int8_t* base, int64_t ld, int K, int rows, int box_rows) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(K), static_cast<cuuint64_t>(rows), 1};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld), static_cast<cuuint64_t>(ld)};   // the third dimension has one entry
  const cuuint32_t box[3] = {2 * kK, static_cast<cuuint32_t>(box_rows), 1};
  return encode_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

}  // namespace
}  // namespace oscars

using namespace oscars;

extern "C" {

oscars_status oscars_quantize_i8(const void* x, int64_t ldx, int32_t dtype, int32_t rows, int32_t cols, int8_t* q,
                                 int64_t ldq, float* scale, void* stream) {
  if (rows < 0 || rows > kMaxSide || cols < 1 || cols > kMaxSide || ldx < cols || ldq < cols || (dtype != OSCARS_F32 && dtype != OSCARS_BF16))
    return OSCARS_EINVAL;
  if (rows == 0) return OSCARS_OK;
  if (!x || !q || !scale || (reinterpret_cast<uintptr_t>(scale) & 3) ||
      (reinterpret_cast<uintptr_t>(x) & (dtype == OSCARS_F32 ? 3 : 1)))
    return OSCARS_EINVAL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == OSCARS_F32 ? quantize<float>(x, ldx, rows, cols, q, ldq, scale, s)
                                            : quantize<__nv_bfloat16>(x, ldx, rows, cols, q, ldq, scale, s);
  return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

oscars_status oscars_gemm_i8_nt(const int8_t* A, int64_t lda, const float* scale_a, const int8_t* B, int64_t ldb,
                                const float* scale_b, const float* bias, int32_t relu, void* C, int64_t ldc,
                                int32_t dtype, int32_t M, int32_t N, int32_t K, void* stream) {
  if (M < 0 || M > kMaxSide || N < 1 || N > kMaxSide || K < 1 || K > kMaxK || lda < K || ldb < K || lda % 16 || ldb % 16 || ldc < N ||
      (dtype != OSCARS_F32 && dtype != OSCARS_BF16))
    return OSCARS_EINVAL;
  if (M == 0) return OSCARS_OK;
  if (!A || !B || !C || !scale_a || !scale_b) return OSCARS_EINVAL;
  if ((reinterpret_cast<uintptr_t>(A) | reinterpret_cast<uintptr_t>(B)) & 15) return OSCARS_EINVAL;
  if ((reinterpret_cast<uintptr_t>(scale_a) | reinterpret_cast<uintptr_t>(scale_b) | reinterpret_cast<uintptr_t>(bias)) & 3)
    return OSCARS_EINVAL;
  if (reinterpret_cast<uintptr_t>(C) & (dtype == OSCARS_F32 ? 3 : 1)) return OSCARS_EINVAL;
  I8Args p{scale_a, scale_b, bias, C, ldc, M, N, K, relu, dtype == OSCARS_BF16, 0, 0, 0, 0, 1, 0, 0};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (few_tokens(M, N)) {
    const cudaError_t e = M == 1 ? launch_few<1>(A, lda, B, ldb, p, s) : launch_few<2>(A, lda, B, ldb, p, s);
    return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
  }
  if (narrow(M, N, K)) {
    // 16 warps where each has two K-blocks or more, so that the codes' latency is waited for less often (8 x 4096 x 4096 6.0 ->
    // 4.7 us), else 8 and two CTAs an SM (8 x 8192 x 2048 4.7, 5.5 with 16)
    const bool many = K > 2048;
    const cudaError_t e = M > 16  ? launch_narrow<4, 8>(A, lda, B, ldb, p, s)
                          : M > 8 ? (many ? launch_narrow<2, 16>(A, lda, B, ldb, p, s) : launch_narrow<2, 8>(A, lda, B, ldb, p, s))
                                  : (many ? launch_narrow<1, 16>(A, lda, B, ldb, p, s) : launch_narrow<1, 8>(A, lda, B, ldb, p, s));
    return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
  }
  int sms, pairs;
  device_room(sms, pairs);
  // the shape with the least estimated time: waves of tiles times the longer of a K-block's products (2 BN
  // clocks), shared-memory traffic (3 clocks a row of codes) and loads (45 bytes a clock), plus fixed parts
  const int nk = (K + kK - 1) / kK;
  double best = 0.0;
  int cl = 1;
  for (int c = 1; c <= 2; ++c) {
    const int mt = ((N + 127) / 128 + c - 1) / c * c;
    for (int bn = 32; bn <= kMaxBN; bn *= 2) {
      const int nt = (M + bn - 1) / bn, rows = 128 + bn / c;
      const int64_t units = static_cast<int64_t>(mt / c) * nt;
      const int room = c == 2 ? pairs : sms;
      double kb = 2.0 * bn;
      kb = kb > 3.0 * rows ? kb : 3.0 * rows;
      kb = kb > rows * kK / 45.0 ? kb : rows * kK / 45.0;
      // few tiles: the K-blocks of each over a cluster of `split` CTAs, whose sums meet in shared memory (us with and
      // without: 33 x 1024 x 1024 6.5, 8.4; 64 x 4096 x 4096 12.2, 12.3; not worth it for 777 x 1003 x 1537 17.7, 12.2)
      for (int split = 1; split <= (c == 1 ? 8 : 1); split *= 2) {
        if (split > 1 && (units * split > (split == 8 ? sms * 3 / 4 : sms * 7 / 8) || nk < 4 * split || bn < 4 * split || bn > 128)) break;
        const double waves = split > 1 ? 1.0 : static_cast<double>((units + room - 1) / room);
        const double cost = waves * ((nk + split - 1) / split * kb + 600.0) + 15.0 * bn + (c == 2 ? 1500.0 : 0.0) + (split > 1 ? 3000.0 : 0.0);
        if (best == 0.0 || cost < best) {
          best = cost;
          cl = c;
          p.BN = bn;
          p.mt = mt;
          p.nt = nt;
          p.split = split;
        }
      }
    }
  }
  const int64_t units = static_cast<int64_t>(p.mt / cl) * p.nt;
  if (units > INT32_MAX / 2) return OSCARS_EINVAL;
  p.units = static_cast<int>(units);
  CUtensorMap mW, mX;
  if (!code_map(&mW, B, ldb, K, N, 128) || !code_map(&mX, A, lda, K, M, p.BN / cl)) return OSCARS_ECUDA;
  const int room = cl == 2 ? pairs : sms, grid = (p.units < room ? p.units : room) * cl;
  const cudaError_t e = p.split > 1 ? launch_i8<1, true>(mW, mX, p, p.units * p.split, s)
                        : cl == 2   ? launch_i8<2, false>(mW, mX, p, grid, s)
                                    : launch_i8<1, false>(mW, mX, p, grid, s);
  return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

}  // extern "C"
