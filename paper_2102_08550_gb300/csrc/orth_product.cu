// The three products of a Newton-Schulz step on the 5th-generation tensor cores
// (tcgen05, sm_103a), for a batch of matrices in one launch:
//
//   kNsSym   A' = X X^T + beta I (X K-major) or X^T X + beta I (X read MN-major)
//            B = c A' A' + gamma I
//   kNsStep  X <- B X (X read MN-major) or X B
//   kNsLast  the same into the caller's matrix
//
// With beta = b / 2c and gamma = a - b^2 / 4c, B is a I + b A + c A A: the
// polynomial takes one product of A' with itself and nothing else (reading A in
// that product's epilogue, 32 rows a load, took 10000 to 20000 clocks a tile, more
// than the products of 1024 columns).
//
// Precision.  tcgen05 multiplies 16-bit operands; a value is kept as one fp16 (11
// bits) or as two whose sum has 22, and a product of values in two halves takes
// three products, high x high, high x low and low x high (the fourth is below
// fp32's last bit), into one fp32 accumulator.  fp32 results take two halves of
// everything, the second stored 2^11 times larger (internal.h): the accumulator takes the
// two mixed products of a K-block first, and the first instruction of high x high scales
// what is there by 2^-11 (scale-input-d), which costs nothing.  bf16 results take
// two halves of X and one of A and B: what X's rounding leaves in the directions in which
// the update is near zero is multiplied by a at every step (485 over five), while the
// roundings of A and B multiply X and stay relative to it (in the Gram product and the last
// step X takes one half as well).  The largest of them is that of A's diagonal, about beta, which
// all of a row is multiplied by: the Gram product keeps it (cut), and the next adds what it
// is worth to B's diagonal (error beside the result's own rounding, which is 1.66e-3,
// after five steps: 512 x 784 1.05 -> 0.81e-3, 100 x 2000 1.75 -> 1.18e-3).  Later steps multiply
// what earlier ones lost, so of more than five steps all but the last three take two halves of A
// and B too (error of 400 x 4096 after eight, in roundings of the result: 1.92 in one half throughout, 1.81 with two in
// all but the last five, 1.14 in all but three, 1.07 in all; 4096 x 4096 2.01 ms, 2.59, 2.98, 3.81).
// fp16 rather than bf16: three more bits at the same rate, and the values are bounded
// (singular values below 2).
//
// The tensor core cuts what an addition to its accumulator leaves below fp32's last
// bit.  Over 4096 products in three passes of 256 additions each that is a loss of
// 1e-5 of a sum of squares, so for fp32 results the accumulator takes kChunk K-blocks
// at a time, and the epilogue adds it, rounded to nearest, to a sum in registers.
// What is cut off a K-block's own additions always makes its sum smaller, by about 2^-22
// of it on average; the factors give that back (kNsWhole).  Error against 64 bits over five
// steps without it, with 2^-23, 2^-22, 3 x 2^-23 and 2^-21: 130 x 3000 3.8, 2.8, 1.9,
// 1.7, 2.4e-6; 80 x 90 2.9, 2.1, 1.7, 2.0, 2.9e-6; 1024 x 1024 3.0, 2.3, 1.7, 1.6, 1.9e-6;
// 385 x 1537 2.8, 1.9, 1.4, 1.7, 2.6e-6 (a library's fp32 products 1.3, 1.1, 2.6, 2.6e-6).
//
// A and B are symmetric: where there is work for more than a wave of tiles, only
// those on and above the diagonal are computed, and the epilogue writes each tile and
// its mirror image, half the work of two of the three products.
//
// Structure: persistent, one CTA per SM or a cluster of two (cta_group::2, a tile
// of 256 x BN) striding over tiles, or a cluster of two or four on the K-blocks of one
// tile; warp 0 streams K-blocks of 64 by TMA
// (128-byte swizzle), warp 1 issues into one of two TMEM accumulators, warps 4-11
// (half of a tile's columns each group of four) run the epilogue of a tile, or the
// sum of a chunk, under the products of the next.
#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "internal.h"
#include "orth_shape.h"

namespace oscars {

namespace {

constexpr int kK = kNsK, kThreads = 384, kMaxBN = kNsMaxBN, kMaxStages = kNsMaxStages;
constexpr int kChunk = 1;                          // K-blocks of one accumulation of an fp32 result
static_assert(kChunk == 1, "an accumulation's mixed products come before its others, which scale them once");
constexpr int kEpiWarps = kNsEpiWarps, kBox = kNsBox, kStg = kNsStg, kStgBytes = kNsStgBytes, kBarBytes = kNsBarBytes;
constexpr int kSmem = kNsSmem;
// at least: one CTA an SM, and no other kernel's cluster beside it (tensor memory)
constexpr size_t kLeast = 164 * 1024;
static_assert(no_cluster_beside(kLeast), "no other cluster's CTA beside this kernel's");

struct Bars {
  uint64_t full[kMaxStages], empty[kMaxStages], accf[2], acce[2];
  uint32_t tmem;
  uint32_t failed;   // kSplit: a part's sums are not all there
};
static_assert(sizeof(Bars) <= kBarBytes, "barriers fit");

constexpr uint32_t kLeaderMask = 0xFEFFFFFFu;   // a pair's barrier of the leader at the same offset
__device__ __forceinline__ void tma_load_3d_pair(void* smem_dst, const CUtensorMap* map, int c0, int c1, int c2, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(smem_dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar) & kLeaderMask)
      : "memory");
}
// kind::f16 takes its operands' type from the instruction descriptor
__device__ __forceinline__ void umma_f16_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                              uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// the same (or a CTA's alone) with what the accumulator holds times 2^-kNsShift
template <int CL>
__device__ __forceinline__ void umma_f16_scaled(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc) {
  if (CL > 1)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.eq.b32 p, 0, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p, %4;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "n"(kNsShift)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.eq.b32 p, 0, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p, %4;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "n"(kNsShift)
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
// after is reads of this SM's own tensor memory, which tcgen05.wait::ld has seen finished before the arrival is issued, and
// no write has to be visible.  At cluster scope an arrival takes 1000 clocks.
__device__ __forceinline__ void mbar_arrive_at(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// 16 bytes into a peer's shared memory (an address from cluster_addr)
__device__ __forceinline__ void st_dsmem_at(uint32_t remote, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(remote), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
               : "memory");
}
__device__ __forceinline__ void st_dsmem_at(uint32_t remote, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote), "r"(v) : "memory");
}
// to = v where a == b, as a select: an array element chosen by lane would go through local memory (16 x 512 x 784 bf16 210 us)
__device__ __forceinline__ void take_if(float& to, float v, int a, int b) {
  asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %2, %3;\n\tselp.f32 %0, %1, %0, p;\n\t}" : "+f"(to) : "f"(v), "r"(a), "r"(b));
}
// fp16 operands (format 0), fp32 accumulator; bits 15 and 16: A, B MN-major
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, int a_mn, int b_mn) {
  return (1u << 4) | (static_cast<uint32_t>(a_mn) << 15) | (static_cast<uint32_t>(b_mn) << 16) |
         (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// tile of a work unit: the matrix, and row and column tile (i <= j on a triangle)
struct Tile {
  int z, i, j;
};
template <int CL, bool kSym, bool kSplit>
__device__ __forceinline__ Tile tile_of(const NsArgs& a, int u) {
  Tile t;
  if (kSym && (kSplit || !a.full)) {
    const int per = a.nt * (a.nt + 1) / 2;
    t.z = u / per;
    int r = u - t.z * per;
    t.i = 0;
    while (r >= a.nt - t.i) r -= a.nt - t.i++;
    t.j = t.i + r;
  } else {
    const int mu = a.mt / CL, per = mu * a.nt;
    t.z = u / per;
    const int r = u - t.z * per;
    t.j = r / mu;   // rows fastest
    t.i = r - t.j * mu;
  }
  return t;
}

template <int EPI, int CL, bool kSums, bool kSplit>
__global__ void __launch_bounds__(kThreads, 1) ns_product_kernel(const __grid_constant__ CUtensorMap mapA,
                                                                 const __grid_constant__ CUtensorMap mapB,
                                                                 const __grid_constant__ CUtensorMap mapD,
                                                                 const __grid_constant__ NsArgs a) {
  constexpr bool kSym = EPI == kNsSym;
  extern __shared__ uint8_t ns_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ns_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* stg = smem;
  uint8_t* ring = smem + kStgBytes;   // [stages][A: halves x 2 boxes | B: halves x BN / CL / 64 boxes]
  const int b_boxes = a.BN / CL / 64, b_half = b_boxes * kBox;
  const int a_bytes = a.a_halves * 2 * kBox, stage_bytes = a_bytes + a.b_halves * b_half;
  // kSplit: the parts' sums of this CTA's columns [part][BN / split / 4][128 rows][4]
  uint8_t* recv = ring + a.stages * stage_bytes;
  Bars* bars = reinterpret_cast<Bars*>(recv + (kSplit ? 128 * a.BN * 4 : 0));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int rank = CL > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int nk = (a.K + kK - 1) / kK;
  // kSplit: the K-blocks of a tile over a cluster of a.split CTAs, whose sums meet in shared memory
  const int part = kSplit ? static_cast<int>(cluster_ctarank()) : 0;
  const int kb0 = kSplit ? nk * part / a.split : 0, kb1 = kSplit ? nk * (part + 1) / a.split : nk;
  const int chunk = kSums ? kChunk : nk;   // K-blocks of one accumulation
  const int u0 = blockIdx.x / (kSplit ? a.split : CL), ustep = gridDim.x / (kSplit ? a.split : CL);

  if (threadIdx.x == 0) {
    prefetch_tmap(&mapA);
    prefetch_tmap(&mapB);
    if (EPI != kNsLast) prefetch_tmap(&mapD);
    for (int i = 0; i < a.stages; ++i) {
      mbar_init(&bars->full[i], 1);
      mbar_init(&bars->empty[i], 1);
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
  if (CL > 1 || kSplit) cluster_sync();   // the peers run, and their barriers are initialised before anything arrives on them
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem;
  pdl_wait();
  pdl_trigger();
  // A launch before this one that gave up a wait has left a matrix unfinished: the caller's is not touched then.
  const int before = EPI == kNsLast && warp >= 4 ? *static_cast<const volatile int*>(a.status) : 0;

  // ---- what the epilogue's warps do with 32 columns of their 32 rows (m0) of matrix z, from column n on
  uint8_t* my = stg + (warp >= 4 ? warp - 4 : 0) * 2 * kStg;
  int nst = 0;
  float extra = 0.f;   // of this lane's row, on D's diagonal; read before the tile's products are there
  auto finish = [&](int z, int m0, int n, bool mirrored, const float (&v)[32]) {
    if constexpr (EPI != kNsLast) {
      uint32_t hi[16], lo[16];
      const int d = m0 + lane - n;   // the column on the diagonal
      constexpr bool kCut = kSym && !kSums;
      const float on = kCut ? a.diag + extra : a.diag;
      const float larger = kSym ? static_cast<float>(1 << kNsShift) : a.d_second;   // (two halves of A and B always meet two)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = fmaf(v[2 * e], a.factor, kSym && d == 2 * e ? on : 0.f);
        const float y = fmaf(v[2 * e + 1], a.factor, kSym && d == 2 * e + 1 ? on : 0.f);
        const __half2 h = __floats2half2_rn(x, y);
        const float2 f = __half22float2(h);
        const __half2 l = __floats2half2_rn((x - f.x) * larger, (y - f.y) * larger);
        hi[e] = *reinterpret_cast<const uint32_t*>(&h);
        lo[e] = *reinterpret_cast<const uint32_t*>(&l);
      }
      if (kCut && m0 == n && a.cut) {   // a box on the diagonal, whose elements are each lane's own
        float mine = 0.f;
#pragma unroll
        for (int e = 0; e < 32; ++e) take_if(mine, v[e], lane, e);
        const float x = fmaf(mine, a.factor, on), kept = __half2float(__float2half_rn(x));
        if (m0 + lane < a.M) a.cut[z * static_cast<int64_t>(a.M) + m0 + lane] = 2.f * kept * (x - kept);
      }
      // one box of 32 x 32: rows as they are, or (kSym) the mirror image
      auto store = [&](const uint32_t (&w)[16], int half, bool mirror) {
        uint8_t* box = my + (nst & 1) * kStg;
        if (lane == 0 && nst >= 2) bulk_wait_read_but_one();   // the store of two boxes ago has read this one
        ++nst;
        __syncwarp();
        if (!mirror) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *reinterpret_cast<uint4*>(box + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) =
                make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e)
            *reinterpret_cast<uint16_t*>(box + e * 64 + (((lane >> 3) ^ ((e >> 1) & 3)) << 4) + (lane & 7) * 2) =
                static_cast<uint16_t>(w[e >> 1] >> (16 * (e & 1)));
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          tma_store_3d(&mapD, box, mirror ? m0 : n, mirror ? n : m0, half * a.batch + z);
          bulk_commit_group();
        }
      };
      store(hi, 0, false);
      if (a.d_halves == 2) store(lo, 1, false);
      if (kSym && mirrored) {
        store(hi, 0, true);
        if (a.d_halves == 2) store(lo, 1, true);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q)
        *reinterpret_cast<float4*>(my + lane * 128 + ((q ^ (lane & 7)) << 4)) =
            make_float4(v[4 * q] * a.factor * a.scale, v[4 * q + 1] * a.factor * a.scale, v[4 * q + 2] * a.factor * a.scale,
                        v[4 * q + 3] * a.factor * a.scale);
      __syncwarp();
      // rows of 32 columns, coalesced whatever the caller's alignment, 16 at a time without a branch between them
      const int col = n + lane, rows = col < a.N && before == 0 ? (a.M - m0 < 32 ? a.M - m0 : 32) : 0;
      const int64_t at0 = z * a.zo + col + static_cast<int64_t>(m0) * a.ldo;
      auto store = [&](auto* out, bool add) {
#pragma unroll
        for (int i0 = 0; i0 < 32; i0 += 16) {
          float x[16], old[16];
          auto* at = out + at0 + i0 * a.ldo;
          if (add) {
#pragma unroll
            for (int i = 0; i < 16; ++i) old[i] = i0 + i < rows ? static_cast<float>(at[i * a.ldo]) : 0.f;
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int rr = i0 + i;
            x[i] = *reinterpret_cast<const float*>(my + rr * 128 + (((lane >> 2) ^ (rr & 7)) << 4) + (lane & 3) * 4);
            if (add) x[i] += old[i];
          }
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (i0 + i < rows) at[i * a.ldo] = static_cast<std::remove_reference_t<decltype(*at)>>(x[i]);
        }
      };
      if (a.out_type == kNsBf16) store(static_cast<__nv_bfloat16*>(a.out), false);
      else store(static_cast<float*>(a.out), a.out_type == kNsAdd);
      __syncwarp();
    }
  };

  if (warp == 0) {
    // ---- TMA producer: the warp stays converged and one elected lane issues (a lane alone, with its box counts
    // divided out of the arguments, took up to 700 clocks a K-block)
    int it = 0, s = 0, ph = 1, armed = 0;
    uint32_t limit = kSpinLimit;
    for (int u = u0; u < a.units; u += ustep) {
      const Tile t = tile_of<CL, kSym, kSplit>(a, u);
      const int m0 = (t.i * CL + rank) * 128, n0 = t.j * a.BN + rank * (a.BN / CL);
      const bool same = kSym && t.i == t.j && b_boxes == 2;   // a tile on the diagonal: B is A
      const uint32_t bytes = CL * (same ? a_bytes : stage_bytes);
      for (int kb = kb0; kb < kb1; ++kb, ++it) {
        if (it >= a.stages) mbar_wait_keep(limit, &bars->empty[s], ph, nullptr, kDevTimeoutEmpty);
        if (elect_one() && limit > 1) {
          uint8_t* at = ring + s * stage_bytes;
          uint64_t* bar = &bars->full[s];
          if (rank == 0) mbar_arrive_expect_tx(bar, bytes);   // a pair's bytes count on the leader's
          auto load = [&](const CUtensorMap* map, int c0, int c1, int z) {
            if (CL > 1) tma_load_3d_pair(at, map, c0, c1, z, bar);
            else tma_load_3d(at, map, c0, c1, z, bar);
          };
          const int k = kb * kK;
          for (int h = 0, z = t.z; h < a.a_halves; ++h, z += a.batch) {
            if (a.a_mn) {
              load(&mapA, m0, k, z);
              at += kBox;
              load(&mapA, m0 + 64, k, z);
              at += kBox;
            } else {
              load(&mapA, k, m0, z);
              at += 2 * kBox;
            }
          }
          if (!same)
            for (int h = 0, z = t.z; h < a.b_halves; ++h, z += a.batch)
              for (int i = 0; i < a.b_loads; ++i, at += a.b_rows * 128)
                load(&mapB, a.b_mn ? n0 + a.b_rows * i : k, a.b_mn ? k : n0 + a.b_rows * i, z);
          armed = it + 1;
        }
        __syncwarp();
        if (++s == a.stages) {
          s = 0;
          ph ^= 1;
        }
      }
    }
    // no copy, and no commit of the leader, may still be on its way when this CTA ends
    armed = __reduce_max_sync(0xffffffffu, armed);
    for (int i = armed > a.stages ? armed - a.stages : 0; i < armed; ++i) {
      if (rank == 0) mbar_wait_warp(&bars->full[i % a.stages], (i / a.stages) & 1, nullptr, kDevTimeoutFull);
      if (!mbar_wait_warp(&bars->empty[i % a.stages], (i / a.stages) & 1, nullptr, kDevTimeoutEmpty)) break;
    }
  } else if (warp == 1 && rank == 0) {
    // ---- MMA issuer (the leader's, of a pair); the warp stays converged and one elected lane issues
    const uint32_t idesc = idesc_f16(128 * CL, a.BN, a.a_mn, a.b_mn);
    const uint32_t ring0 = smem_u32(ring);
    const uint64_t astep = a.a_mn ? 128 : 2, bstep = a.b_mn ? 128 : 2;   // 16 of K in the address field
    const uint64_t alo = 2 * kBox >> 4, blo = b_half >> 4;               // from the first half to the second
    int s = 0, ph = 0, t = 0;   // t: accumulations begun
    uint32_t limit = kSpinLimit;
    for (int u = u0; u < a.units; u += ustep) {
      bool same = false;
      if (kSym) {
        const Tile tl = tile_of<CL, kSym, kSplit>(a, u);
        same = tl.i == tl.j && b_boxes == 2;
      }
      const int b_off = same ? 0 : a_bytes;
      for (int k0 = kb0; k0 < kb1; k0 += chunk, ++t) {
        const int b = t & 1, k1 = k0 + chunk < kb1 ? k0 + chunk : kb1;
        if (t >= 2) mbar_wait_keep(limit, &bars->acce[b], ((t >> 1) + 1) & 1, nullptr, kDevTimeoutAccum);
        tc_fence_after();
        const uint32_t acc = tmem + static_cast<uint32_t>(b * kMaxBN);
        for (int kb = k0; kb < k1; ++kb) {
          mbar_wait_keep(limit, &bars->full[s], ph, nullptr, kDevTimeoutFull);
          tc_fence_after();
          const uint32_t at = ring0 + s * stage_bytes;
          const uint64_t ad = a.a_mn ? smem_desc_mn128(at, kBox) : smem_desc_k128(at);
          const uint64_t bd = a.b_mn ? smem_desc_mn128(at + b_off, kBox) : smem_desc_k128(at + b_off);
          if (elect_one() && limit > 1) {
            uint32_t more = kb == k0 ? 0u : 1u;
            auto issue = [&](uint64_t x, uint64_t y, int n = kK / 16) {
#pragma unroll
              for (int j = 0; j < kK / 16; ++j) {
                if (j >= n) break;
                if (CL > 1) umma_f16_pair(acc, x + j * astep, y + j * bstep, idesc, more);
                else umma_bf16(acc, x + j * astep, y + j * bstep, idesc, more);
                more = 1u;
              }
            };
            if (kSums || a.b_halves == 2) issue(ad, bd + blo);
            if (kSums || a.a_halves == 2) issue(ad + alo, bd);
            if (kSums) {   // kChunk is 1: the accumulator holds these two products alone
              umma_f16_scaled<CL>(acc, ad, bd, idesc);
              issue(ad + astep, bd + bstep, kK / 16 - 1);
            } else {
              issue(ad, bd);
            }
            if (CL > 1) umma_commit_pair(&bars->empty[s]);
            else umma_commit(&bars->empty[s]);
          }
          __syncwarp();
          if (++s == a.stages) {
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
  } else if (warp >= 4) {
    // ---- epilogue: thread = one accumulator row and half of its columns
    const int quarter = warp & 3, span = a.BN / 2, cb = (warp >> 2) == 1 ? 0 : span;
    int t = 0;
    // the accumulator may be written again (by accumulation t + 2)
    auto release = [&](int b) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (CL > 1) mbar_arrive_at(cluster_addr(&bars->acce[b], 0));
        else mbar_arrive(&bars->acce[b]);
      }
    };
    // a part's sums go to the CTA that owns the columns, four columns of 32 rows (512 bytes in a row) a store.  Read by
    // their owner from the peers, 32 loads a thread took 12000 clocks; stored 16 bytes a row, 4600.
    auto keep = [&](int c, const float (&v)[32]) {
      const int owned = a.BN / a.split, owner = c / owned;
      const uint32_t at = cluster_addr(recv + (((part * owned + c % owned) / 4) * 128 + 32 * quarter + lane) * 16, owner);
#pragma unroll
      for (int q = 0; q < 8; ++q)
        st_dsmem_at(at + q * 128 * 16, make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]));
    };
    // Every wait of this CTA that runs out ends in one of the accumulator's, so those are recorded; its peers leave the tile
    // alone then too.
    auto give_up = [&] {
      if (lane == 0) atomicCAS(a.status, kDevOk, kDevTimeoutAccum);
      if (kSplit && lane < a.split) st_dsmem_at(cluster_addr(&bars->failed, lane), 1u);
    };
    for (int u = u0; u < a.units; u += ustep) {
      const Tile tl = tile_of<CL, kSym, kSplit>(a, u);
      const int m0 = (tl.i * CL + rank) * 128 + 32 * quarter, n0 = tl.j * a.BN + cb;
      const uint32_t row0 = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + cb;
      if (kSym && !kSums && a.add)
        extra = tl.i == tl.j && m0 + lane < a.M ? a.factor * a.add[tl.z * static_cast<int64_t>(a.M) + m0 + lane] : 0.f;
      if constexpr (kSums) {
        float sum[kMaxBN / 64][32];
#pragma unroll
        for (int g = 0; g < kMaxBN / 64; ++g)
#pragma unroll
          for (int e = 0; e < 32; ++e) sum[g][e] = 0.f;
        bool ok = true;
        for (int k0 = kb0; k0 < kb1; k0 += chunk, ++t) {
          const int b = t & 1;
          if (!(ok = mbar_wait_warp(&bars->accf[b], (t >> 1) & 1, nullptr, kDevTimeoutAccum))) break;
          tc_fence_after();
#pragma unroll
          for (int g = 0; g < kMaxBN / 64; ++g)
            if (32 * g < span) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                float v[16];
                tmem_ld_32x32b_x16(row0 + b * kMaxBN + 32 * g + 16 * h, v);
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[g][16 * h + e] += v[e];
              }
            }
          release(b);
        }
        if (!ok) {
          give_up();
          break;
        }
#pragma unroll
        for (int g = 0; g < kMaxBN / 64; ++g)
          if (kSplit ? 32 * g < span : 32 * g < span && n0 + 32 * g < a.N && m0 < a.M) {
            if (kSplit) keep(cb + 32 * g, sum[g]);
            else finish(tl.z, m0, n0 + 32 * g, tl.i != tl.j && (kSplit || !a.full), sum[g]);
          }
      } else {
        const int b = t & 1;
        if (!mbar_wait_warp(&bars->accf[b], (t >> 1) & 1, nullptr, kDevTimeoutAccum)) {
          give_up();
          break;
        }
        tc_fence_after();
        for (int c0 = 0; c0 < span && (kSplit || (n0 + c0 < a.N && m0 < a.M)); c0 += 32) {
          float v[32];
          tmem_ld_32x32b_x32(row0 + b * kMaxBN + c0, v);
          if (kSplit) keep(cb + c0, v);
          else finish(tl.z, m0, n0 + c0, tl.i != tl.j && (kSplit || !a.full), v);
        }
        release(b);
        ++t;
      }
    }
    if (lane == 0) bulk_wait_all();
  }
  tc_fence_before();
  if (CL > 1 || kSplit) cluster_sync();   // the pair's products and arrivals are done in both CTAs; every part's sums are there
  else __syncthreads();
  if constexpr (kSplit) {
    // each CTA adds up its columns of the tile over the parts, in their order
    const uint32_t missing = bars->failed;   // (read at each turn it took 1024 x 1024 fp32 from 162.4 to 163.0 us)
    const int quarter = warp & 3, span = a.BN / a.split;
    const Tile tl = tile_of<CL, kSym, kSplit>(a, u0);
    const int m0 = tl.i * 128 + 32 * quarter;
    for (int c0 = 32 * ((warp >> 2) - 1); warp >= 4 && missing == 0 && c0 < span; c0 += 64) {
      const int c = part * span + c0, n = tl.j * a.BN + c;
      if (n >= a.N || m0 >= a.M) break;
      float v[32];
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] = 0.f;
      for (int p = 0; p < a.split; ++p) {
        const uint8_t* at = recv + (((p * span + c0) / 4) * 128 + 32 * quarter + lane) * 16;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float4 f = *reinterpret_cast<const float4*>(at + q * 128 * 16);
          v[4 * q] += f.x, v[4 * q + 1] += f.y, v[4 * q + 2] += f.z, v[4 * q + 3] += f.w;
        }
      }
      finish(tl.z, m0, n, tl.i != tl.j && (kSplit || !a.full), v);
    }
    if (warp >= 4 && lane == 0) bulk_wait_all();
  }
  if (warp == 2) {
    tc_fence_after();
    if (CL == 1) tmem_dealloc(tmem, 512);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

constexpr int kMaxDevices = 64;
struct DevInfo {
  std::atomic<int> sms{0}, pairs{0}, fours{0};
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

// {SMs, clusters of two and of four that run at once} of the current device, queried once
void device_room(int& sms, int& pairs, int& fours) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  sms = g_dev[dev].sms.load(std::memory_order_relaxed);
  pairs = g_dev[dev].pairs.load(std::memory_order_relaxed);
  fours = g_dev[dev].fours.load(std::memory_order_relaxed);
  if (sms > 0 && pairs > 0 && fours > 0) return;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) sms = 1;
  auto clusters = [](int size) {
    int n = 0;
    cudaLaunchAttribute attr[1];
    if (allow_smem(ns_product_kernel<kNsStep, 1, true, true>, kSmem) == cudaSuccess) {
      cudaLaunchConfig_t cfg = config(attr, size, size, kSmem, nullptr);
      if (cudaOccupancyMaxActiveClusters(&n, ns_product_kernel<kNsStep, 1, true, true>, &cfg) != cudaSuccess) n = 0;
    }
    cudaGetLastError();
    return n < 1 ? 1 : n;
  };
  pairs = clusters(2);
  fours = clusters(4);
  g_dev[dev].sms.store(sms, std::memory_order_relaxed);
  g_dev[dev].pairs.store(pairs, std::memory_order_relaxed);
  g_dev[dev].fours.store(fours, std::memory_order_relaxed);
}

template <int EPI, int CL, bool kSums, bool kSplit>
cudaError_t launch_t(const CUtensorMap& mA, const CUtensorMap& mB, const CUtensorMap& mD, const NsArgs& a, int grid,
                     cudaStream_t s) {
  size_t smem = 1024 + kStgBytes + static_cast<size_t>(a.stages) * ((a.a_halves * 2 + a.b_halves * (a.BN / CL / 64)) * kBox) + (kSplit ? 128 * a.BN * 4 : 0) + kBarBytes;
  if (smem < kLeast) smem = kLeast;
  cudaError_t e = allow_smem(ns_product_kernel<EPI, CL, kSums, kSplit>, kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = config(attr, kSplit ? a.split : CL, grid, smem, s);
  attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
  ++cfg.numAttrs;
  return cudaLaunchKernelEx(&cfg, ns_product_kernel<EPI, CL, kSums, kSplit>, mA, mB, mD, a);
}

template <int EPI, bool kSums>
cudaError_t launch_s(int cl, const CUtensorMap& mA, const CUtensorMap& mB, const CUtensorMap& mD, const NsArgs& a, int grid,
                     cudaStream_t s) {
  return a.split > 1 ? launch_t<EPI, 1, kSums, true>(mA, mB, mD, a, a.units * a.split, s)
         : cl == 2   ? launch_t<EPI, 2, kSums, false>(mA, mB, mD, a, grid, s)
                     : launch_t<EPI, 1, kSums, false>(mA, mB, mD, a, grid, s);
}

template <int EPI>
cudaError_t launch_e(int cl, const CUtensorMap& mA, const CUtensorMap& mB, const CUtensorMap& mD, const NsArgs& a, int grid,
                     cudaStream_t s) {
  return a.a_halves + a.b_halves == 4 ? launch_s<EPI, true>(cl, mA, mB, mD, a, grid, s)
                                      : launch_s<EPI, false>(cl, mA, mB, mD, a, grid, s);
}

}  // namespace

cudaError_t launch_ns_product(int epi, const NsMaps& A, const NsMaps& B, const NsMaps& D, NsArgs a, cudaStream_t s) {
  NsRoom has;
  device_room(has.sms, has.pairs, has.fours);
  const NsShape sh = ns_shape({epi == kNsSym, a.batch, a.M, a.N, a.K, a.a_halves, a.b_halves}, has);
  if (sh.units > INT32_MAX / 4) return cudaErrorInvalidValue;   // refused by the entries
  const int cl = sh.cl;
  a.BN = sh.BN, a.mt = sh.mt, a.nt = sh.nt, a.split = sh.split, a.full = sh.full, a.stages = sh.stages;
  a.units = static_cast<int>(sh.units);
  // K-major boxes of 128 rows where the tile has them: half as many copies
  a.b_rows = a.b_mn || a.BN / cl % 128 ? 64 : 128;
  a.b_loads = a.BN / cl / a.b_rows;
  const CUtensorMap &mA = a.a_mn ? A.load64 : A.load128, &mB = a.b_rows == 64 ? B.load64 : B.load128, &mD = D.store;
  const int room = cl == 2 ? has.pairs : has.sms, grid = (a.units < room ? a.units : room) * cl;
  switch (epi) {
    case kNsSym: return launch_e<kNsSym>(cl, mA, mB, mD, a, grid, s);
    case kNsStep: return launch_e<kNsStep>(cl, mA, mB, mD, a, grid, s);
    default: return launch_e<kNsLast>(cl, mA, mB, mD, a, grid, s);
  }
}

}  // namespace oscars
