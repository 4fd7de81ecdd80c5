// Layer norm, forward and backward, of groups of rows with parameters of their own.
//
//   y = (x - mean) rstd gamma + beta,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   dx = rstd (h - mean(h) - xh mean(h xh)),  h = dy gamma,  xh = (x - mean) rstd
//   dgamma = sum over the group's rows of dy xh,  dbeta = sum of dy
//
// Bound by memory: forward reads x and writes y, backward reads dy and x and writes dx.  8192 x 4096 bf16 forward 24.3 us (5.5
// TB/s; a copy of as many bytes 21.1), 16384 x 4096 bf16 backward 67.4 us (6.0 TB/s; twice the rows 124 us, 6.5 TB/s).
// Additions, products and their sums go two at a time (f32x2), which takes half the issue slots.
#include <type_traits>

#include "../../include/oscars.h"
#include "common.cuh"
#include "internal.h"
#include "rows.cuh"

namespace oscars {

namespace {

constexpr int kMaxSide = 1 << 30, kMaxGroups = 65535;
constexpr int kThreads = 256;

// the sum of a value over a block of kThreads, in each of them, in a fixed order
__device__ __forceinline__ float block_sum(float v, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) v += part[i];
  __syncthreads();
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

// ------------------------------------------------------------------ rows through shared memory
// Up to 8192 columns: TPR threads take a row, a block 512 / TPR rows at a time; a thread owns 8 kTurns columns.  kMats matrices'
// rows come through a ring in shared memory in which each thread reads what it has copied itself (cp.async, no barrier).
// Where rows are not 16-byte aligned, neighbouring threads take neighbouring columns.  Up to five rows at a time are copied from
// the 16 bytes on in which they begin, with a barrier of the row's threads in between (2991 x 5541 fp32 backward 47 us, 56
// without); more rows at a time hide the latency of loads of single values when they are due (16030 x 22 fp32 7.8 us, 11 copied).
constexpr int kBlock = 512;

__device__ __forceinline__ void copy16(void* to, const void* from, int bytes) {   // zeros behind the first `bytes`
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy16(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }


template <typename T, int TPR, int kTurns, bool kVec, int kMats>
struct Rows {
  static constexpr int kSize = sizeof(T), kLanes = kBlock / TPR, kCap = TPR * kTurns * 8;
  static constexpr int kPieces = kTurns * kSize / 2;          // of 16 bytes, of a thread's columns of one matrix
  static constexpr int kRow = kCap * kSize + 16;              // a row and what lies in front of it in its first 16 bytes
  static constexpr bool kDirect = !kVec && kLanes > 5;
  static constexpr int kStage = kMats * (kVec ? kPieces * kBlock * 16 : kLanes * kRow);
  static constexpr int kDepth = kDirect ? 1 : 200704 / kStage < 6 ? 200704 / kStage : 6;
  static constexpr int kBytes = kDirect ? 0 : kDepth * kStage;

  static constexpr int kPer = kVec ? 16 / static_cast<int>(sizeof(T)) : 1;         // neighbouring columns of a thread
  __device__ __forceinline__ static int column(int i, int e) {
    const int t = threadIdx.x % TPR, c = i * 8 + e;
    return (c / kPer * TPR + t) * kPer + c % kPer;
  }
  __device__ __forceinline__ static int in_front(const T* row) { return static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15); }
  __device__ __forceinline__ static uint8_t* lane_row(uint8_t* ring, int stage, int m) {
    return ring + stage * kStage + (m * kLanes + threadIdx.x / TPR) * kRow;
  }
  // a row's threads are here, and each of them sees what the others have copied
  __device__ __forceinline__ static void meet() {
    if (TPR == 32) __syncwarp();
    else bar_named(1 + threadIdx.x / TPR, TPR);
  }
  // whether all of this thread's columns are inside the row
  __device__ __forceinline__ static bool inside(int cols) { return column(kTurns - 1, 7) < cols; }
  // Turn i's columns are those from i TPR 8 on, of all of a row's threads: none of them, some or all are inside the row, the same
  // for all threads.  kFull: all are, of every turn.  (With two turns alone the questions cost more than they save: 4104 columns of
  // bf16 backward 89 us for 75.)
  static constexpr bool kByTurn = kTurns > 2;
  template <bool kFull>
  __device__ __forceinline__ static bool none(int i, int cols) { return kByTurn && !kFull && i * TPR * 8 >= cols; }
  template <bool kFull>
  __device__ __forceinline__ static bool whole(int i, int cols) { return kFull || (kByTurn && (i + 1) * TPR * 8 <= cols); }
  // begin the copy of row `row` of a matrix that starts at `first` to a stage
  template <bool kFull>
  __device__ __forceinline__ static void request(uint8_t* ring, int stage, int m, const T* row, const T* first, int cols) {
    constexpr int kPiece = 16 / kSize;                       // columns of 16 bytes
    if constexpr (kVec) {
      uint8_t* to = ring + stage * kStage + (m * kPieces * kBlock + threadIdx.x) * 16;
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        constexpr int kAtOnce = 8 / kPiece;                    // pieces of a turn
        const int at = column(p * kPiece / 8, p * kPiece % 8), left = (cols - at) * kSize;
        if (none<kFull>(p / kAtOnce, cols)) continue;
        if (kFull || left >= 16) copy16(to + p * kBlock * 16, row + at);
        else copy16(to + p * kBlock * 16, row + (left > 0 ? at : 0), left > 0 ? left : 0);
      }
    } else if constexpr (!kDirect) {   // whole 16 bytes, with a piece of the row before in front; the matrix's own first ones one at a time
      const int t = threadIdx.x % TPR, front = in_front(row), bytes = front + cols * kSize;
      uint8_t* to = lane_row(ring, stage, m);
      const uint8_t* from = reinterpret_cast<const uint8_t*>(row) - front;
      const bool inside = from >= reinterpret_cast<const uint8_t*>(first);
      if (!inside && t < (16 - front) / kSize && t < cols) reinterpret_cast<T*>(to + front)[t] = row[t];
      for (int at = t * 16; at < bytes; at += TPR * 16)
        if (inside || at > 0) copy16(to + at, from + at, bytes - at >= 16 ? 16 : bytes - at);
    }
  }
  // this thread's columns of it, of turns that have some (zeros behind the row's end)
  template <bool kFull>
  __device__ __forceinline__ static void take(uint8_t* ring, int stage, int m, const T* row, int cols, float2 (&v)[kTurns][4]) {
    if constexpr (kVec) {
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        if (none<kFull>(p * kTurns / kPieces, cols)) continue;
        const uint4 w = *reinterpret_cast<const uint4*>(ring + stage * kStage + ((m * kPieces + p) * kBlock + threadIdx.x) * 16);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int i = 0; i < 2; ++i) v[p / 2][p % 2 * 2 + i] = make_float2(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[p][i] = make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xFFFF0000u));
        }
      }
    } else {
      const T* from = kDirect ? row : reinterpret_cast<const T*>(lane_row(ring, stage, m) + in_front(row));
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        if (none<kFull>(i, cols)) continue;
        if (whole<kFull>(i, cols)) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[i][e] = make_float2(to_f32(from[column(i, 2 * e)]), to_f32(from[column(i, 2 * e + 1)]));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[i][e] = make_float2(column(i, 2 * e) < cols ? to_f32(from[column(i, 2 * e)]) : 0.f,
                                  column(i, 2 * e + 1) < cols ? to_f32(from[column(i, 2 * e + 1)]) : 0.f);
        }
      }
    }
  }
  template <bool kFull>
  __device__ __forceinline__ static void put(T* row, int cols, const float2 (&v)[kTurns][4]) {
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      if (none<kFull>(i, cols)) continue;
      const float w[8] = {v[i][0].x, v[i][0].y, v[i][1].x, v[i][1].y, v[i][2].x, v[i][2].y, v[i][3].x, v[i][3].y};
      if (!kFull && column(i, 7) >= cols) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (column(i, e) < cols) row[column(i, e)] = static_cast<T>(w[e]);
      } else if constexpr (kVec && sizeof(T) == 2) {
        store8(row + column(i, 0), 8, true, w);
      } else if constexpr (kVec) {
#pragma unroll
        for (int h = 0; h < 8; h += 4) *reinterpret_cast<float4*>(row + column(i, h)) = make_float4(w[h], w[h + 1], w[h + 2], w[h + 3]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) row[column(i, e)] = static_cast<T>(w[e]);
      }
    }
  }
  // a group's parameters, or `none` if there are none
  __device__ __forceinline__ static void params(const float* p, int cols, bool vec, float none, float2 (&v)[kTurns][4]) {
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      float w[8];
      if (kVec && p && vec && (i + 1) * TPR * 8 <= cols) {
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
          const float4 f = *reinterpret_cast<const float4*>(p + column(i, h));
          w[h] = f.x, w[h + 1] = f.y, w[h + 2] = f.z, w[h + 3] = f.w;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = p && column(i, e) < cols ? p[column(i, e)] : none;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = make_float2(w[2 * e], w[2 * e + 1]);
    }
  }
};

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// Sums of N values over a row's threads, in each of them, in a fixed order.  `parts` alternates between two places, so that one
// barrier is enough: a sum's parts are read before those of the one after the next are written.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*parts)[2]) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
  if (TPR > 32) {
    const int lane = threadIdx.x / TPR, t = threadIdx.x % TPR;
    float(*part)[2] = parts + lane * (TPR / 32);
    if ((t & 31) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) part[t >> 5][n] = v[n];
    bar_named(1 + lane, TPR);
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = part[0][n];
#pragma unroll
    for (int i = 1; i < TPR / 32; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] += part[i][n];
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
  int groups, chunks, per;            // per: rows of a chunk
};

// 1 / sqrt(v) of a normal number: the approximation (2 steps off) and one Newton step
__device__ __forceinline__ float inverse_sqrt(float v) {
  const float r = rsqrtf(v);
  return fmaf(r * 0.5f, fmaf(-v * r, r, 1.f), r);
}

// Sum of squares in the whole range of fp32 only where the plain one left it.
__device__ __forceinline__ float inverse_std(const Squares& s, int cols, float eps) {
  if (s.big == 0.f && s.small == 0.f && eps >= 0x1p-120f) return 1.f / sqrtf(s.mid / cols + eps);
  return static_cast<float>(1.0 / sqrt(s.total() / cols + eps));
}

// Mean and squares of deviations from registers: two exchanges between a row's threads, each behind one barrier, are what a row
// waits for, so that four rows at a time or more are under way.  Rows that fill all turns (kFull) go without bounds: 8192 x 4096 bf16
// 30.0 -> 24.2 us.
template <typename T, int TPR, int kTurns, bool kVec, bool kFull>
__global__ void __launch_bounds__(kBlock, 1) layer_norm_kernel(const __grid_constant__ FwdArgs a) {
  using R = Rows<T, TPR, kTurns, kVec, 1>;
  constexpr int kD = R::kDepth;
  extern __shared__ __align__(16) uint8_t fwd_smem[];
  __shared__ float parts[2][kBlock / 32][2];
  const int t = threadIdx.x % TPR, lane = threadIdx.x / TPR;
  const int group = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int r1 = min((chunk + 1) * a.per, a.rows);
  const int64_t first = static_cast<int64_t>(group) * a.rows;
  pdl_wait();
  pdl_trigger();
  const T* x = static_cast<const T*>(a.x) + first * a.ldx;
  auto request = [&](int r, int stage) {
    if (r < r1) R::template request<kFull>(fwd_smem, stage, 0, x + r * a.ldx, static_cast<const T*>(a.x), a.cols);
    copies_done();
  };
  int r = chunk * a.per + lane;
#pragma unroll
  for (int i = 0; i < kD - 1; ++i) request(r + i * R::kLanes, i);
  float2 g[kTurns][4], b[kTurns][4];
  R::params(a.gamma ? a.gamma + group * a.pstride : nullptr, a.cols, a.pvec, 1.f, g);
  R::params(a.beta ? a.beta + group * a.pstride : nullptr, a.cols, a.pvec, 0.f, b);
  const float each = 1.f / a.cols;
  for (int stage = 0; r < r1; r += R::kLanes) {
    request(r + (kD - 1) * R::kLanes, stage == 0 ? kD - 1 : stage - 1);
    copies_wait<kD - 1>();
    if constexpr (!kVec && !R::kDirect) R::meet();
    float2 v[kTurns][4];
    R::template take<kFull>(fwd_smem, stage, 0, x + r * a.ldx, a.cols, v);
    float2 pair = both(0.f);
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
      if (!R::template none<kFull>(i, a.cols)) pair = __fadd2_rn(pair, __fadd2_rn(__fadd2_rn(v[i][0], v[i][1]), __fadd2_rn(v[i][2], v[i][3])));
    float sum[1] = {pair.x + pair.y}, none[1] = {0.f};
    row_sums<TPR>(sum, parts[0]);
    float mean = sum[0] * each;
    mean = fmaf(fmaf(-mean, static_cast<float>(a.cols), sum[0]), each, mean);   // the quotient, whatever 1 / cols was rounded to
    if (!(fabsf(sum[0]) < 0x1p127f)) {   // the sum may have left fp32 where the mean does not; all of the row's threads come here
      sum[0] = 0.f;
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        if (R::template none<kFull>(i, a.cols)) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[0] += v[i][e].x * 0x1p-32f + v[i][e].y * 0x1p-32f;
      }
      row_sums<TPR>(sum, parts[1]);
      mean = sum[0] / a.cols * 0x1p32f;
      row_sums<TPR>(none, parts[0]);   // keeps the two places in turn
    }
    Squares sq;
    bool plain = true;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      if (R::template none<kFull>(i, a.cols)) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = __fadd2_rn(v[i][e], both(-mean));
      if (!kFull && R::column(i, 7) >= a.cols) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (R::column(i, 2 * e) >= a.cols) v[i][e].x = 0.f;
          if (R::column(i, 2 * e + 1) >= a.cols) v[i][e].y = 0.f;
        }
      }
      float2 s = both(0.f);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __ffma2_rn(v[i][e], v[i][e], s);
      sq.mid += s.x + s.y;
      plain = plain && ((s.x + s.y > 1e-20f && s.x + s.y < 1e25f) || R::column(i, 0) >= a.cols);
    }
    if (!plain) {   // squares may have left fp32's range, or are zeros
      sq.mid = 0.f;
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        if (R::template none<kFull>(i, a.cols)) continue;
        const float w[8] = {v[i][0].x, v[i][0].y, v[i][1].x, v[i][1].y, v[i][2].x, v[i][2].y, v[i][3].x, v[i][3].y};
        sq.add(w);
      }
    }
    float two[2] = {sq.mid, sq.big != 0.f || sq.small != 0.f ? 1.f : 0.f};
    row_sums<TPR>(two, parts[1]);
    float rstd = inverse_sqrt(fmaf(two[0], each, a.eps));
    if (two[1] != 0.f || !(a.eps >= 0x1p-120f)) {
      float far[2] = {sq.big, sq.small};
      row_sums<TPR>(far, parts[0]);
      row_sums<TPR>(none, parts[1]);
      sq.mid = two[0], sq.big = far[0], sq.small = far[1];
      rstd = inverse_std(sq, a.cols, a.eps);
    }
    if (t == 0) {
      if (a.mean) a.mean[first + r] = mean;
      if (a.rstd) a.rstd[first + r] = rstd;
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      if (R::template none<kFull>(i, a.cols)) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = __ffma2_rn(__fmul2_rn(v[i][e], both(rstd)), g[i][e], b[i][e]);
    }
    R::template put<kFull>(static_cast<T*>(a.y) + (first + r) * a.ldy, a.cols, v);
    if (++stage >= kD) stage = 0;
  }
}

// Wide rows: a block each, read again from L2 for the squares and for the result.
template <typename T>
__global__ void __launch_bounds__(kThreads) wide_norm_kernel(const __grid_constant__ FwdArgs a) {
  __shared__ float part[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  T* y = static_cast<T*>(a.y) + row * a.ldy;
  const int64_t group = row / a.rows;
  const float *gamma = a.gamma ? a.gamma + group * a.pstride : nullptr, *beta = a.beta ? a.beta + group * a.pstride : nullptr;
  auto each = [&](auto&& f) {   // f(first column, its 8 values), zeros behind the row's end
    for (int64_t at = threadIdx.x * 8; at < a.cols; at += kThreads * 8) {
      float v[8];
      load8(x + at, a.cols - static_cast<int>(at), a.xvec, v);
      f(static_cast<int>(at), v);
    }
  };
  float sum = 0.f;
  each([&](int, float (&v)[8]) { sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); });
  sum = block_sum(sum, part);
  float mean = sum / a.cols;
  if (!(fabsf(sum) < INFINITY)) {
    sum = 0.f;
    each([&](int, float (&v)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += v[e] * 0x1p-32f;
    });
    sum = block_sum(sum, part);
    mean = sum / a.cols * 0x1p32f;
  }
  Squares sq;
  each([&](int at, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = at + e < a.cols ? v[e] - mean : 0.f;
    sq.add(v);
  });
  sq.mid = block_sum(sq.mid, part);
  sq.big = block_sum(sq.big, part);
  sq.small = block_sum(sq.small, part);
  const float rstd = inverse_std(sq, a.cols, a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  each([&](int at, float (&v)[8]) {
    float g[8], b[8];
    params8(gamma, at, a.cols, a.pvec, 1.f, g);
    params8(beta, at, a.cols, a.pvec, 0.f, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fmaf((v[e] - mean) * rstd, g[e], b[e]);
    store8(y + at, a.cols - at, a.yvec, v);
  });
}

constexpr int kWide = 8192;       // columns that one pass takes

// Calls f with a row's threads and each one's turns as types.  What a row costs beside its values (sums over the threads, the
// copies' addresses) is as much as about 16 values a thread: the forward pass has 32 a thread, the backward pass, which
// keeps more of each in registers, 16.
template <int kTurns, typename F>
cudaError_t by_width(int cols, F&& f) {
  using std::integral_constant;
  constexpr int kWarp = 32 * 8 * kTurns;   // columns of a warp
  auto warps = [&](auto n) { return f(integral_constant<int, 32 * n()>(), integral_constant<int, kTurns>()); };
  if (cols <= 256) return f(integral_constant<int, 32>(), integral_constant<int, 1>());
  if (cols <= 512) return f(integral_constant<int, 32>(), integral_constant<int, 2>());
  // fewer idle threads, more rows at a time: 9746 x 4104 bf16 forward 45 us on five warps a row, 60 on eight
  if constexpr (kTurns == 2) {
    if (cols <= 2 * kWarp) return warps(integral_constant<int, 2>());
  } else {
    if (cols <= kWarp) return warps(integral_constant<int, 1>());
    if (cols <= 2 * kWarp) return warps(integral_constant<int, 2>());
    if (cols <= 3 * kWarp) return warps(integral_constant<int, 3>());
  }
  if (cols <= 4 * kWarp) return warps(integral_constant<int, 4>());
  if constexpr (kTurns == 4) {
    if (cols <= 5 * kWarp) return warps(integral_constant<int, 5>());
  }
  if (cols <= 6 * kWarp) return warps(integral_constant<int, 6>());
  if (cols <= 8 * kWarp) return warps(integral_constant<int, 8>());
  if constexpr (kTurns == 2) {
    if (cols <= 10 * kWarp) return warps(integral_constant<int, 10>());
    if (cols <= 12 * kWarp) return warps(integral_constant<int, 12>());
    return warps(integral_constant<int, 16>());
  }
  return cudaErrorInvalidValue;
}
// rows that a block takes at a time
template <int kTurns>
int lanes_of(int cols) {
  int lanes = 1;
  by_width<kTurns>(cols, [&](auto tpr, auto) {
    lanes = kBlock / tpr();
    return cudaSuccess;
  });
  return lanes;
}
constexpr int kForward = 4, kBackward = 2;

template <typename T, bool kVec>
cudaError_t forward_rows(const FwdArgs& a, cudaStream_t s) {
  return by_width<kForward>(a.cols, [&](auto tpr, auto turns) {
    constexpr int kBytes = Rows<T, tpr(), turns(), kVec, 1>::kBytes;
    auto launch = [&](auto kernel) {
      const cudaError_t e = allow_smem(kernel, kBytes);
      return e != cudaSuccess ? e : launch_dependent(kernel, dim3(static_cast<unsigned>(a.groups) * a.chunks), kBlock / tpr() * tpr(), kBytes, s, a);
    };
    if (kVec && a.cols == tpr() * turns() * 8) return launch(layer_norm_kernel<T, tpr(), turns(), kVec, kVec>);
    return launch(layer_norm_kernel<T, tpr(), turns(), kVec, false>);
  });
}

template <typename T>
cudaError_t forward(FwdArgs a, cudaStream_t s) {
  if (a.cols > kWide) return launch_dependent(wide_norm_kernel<T>, dim3(static_cast<unsigned>(a.total)), kThreads, 0, s, a);
  // a block an SM, each with a row for all of its lanes at least
  const int lanes = lanes_of<kForward>(a.cols);
  int64_t chunks = 152 / a.groups;
  const int64_t most = (static_cast<int64_t>(a.rows) + lanes - 1) / lanes;
  chunks = chunks < most ? chunks : most;
  if (chunks < 1) chunks = 1;
  a.per = static_cast<int>((a.rows + chunks - 1) / chunks);
  a.chunks = (a.rows + a.per - 1) / a.per;
  return a.xvec && a.yvec ? forward_rows<T, true>(a, s) : forward_rows<T, false>(a, s);
}

// ------------------------------------------------------------------ backward, any number of columns
struct BwdArgs {
  const void *dy, *x;
  void* dx;
  const float *gamma, *mean, *rstd;
  float *dgamma, *dbeta, *part;       // part: [group][chunk][2][cols]
  int64_t lddy, ldx, lddx, pstride, dstride, total;
  int groups, rows, cols, chunks, per;   // per: rows of a chunk
  int dyvec, xvec, dxvec, pvec, clustered;
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
  each([&](int at, float (&h)[8], float (&xh)[8]) {   // eight at a time: n / 2048 additions in sequence
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at + e < a.cols) t = fmaf(h[e], xh[e], t);   // (h is 0 behind the row's end, and xh may be infinite)
    sh += ((h[0] + h[1]) + (h[2] + h[3])) + ((h[4] + h[5]) + (h[6] + h[7]));
    shx += t;
  });
  sh = block_sum(sh, part) / a.cols;
  shx = block_sum(shx, part) / a.cols;
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

// The sums of up to eight chunks, a column a thread, in their order.
constexpr int kFewChunks = 8;
__global__ void __launch_bounds__(kThreads) norm_join_few_kernel(const __grid_constant__ BwdArgs a) {
  pdl_wait();
  pdl_trigger();
  const int64_t col = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const int group = blockIdx.z, which = blockIdx.y;
  float* to = which == 0 ? a.dgamma : a.dbeta;
  if (!to || col >= a.cols) return;
  const float* from = a.part + (static_cast<int64_t>(group) * a.chunks * 2 + which) * a.cols + col;
  float v[kFewChunks];
#pragma unroll
  for (int i = 0; i < kFewChunks; ++i) v[i] = i < a.chunks ? from[static_cast<int64_t>(i) * 2 * a.cols] : 0.f;
#pragma unroll
  for (int i = 1; i < kFewChunks; ++i) v[0] += v[i];
  to[group * a.dstride + col] = v[0];
}

// The chunks' sums of a column, kJoinLanes threads a column, in a fixed order.  32 where a call has more chunks than 64, so that
// they are requested together (152 chunks of 16384 x 4096: 67.7 us for 69.5 with eight; 64 of 64 x 8192 fp32: 8.8 us for 7.6).
template <int kJoinLanes>
__global__ void __launch_bounds__(kColTile * kJoinLanes) norm_join_kernel(const __grid_constant__ BwdArgs a) {
  __shared__ float sums[kJoinLanes][kColTile + 1];
  pdl_wait();
  pdl_trigger();
  const int c = threadIdx.x % kColTile, lane = threadIdx.x / kColTile;
  const int64_t col = static_cast<int64_t>(blockIdx.x) * kColTile + c;
  const int group = blockIdx.z, which = blockIdx.y;
  float* to = which == 0 ? a.dgamma : a.dbeta;
  if (!to) return;
  float s = 0.f;
  if (col < a.cols) {
    const float* from = a.part + (static_cast<int64_t>(group) * a.chunks * 2 + which) * a.cols + col;
#pragma unroll 5
    for (int i = lane; i < a.chunks; i += kJoinLanes) s += from[static_cast<int64_t>(i) * 2 * a.cols];
  }
  sums[lane][c] = s;
  __syncthreads();
  if constexpr (kJoinLanes == 32) {   // a warp takes a column: its lanes' sums meet in shuffles
    s = sums[c][lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int64_t out = static_cast<int64_t>(blockIdx.x) * kColTile + lane;
    if (c == 0 && out < a.cols) to[group * a.dstride + out] = s;
  } else if (lane == 0 && col < a.cols) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kJoinLanes; ++i) s += sums[i][c];
    to[group * a.dstride + col] = s;
  }
}

// ------------------------------------------------------------------ backward, up to 8192 columns
// One pass: a CTA takes a chunk of a group's rows, and a thread's columns' sums over them stay in its registers.
// A group's chunks meet in a cluster of up to eight CTAs, or, of a large call, in the workspace and a second kernel.
template <typename T, int TPR, int kTurns, bool kVec>
constexpr int backward_smem() {
  using R = Rows<T, TPR, kTurns, kVec, 2>;
  constexpr int sums = 2 * R::kLanes * R::kCap * 4;   // at the end
  return R::kBytes > sums ? R::kBytes : sums;
}

template <typename T, int TPR, int kTurns, bool kVec>
__global__ void __launch_bounds__(kBlock, 1) norm_backward_kernel(const __grid_constant__ BwdArgs a) {
  using R = Rows<T, TPR, kTurns, kVec, 2>;
  constexpr int kLanes = R::kLanes, kD = R::kDepth, kCap = R::kCap, kUsed = kLanes * TPR;   // kUsed: threads of the block
  extern __shared__ __align__(16) uint8_t bwd_smem[];
  __shared__ float parts[2][kBlock / 32][2];
  const int lane = threadIdx.x / TPR;
  const int group = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int r1 = min((chunk + 1) * a.per, a.rows);
  const int64_t first = static_cast<int64_t>(group) * a.rows;
  if (a.clustered) cluster_arrive();   // waited for before the sums of the peers are read
  pdl_wait();
  pdl_trigger();
  const T *dy = static_cast<const T*>(a.dy) + first * a.lddy, *x = static_cast<const T*>(a.x) + first * a.ldx;
  float2 dg[kTurns][4] = {}, db[kTurns][4] = {};
  // warps of which all columns are inside the row go without bounds
  auto all_rows = [&](auto with) {
    constexpr bool kFull = with();
    auto request = [&](int r, int stage) {
      if (r < r1) {
        R::template request<kFull>(bwd_smem, stage, 0, dy + r * a.lddy, static_cast<const T*>(a.dy), a.cols);
        R::template request<kFull>(bwd_smem, stage, 1, x + r * a.ldx, static_cast<const T*>(a.x), a.cols);
      }
      copies_done();
    };
    int r = chunk * a.per + lane;
#pragma unroll
    for (int i = 0; i < kD - 1; ++i) request(r + i * kLanes, i);
    float2 g[kTurns][4];
    R::params(a.gamma ? a.gamma + group * a.pstride : nullptr, a.cols, a.pvec, 1.f, g);
    float mean = r < r1 ? a.mean[first + r] : 0.f, rstd = r < r1 ? a.rstd[first + r] : 0.f;
    const float each = 1.f / a.cols;
    for (int it = 0, stage = 0; r < r1; r += kLanes, ++it) {
      request(r + (kD - 1) * kLanes, stage == 0 ? kD - 1 : stage - 1);
      copies_wait<kD - 1>();
      if constexpr (!kVec && !R::kDirect) R::meet();
      float2 h[kTurns][4], xh[kTurns][4];
      R::template take<kFull>(bwd_smem, stage, 0, dy + r * a.lddy, a.cols, h);
      R::template take<kFull>(bwd_smem, stage, 1, x + r * a.ldx, a.cols, xh);
      const float mu = mean, rs = rstd;
      if (r + kLanes < r1) {
        mean = a.mean[first + r + kLanes];
        rstd = a.rstd[first + r + kLanes];
      }
      float2 sh = both(0.f), shx = both(0.f);
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        if (R::template none<kFull>(i, a.cols)) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          xh[i][e] = __fmul2_rn(__fadd2_rn(xh[i][e], both(-mu)), both(rs));
          dg[i][e] = __ffma2_rn(h[i][e], xh[i][e], dg[i][e]);
          db[i][e] = __fadd2_rn(db[i][e], h[i][e]);
          h[i][e] = __fmul2_rn(h[i][e], g[i][e]);
          sh = __fadd2_rn(sh, h[i][e]);
          shx = __ffma2_rn(h[i][e], xh[i][e], shx);
        }
      }
      if (a.dx) {
        float means[2] = {sh.x + sh.y, shx.x + shx.y};
        row_sums<TPR>(means, parts[it & 1]);
        if (!(fabsf(means[1]) < INFINITY)) {
          // Behind the row's end xh is -mean rstd, which may leave fp32 where no column's does (a constant row of 2^126), and 0
          // times that is no number: the sum again, of the columns alone.  All of the row's threads come here.  (16384 x 520 bf16
          // 18.0 us, 17.7 with the fault; 18.9 with xh set to 0 behind the end in every row.  9746 x 4104: 61.9, 61.1, 63.3.)
          float again[1] = {0.f}, turn[1] = {0.f};
#pragma unroll
          for (int i = 0; i < kTurns; ++i) {
            if (R::template none<kFull>(i, a.cols)) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (kFull || R::column(i, 2 * e) < a.cols) again[0] = fmaf(h[i][e].x, xh[i][e].x, again[0]);
              if (kFull || R::column(i, 2 * e + 1) < a.cols) again[0] = fmaf(h[i][e].y, xh[i][e].y, again[0]);
            }
          }
          row_sums<TPR>(again, parts[~it & 1]);
          row_sums<TPR>(turn, parts[it & 1]);   // keeps the two places in turn
          means[1] = again[0];
        }
        const float2 mh = both(-means[0] * each), mhx = both(-means[1] * each);
#pragma unroll
        for (int i = 0; i < kTurns; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!R::template none<kFull>(i, a.cols)) h[i][e] = __fmul2_rn(both(rs), __ffma2_rn(xh[i][e], mhx, __fadd2_rn(h[i][e], mh)));
        R::template put<kFull>(static_cast<T*>(a.dx) + (first + r) * a.lddx, a.cols, h);
      } else if constexpr (!kVec && !R::kDirect) {
        R::meet();   // the stage has been read
      }
      if (++stage >= kD) stage = 0;
    }
  };
  if (kVec && __all_sync(0xffffffffu, R::inside(a.cols))) all_rows(std::bool_constant<kVec>());
  else all_rows(std::false_type());
  if (!a.dgamma && !a.dbeta) {
    if (a.clustered) cluster_wait();
    return;
  }

  // the rows' lanes, then the chunks
  copies_wait<0>();
  __syncthreads();
  float* sums = reinterpret_cast<float*>(bwd_smem);   // [2][kLanes][kCap]
#pragma unroll
  for (int i = 0; i < kTurns; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sums[lane * kCap + R::column(i, e)] = e % 2 == 0 ? dg[i][e / 2].x : dg[i][e / 2].y;
      sums[(kLanes + lane) * kCap + R::column(i, e)] = e % 2 == 0 ? db[i][e / 2].x : db[i][e / 2].y;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * kCap; i += kUsed) {
    const int which = i / kCap, c = i % kCap;
    if (c >= a.cols) continue;
    float* at = sums + which * kLanes * kCap + c;
    float s = 0.f;
#pragma unroll
    for (int l = 0; l < kLanes; ++l) s += at[l * kCap];
    if (a.clustered) {
      *at = s;
    } else {
      float* to = a.chunks > 1 ? a.part + ((static_cast<int64_t>(group) * a.chunks + chunk) * 2 + which) * a.cols
                               : (which == 0 ? a.dgamma : a.dbeta);
      if (to) to[(a.chunks > 1 ? 0 : group * a.dstride) + c] = s;
    }
  }
  if (a.clustered) {
    cluster_wait();    // every CTA of the cluster runs
    cluster_sync();    // and has its sums
    for (int i = chunk * kUsed + threadIdx.x; i < 2 * a.cols; i += a.chunks * kUsed) {
      const int which = i >= a.cols, c = i - which * a.cols;
      float s = 0.f;
      for (int k = 0; k < a.chunks; ++k) s += ld_dsmem_f32(sums + which * kLanes * kCap + c, k);
      float* to = which == 0 ? a.dgamma : a.dbeta;
      if (to) to[group * a.dstride + c] = s;
    }
    cluster_sync();    // no CTA ends while its sums are read
  }
}

// ------------------------------------------------------------------ backward, how it is split
constexpr int kCtas = 152;        // chunks of all groups: one CTA an SM
constexpr int kCluster = 8, kFewRows = 8;

struct Split {
  int chunks, per, clustered;
};
// One pass: a chunk for each SM, each with a row for all of its lanes at least.  Up to 16 chunks of a group are made eight, which
// meet in a cluster, where they are short: up to kFewRows turns cost less than a second launch.
// Wide rows: chunks of columns' tiles enough to fill the card, each of 64 rows or more.
// In both a thread adds up so few rows of its columns in sequence that a term takes at most 256 + rows / 64 additions in all (the
// lanes, and chunks 16 at most).  Where a chunk for each SM would have more: as many as take the least time in waves of an SM
// each, whose beginning and end cost as much as 16 rows (77 x 1000 x 4104 bf16 803 us with a chunk an SM, 614 with as few as the
// bound allows, 479 so; 152 x 700 x 4200, which fills the card without, 578 and 592).
Split split_rows(int groups, int rows, int cols) {
  int64_t want, most;
  const int lanes = cols <= kWide ? lanes_of<kBackward>(cols) : kRowLanes;
  const int64_t run = lanes * (236 - lanes + rows / 64), need = (rows + run - 1) / run;
  bool waves = false;
  if (cols <= kWide) {
    want = kCtas / groups;
    waves = want < need;
    if (waves) {
      auto time = [&](int64_t c) { return (groups * c + kCtas - 1) / kCtas * (rows / (c * lanes) + 16); };
      want = need;
      for (int64_t c = need + 1; c <= 4 * need; ++c)
        if (time(c) < time(want)) want = c;
    }
    most = (static_cast<int64_t>(rows) + lanes - 1) / lanes;
  } else {
    const int64_t tiles = (static_cast<int64_t>(cols) + kColTile - 1) / kColTile * groups;
    want = (1216 + tiles - 1) / tiles;
    want = want > need ? want : need;
    most = (static_cast<int64_t>(rows) + 63) / 64;
  }
  want = want < most ? want : most;
  if (want < 1) want = 1;
  if (cols <= kWide && !waves && want > kCluster && want <= 2 * kCluster && most <= kFewRows * kCluster) want = kCluster;
  Split s;
  s.per = static_cast<int>((rows + want - 1) / want);
  if (s.per < 1) s.per = 1;
  s.chunks = rows > 0 ? (rows + s.per - 1) / s.per : 1;
  s.clustered = cols <= kWide && !waves && s.chunks > 1 && s.chunks <= kCluster;
  return s;
}

int64_t workspace_bytes_of(int groups, int rows, int cols) {
  const Split s = split_rows(groups, rows, cols);
  return s.chunks > 1 && !s.clustered ? static_cast<int64_t>(groups) * s.chunks * 2 * cols * 4 : 0;
}

template <typename T, bool kVec>
cudaError_t one_pass(const BwdArgs& a, cudaStream_t s) {
  return by_width<kBackward>(a.cols, [&](auto tpr, auto turns) {
    constexpr int kBytes = backward_smem<T, tpr(), turns(), kVec>();
    auto kernel = norm_backward_kernel<T, tpr(), turns(), kVec>;
    const cudaError_t e = allow_smem(kernel, kBytes);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.chunks;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.groups) * a.chunks);
    cfg.blockDim = dim3(kBlock / tpr() * tpr());
    cfg.dynamicSmemBytes = kBytes;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = a.clustered ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
  });
}

// (few chunks by blocks of 32 columns too: 100 x 300 x 8192 fp32, three each, 520 us for 475)
cudaError_t join(const BwdArgs& a, cudaStream_t s) {
  if (a.chunks <= kFewChunks) return launch_dependent(norm_join_few_kernel, dim3((a.cols + kThreads - 1) / kThreads, 2, a.groups), kThreads, 0, s, a);
  const dim3 grid((a.cols + kColTile - 1) / kColTile, 2, a.groups);
  return a.chunks > 64 ? launch_dependent(norm_join_kernel<32>, grid, kColTile * 32, 0, s, a)
                       : launch_dependent(norm_join_kernel<8>, grid, kColTile * 8, 0, s, a);
}

template <typename T>
cudaError_t backward(BwdArgs a, cudaStream_t s) {
  const Split split = split_rows(a.groups, a.rows, a.cols);
  a.chunks = split.chunks;
  a.per = split.per;
  a.clustered = split.clustered;
  const bool params = a.dgamma || a.dbeta;
  cudaError_t e;
  if (a.cols <= kWide) {
    e = a.dyvec && a.xvec && (!a.dx || a.dxvec) ? one_pass<T, true>(a, s) : one_pass<T, false>(a, s);
    if (e == cudaSuccess && params && a.chunks > 1 && !a.clustered) e = join(a, s);
    return e;
  }
  e = cudaSuccess;
  if (params) {
    e = launch_dependent(norm_columns_kernel<T>, dim3((a.cols + kColTile - 1) / kColTile, a.chunks, a.groups), kThreads, 0, s, a);
    if (e == cudaSuccess && a.chunks > 1) e = join(a, s);
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
            rows_16(x, ldx, size), rows_16(y, ldy, size), rows_16(gamma, param_stride, 4) && at_bytes(beta, 16), groups, 0, 0};
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
