// Rows in 4 bits: codes with a scale for each block, and back.
//
//   MX: e = floor(log2 |block|) - 2, c = e2m1(x 2^-e)
//   NV: t = |row| / 2688, b = e4m3(|block| / (6 t)), c = e2m1(x / (b t))
//
// A thread takes eight neighbouring values, so that a warp's loads are whole lines and its codes too; a block's
// threads (two or four) meet in shuffles, and the four scales of a tile's row are written by one of them.
// Bound by memory: values in, codes and scales out (or the other way round).
#include "common.cuh"
#include "fp4.cuh"
#include "internal.h"
#include "rows.cuh"

namespace oscars {

namespace {

constexpr int kThreads = 256, kKeep = 4;

__device__ __forceinline__ uint32_t magnitude8(const float (&v)[8]) {   // in order, infinity above every number and NaN above it
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  return m;
}

struct QuantArgs {
  const void* x;
  uint8_t *q, *scales;
  float* row_scale;
  int64_t ldx, ldq, units;   // units (OSCARS_MXFP4): half warps of 128 columns
  int rows, cols, tiles, vec;
};

// ------------------------------------------------------------------ OSCARS_MXFP4
// Blocks are on their own: a half warp takes 128 columns of a row, a tile's four blocks.
template <typename T>
__global__ void __launch_bounds__(kThreads) quantize_mx_kernel(const __grid_constant__ QuantArgs a) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 15;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (kThreads / 16), whole = (a.units + 1) / 2 * 2;   // whole warps
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kThreads / 16) + threadIdx.x / 16; u < whole; u += step) {
    const bool live = u < a.units;
    const int64_t row = live ? u / a.tiles : 0;
    const int tile = live ? static_cast<int>(u - row * a.tiles) : 0, at = tile * 128 + lane * 8;
    float v[8];
    load8(static_cast<const T*>(a.x) + row * a.ldx + at, live ? a.cols - at : 0, a.vec, v);
    uint32_t m = magnitude8(v);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const uint32_t exp = m >> 23;
    const bool number = exp < 255;
    const uint32_t byte = number ? (exp > 2 ? exp - 2 : 0) : 255;
    // 2^-e: from 2^127 (byte 0) to 2^-125
    const float to = __uint_as_float((254 - byte) << 23);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = number ? v[e] * to : 0.f;
    uint32_t word = byte << (8 * ((lane >> 2) & 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
    if (!live) continue;
    if (at / 32 * 32 < a.cols) *reinterpret_cast<uint32_t*>(a.q + row * a.ldq + at / 2) = eight_codes(v);
    if (lane == 0) *reinterpret_cast<uint32_t*>(a.scales + fp4_scale_at(row, tile, a.tiles)) = word;
  }
}

// ------------------------------------------------------------------ OSCARS_NVFP4
// A row on TPR threads; up to kKeep turns stay in registers between the row's maximum and the codes.
template <typename T, int TPR>
__global__ void __launch_bounds__(kThreads) quantize_nv_kernel(const __grid_constant__ QuantArgs a) {
  constexpr int kRows = kThreads / TPR;
  __shared__ uint32_t part[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / TPR;
  const int t = threadIdx.x % TPR, turns = (a.cols + TPR * 8 - 1) / (TPR * 8);
  if (TPR == 32 && row >= a.rows) return;
  const bool live = row < a.rows;
  const T* x = static_cast<const T*>(a.x) + (live ? row : 0) * a.ldx;
  Held8<T> held[kKeep];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kKeep; ++i) held[i].load(x + (i * TPR + t) * 8, a.cols - (i * TPR + t) * 8, a.vec);
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    float v[8];
    held[i].get(v);
    m = max(m, magnitude8(v));
  }
  for (int i = kKeep; i < turns; ++i) {
    float v[8];
    load8(x + (i * TPR + t) * 8, a.cols - (i * TPR + t) * 8, a.vec, v);
    m = max(m, magnitude8(v));
  }
  m = __reduce_max_sync(0xffffffffu, m);
  if (TPR > 32) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) m = max(m, part[threadIdx.x / TPR * (TPR / 32) + i]);
    if (!live) return;   // whole warps
  }
  const float top = __uint_as_float(m);
  const bool number = m < 0x7F800000u;
  const float scale = m == 0 || !number ? top : fmaxf(top / 2688.f, 0x1p-110f);
  const float g = m == 0 || !number ? 0.f : 1.f / (6.f * scale);
  if (t == 0) a.row_scale[row] = scale;
  uint8_t* q = a.q + row * a.ldq;
  auto write = [&](int at, float (&v)[8]) {   // all lanes of the warp
    uint32_t bm = magnitude8(v);
    bm = max(bm, __shfl_xor_sync(0xffffffffu, bm, 1));
    uint32_t byte = 0;
    if (number) {
      uint16_t b;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(0.f), "f"(fminf(__uint_as_float(bm) * g, 448.f)));
      byte = b & 0xFFu;
    }
    const float s = e4m3_value(byte) * scale, r = byte != 0 ? 1.f / s : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = byte != 0 ? v[e] * r : 0.f;
    uint32_t word = byte << (8 * ((t >> 1) & 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 2);
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    if (at / 32 * 32 < a.cols) *reinterpret_cast<uint32_t*>(q + at / 2) = eight_codes(v);
    if (t % 8 == 0 && at < a.cols) *reinterpret_cast<uint32_t*>(a.scales + fp4_scale_at(row, at / 64, a.tiles)) = word;
  };
#pragma unroll
  for (int i = 0; i < kKeep; ++i)
    if ((i * TPR + t / 32 * 32) * 8 < a.cols) {
      float v[8];
      held[i].get(v);
      write((i * TPR + t) * 8, v);
    }
  for (int i = kKeep; i < turns; ++i) {
    if ((i * TPR + t / 32 * 32) * 8 >= a.cols) break;
    float v[8];
    load8(x + (i * TPR + t) * 8, a.cols - (i * TPR + t) * 8, a.vec, v);
    write((i * TPR + t) * 8, v);
  }
}

// ------------------------------------------------------------------ back
struct DequantArgs {
  const uint8_t *q, *scales;
  const float* row_scale;
  void* x;
  int64_t ldq, ldx, units;   // units of eight columns
  int rows, cols, tiles, vec, mx, per;   // per: units of a row
};

template <typename T>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const __grid_constant__ DequantArgs a) {
  pdl_wait();
  pdl_trigger();
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; u < a.units; u += static_cast<int64_t>(gridDim.x) * kThreads) {
    const int64_t row = u / a.per;
    const int at = static_cast<int>(u - row * a.per) * 8;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(a.q + row * a.ldq + at / 2);
    const int block = at / (a.mx ? 32 : 16);
    const uint32_t byte = a.scales[fp4_scale_at(row, block / 4, a.tiles) + block % 4];
    const float s = a.mx ? e8m0_value(byte) : e4m3_value(byte), t = a.row_scale ? a.row_scale[row] : 1.f;
    uint32_t h[4];
    eight_values(w, h);
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
      v[2 * i] = f.x * s * t;
      v[2 * i + 1] = f.y * s * t;
    }
    T* to = static_cast<T*>(a.x) + row * a.ldx + at;
    store8(to, a.cols - at, a.vec, v);
  }
}

bool at_bytes(const void* p, int n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool format_ok(int f) { return f == OSCARS_MXFP4 || f == OSCARS_NVFP4; }
bool sizes_ok(int rows, int cols, int format) {
  return rows >= 0 && rows <= kFp4MaxSide && cols >= 1 && cols <= kFp4MaxSide && format_ok(format);
}
unsigned blocks_for(int64_t n, int per) {
  const int64_t b = (n + per - 1) / per;
  return static_cast<unsigned>(b < (1 << 30) ? b : 1 << 30);
}

template <typename T>
cudaError_t quantize(const QuantArgs& a, int format, cudaStream_t s) {
  if (format == OSCARS_MXFP4) return launch_dependent(quantize_mx_kernel<T>, dim3(blocks_for(a.units, kThreads / 16)), kThreads, 0, s, a);
  if (a.cols <= 32 * 8 * kKeep) return launch_dependent(quantize_nv_kernel<T, 32>, dim3((a.rows + 7) / 8), kThreads, 0, s, a);
  if (a.cols <= 128 * 8 * kKeep) return launch_dependent(quantize_nv_kernel<T, 128>, dim3((a.rows + 1) / 2), kThreads, 0, s, a);
  return launch_dependent(quantize_nv_kernel<T, kThreads>, dim3(a.rows), kThreads, 0, s, a);
}

}  // namespace
}  // namespace oscars

using namespace oscars;

extern "C" {

oscars_status oscars_fp4_scale_bytes(int32_t rows, int32_t cols, int32_t format, int64_t* bytes) {
  if (!bytes || !sizes_ok(rows, cols, format)) return OSCARS_EINVAL;
  *bytes = (static_cast<int64_t>(rows) + 127) / 128 * fp4_tiles(cols, format) * 512;
  return OSCARS_OK;
}

oscars_status oscars_quantize_fp4(const void* x, int64_t ldx, int32_t dtype, int32_t rows, int32_t cols, int32_t format, uint8_t* q,
                                  int64_t ldq, uint8_t* scales, float* row_scale, void* stream) {
  if (!sizes_ok(rows, cols, format) || (dtype != OSCARS_F32 && dtype != OSCARS_BF16) || ldx < cols || ldq % 16 || ldq < fp4_row_bytes(cols))
    return OSCARS_EINVAL;
  if (rows == 0) return OSCARS_OK;
  const int size = dtype == OSCARS_F32 ? 4 : 2;
  if (!x || !q || !scales || !at_bytes(x, size) || !at_bytes(q, 16) || !at_bytes(scales, 16) || !at_bytes(row_scale, 4) ||
      (format == OSCARS_NVFP4) != (row_scale != nullptr))
    return OSCARS_EINVAL;
  const int tiles = fp4_tiles(cols, format);
  QuantArgs a{x, q, scales, row_scale, ldx, ldq, static_cast<int64_t>(rows) * tiles, rows, cols, tiles,
              at_bytes(x, 16) && ldx * size % 16 == 0};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == OSCARS_F32 ? quantize<float>(a, format, s) : quantize<__nv_bfloat16>(a, format, s);
  return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

oscars_status oscars_dequantize_fp4(const uint8_t* q, int64_t ldq, const uint8_t* scales, const float* row_scale, int32_t format,
                                    int32_t rows, int32_t cols, void* x, int64_t ldx, int32_t dtype, void* stream) {
  if (!sizes_ok(rows, cols, format) || (dtype != OSCARS_F32 && dtype != OSCARS_BF16) || ldx < cols || ldq % 16 || ldq < fp4_row_bytes(cols))
    return OSCARS_EINVAL;
  if (rows == 0) return OSCARS_OK;
  const int size = dtype == OSCARS_F32 ? 4 : 2;
  if (!x || !q || !scales || !at_bytes(x, size) || !at_bytes(q, 16) || !at_bytes(scales, 16) || !at_bytes(row_scale, 4)) return OSCARS_EINVAL;
  const int per = (cols + 7) / 8;
  DequantArgs a{q, scales, row_scale, x, ldq, ldx, static_cast<int64_t>(rows) * per, rows, cols, fp4_tiles(cols, format),
                at_bytes(x, 16) && ldx * size % 16 == 0, format == OSCARS_MXFP4, per};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const dim3 grid(blocks_for(a.units, kThreads));
  const cudaError_t e = dtype == OSCARS_F32 ? launch_dependent(dequantize_kernel<float>, grid, kThreads, 0, s, a)
                                            : launch_dependent(dequantize_kernel<__nv_bfloat16>, grid, kThreads, 0, s, a);
  return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

}  // extern "C"
