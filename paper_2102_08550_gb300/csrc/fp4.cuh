// Matrices in 4 bits: where their parts lie, and what their bits mean (include/oscars.h, oscars_quantize_fp4).
#pragma once

#include <cuda_fp16.h>

#include "../../include/oscars.h"
#include "common.cuh"

namespace oscars {

constexpr int kFp4MaxSide = 1 << 30;   // rows, columns, tokens, channels

__host__ __device__ constexpr int fp4_block(int format) { return format == OSCARS_MXFP4 ? 32 : 16; }
// tiles of 4 blocks of a row
__host__ __device__ constexpr int fp4_tiles(int cols, int format) {
  return format == OSCARS_MXFP4 ? (cols + 127) / 128 : (cols + 63) / 64;
}
// bytes of a row's codes, whole groups of 32 columns
__host__ __device__ constexpr int64_t fp4_row_bytes(int cols) { return (static_cast<int64_t>(cols) + 31) / 32 * 16; }
// where the scales of tile j of row i lie (4 bytes)
__host__ __device__ constexpr int64_t fp4_scale_at(int64_t i, int j, int tiles) {
  return ((i >> 7) * tiles + j) * 512 + (i & 31) * 16 + ((i >> 5) & 3) * 4;
}

// 2^(byte - 127), 255 a NaN
__device__ __forceinline__ float e8m0_value(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7FFFFFFFu : byte << 23);
}
// two 8-bit scales as fp16 (exact)
__device__ __forceinline__ __half2 e4m3_pair(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
  return *reinterpret_cast<const __half2*>(&h);
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) { return __low2float(e4m3_pair(byte & 0xFFu)); }
// eight values to codes, the first in the low bits; ties to even codes, magnitudes over 6 to 6
__device__ __forceinline__ uint32_t eight_codes(const float (&v)[8]) {
  uint32_t w;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(w)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return w;
}
// and back, in pairs (fp16, exact)
__device__ __forceinline__ void eight_values(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
}

}  // namespace oscars
