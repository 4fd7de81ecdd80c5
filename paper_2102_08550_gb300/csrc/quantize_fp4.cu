// Rows in 4 bits: codes with a scale for each block, and back.
//
//   MX: e = floor(log2 |block|) - 2, c = e2m1(x 2^-e)
//   NV: t = |row| / 2688, b = e4m3(|block| / (6 t)), c = e2m1(x / (b t))
//
// A thread takes 16 neighbouring values: a block of NV, half of one of MX, whose halves meet in a shuffle; the four scales of
// a tile's row are written by one of its threads.
// Bound by memory: values in, codes and scales out (or the other way round).  8192 x 4096 bf16: NV 13.4 us (6.4 TB/s), MX 11.9
// (values in L2), back 12.4; with eight values a thread, whose blocks' divisions and exchanges every other thread repeats, 20.6,
// 27.4 and 24.7.
#include <type_traits>

#include "common.cuh"
#include "fp4.cuh"
#include "internal.h"
#include "rows.cuh"

namespace oscars {

namespace {

constexpr int kThreads = 256, kUnit = 16;

// n / d for n < 2^31 by a multiplication (d of a launch is one number): T. Granlund, P. L. Montgomery, "Division by invariant
// integers using multiplication", 1994, their multiplier less 2^32, which n < 2^31
// lets be added without a carry
struct Divide {
  uint32_t d, m;
  int s;
};
Divide divide_by(uint32_t d) {
  int s = 0;
  while ((uint64_t(1) << s) < d) ++s;
  return {d, static_cast<uint32_t>(((uint64_t(1) << 32) * ((uint64_t(1) << s) - d)) / d + 1), s};
}
__device__ __forceinline__ uint32_t operator/(uint32_t n, const Divide& v) { return (__umulhi(n, v.m) + n) >> v.s; }

// 16 values of a row as they were read (n of them are inside it).  wide: 32 for 32-byte accesses, 16 for 16-byte ones, 0 for a
// matrix from `begin` to `end` whose rows start anywhere: the 16 bytes that hold the values are read and shifted.
template <typename T>
struct Held {
  static constexpr int kWords = kUnit * sizeof(T) / 4;
  uint32_t w[kWords];

  __device__ __forceinline__ void load(const T* p, int n, int wide, const void* begin, const void* end) {
    const int front = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15);
    const uint8_t* from = reinterpret_cast<const uint8_t*>(p) - front;
    if (n >= kUnit && wide == 32) {
#pragma unroll
      for (int i = 0; i < kWords; i += 8)
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]), "=r"(w[i + 4]), "=r"(w[i + 5]), "=r"(w[i + 6]), "=r"(w[i + 7])
                     : "l"(reinterpret_cast<const uint32_t*>(p) + i)
                     : "memory");
    } else if (n >= kUnit && wide == 16) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const uint4 a = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint32_t*>(p) + i);
        w[i] = a.x, w[i + 1] = a.y, w[i + 2] = a.z, w[i + 3] = a.w;
      }
    } else if (wide == 0 && n >= kUnit && from >= static_cast<const uint8_t*>(begin) &&
               from + 4 * kWords + 16 <= static_cast<const uint8_t*>(end)) {
      uint32_t r[kWords + 4];
#pragma unroll
      for (int i = 0; i < kWords + 4; i += 4) {   // the last 16 bytes hold none of the values if the first hold all of theirs
        const uint4 a = i < kWords || front > 0 ? *reinterpret_cast<const uint4*>(from + 4 * i) : make_uint4(0u, 0u, 0u, 0u);
        r[i] = a.x, r[i + 1] = a.y, r[i + 2] = a.z, r[i + 3] = a.w;
      }
      const bool two = front & 8, one = front & 4;
#pragma unroll
      for (int i = 0; i < kWords + 2; ++i) r[i] = two ? r[i + 2] : r[i];
#pragma unroll
      for (int i = 0; i < kWords + 1; ++i) r[i] = one ? r[i + 1] : r[i];
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = sizeof(T) == 4 ? r[i] : __funnelshift_r(r[i], r[i + 1], (front & 2) * 8);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = i < n ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
    } else {
      const unsigned short* u = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
      for (int i = 0; i < kWords; ++i)
        w[i] = (2 * i < n ? u[2 * i] : 0u) | (2 * i + 1 < n ? static_cast<uint32_t>(u[2 * i + 1]) << 16 : 0u);
    }
  }
  // the largest magnitude, as fp32's bits: in order, infinity above every number and NaN above it
  __device__ __forceinline__ uint32_t magnitude() const {
    uint32_t m = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
      return m;
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
      return max(m << 16, m & 0xFFFF0000u);
    }
  }
  // the codes of the values times `by`
  __device__ __forceinline__ uint2 codes(float by) const {
    uint32_t out[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float2 f;
        if constexpr (sizeof(T) == 4) f = make_float2(__uint_as_float(w[8 * h + 2 * i]), __uint_as_float(w[8 * h + 2 * i + 1]));
        else f = make_float2(__uint_as_float(w[4 * h + i] << 16), __uint_as_float(w[4 * h + i] & 0xFFFF0000u));
        f = __fmul2_rn(f, make_float2(by, by));
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
      }
      out[h] = eight_codes(v);
    }
    return make_uint2(out[0], out[1]);
  }
};

// Rows that are not 16-byte aligned: the G lanes of a group, whose units lie one behind the other from `base` on (n values up to
// the row's end), exchange them through the warp's own part of shared memory and write neighbouring ones.
constexpr int kPitch = kUnit + 1, kExchange = 32 * kPitch;

template <int G, typename T>
__device__ __forceinline__ void store_apart(const float (&f)[kUnit], T* base, int n, float* room) {
  const int lane = threadIdx.x & 31, l = lane % G;
  room += lane / G * G * kPitch;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kUnit; ++i) room[l * kPitch + i] = f[i];
  __syncwarp();
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
      const int e = j * G + l;
      if (e < n) base[e] = room[e + e / kUnit];
    }
  } else {   // in words of two; the first and the last may be half the neighbours'
    const int odd = static_cast<int>(reinterpret_cast<uintptr_t>(base) >> 1 & 1), most = n < G * kUnit ? n : G * kUnit;
#pragma unroll
    for (int j = 0; j <= kUnit / 2; ++j) {
      const int e = (j * G + l) * 2 - odd, f = e + 1;
      const float a = e >= 0 && e < most ? room[e + e / kUnit] : 0.f, b = f < most ? room[f + f / kUnit] : 0.f;
      if (e >= 0 && f < most) *reinterpret_cast<uint32_t*>(base + e) = pack_bf16x2(a, b);
      else if (e >= 0 && e < most) base[e] = static_cast<T>(a);
      else if (f >= 0 && f < most) base[f] = static_cast<T>(b);
    }
  }
}

struct QuantArgs {
  const void *x, *end;   // end: behind the last value
  uint8_t *q, *scales;
  float* row_scale;
  int64_t ldx, ldq;
  uint32_t units;       // OSCARS_MXFP4: threads, eight for each tile of a row, of rows from `first` on
  Divide per;           // of a row
  int64_t first;
  int rows, cols, tiles, wide;
};

// ------------------------------------------------------------------ OSCARS_MXFP4
// Blocks are on their own: a thread takes kN units, whose loads are in flight together.
template <typename T, int kN>
__global__ void __launch_bounds__(kThreads) quantize_mx_kernel(const __grid_constant__ QuantArgs a) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const uint32_t u0 = blockIdx.x * (kThreads * kN) + threadIdx.x;
  Held<T> held[kN];
  uint32_t row[kN];
  int at[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const uint32_t u = u0 + i * kThreads;
    row[i] = u < a.units ? u / a.per : 0;
    at[i] = u < a.units ? static_cast<int>(u - row[i] * a.per.d) * kUnit : -1;
    held[i].load(static_cast<const T*>(a.x) + row[i] * a.ldx + (at[i] < a.cols ? at[i] : 0), at[i] < 0 ? 0 : a.cols - at[i], a.wide, a.x, a.end);
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    uint32_t m = held[i].magnitude();
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    const uint32_t exp = m >> 23;
    const bool number = exp < 255;
    const uint32_t byte = number ? (exp > 2 ? exp - 2 : 0) : 255;
    uint32_t word = byte << (8 * ((lane >> 1) & 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 2);
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    if (at[i] < 0) continue;
    uint2 c = held[i].codes(__uint_as_float((254 - byte) << 23));   // 2^-e: from 2^127 (byte 0) to 2^-125
    if (!number) c = make_uint2(0u, 0u);
    if (at[i] / 32 * 32 < a.cols) *reinterpret_cast<uint2*>(a.q + row[i] * a.ldq + at[i] / 2) = c;
    if (lane % 8 == 0) *reinterpret_cast<uint32_t*>(a.scales + fp4_scale_at(a.first + row[i], at[i] / 128, a.tiles)) = word;
  }
}

// ------------------------------------------------------------------ OSCARS_NVFP4
// A row on TPR threads; up to kKeep turns stay in registers between the row's maximum and the codes.
constexpr int kKeep = 2;

template <typename T, int TPR>
__global__ void __launch_bounds__(kThreads / TPR * TPR) quantize_nv_kernel(const __grid_constant__ QuantArgs a) {
  constexpr int kRows = kThreads / TPR;
  __shared__ uint32_t part[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / TPR;
  const int t = threadIdx.x % TPR, turns = (a.cols + TPR * kUnit - 1) / (TPR * kUnit);
  if (TPR == 32 && row >= a.rows) return;
  const bool live = row < a.rows;
  const T* x = static_cast<const T*>(a.x) + (live ? row : 0) * a.ldx;
  auto load = [&](Held<T>& h, int i) {
    const int at = (i * TPR + t) * kUnit;
    h.load(x + (at < a.cols ? at : 0), a.cols - at, a.wide, a.x, a.end);
  };
  Held<T> held[kKeep];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kKeep; ++i) load(held[i], i);
#pragma unroll
  for (int i = 0; i < kKeep; ++i) m = max(m, held[i].magnitude());
  for (int i = kKeep; i < turns; ++i) {
    Held<T> h;
    load(h, i);
    m = max(m, h.magnitude());
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
  auto write = [&](int at, const Held<T>& h) {   // all lanes of the warp
    uint32_t byte = 0;
    if (number) {
      uint16_t b;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(0.f), "f"(fminf(__uint_as_float(h.magnitude()) * g, 448.f)));
      byte = b & 0xFFu;
    }
    uint2 c = h.codes(byte != 0 ? 1.f / (e4m3_value(byte) * scale) : 0.f);
    if (byte == 0) c = make_uint2(0u, 0u);
    uint32_t word = byte << (8 * (t & 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 1);
    word |= __shfl_xor_sync(0xffffffffu, word, 2);
    if (at / 32 * 32 < a.cols) *reinterpret_cast<uint2*>(q + at / 2) = c;
    if (t % 4 == 0 && at < a.cols) *reinterpret_cast<uint32_t*>(a.scales + fp4_scale_at(row, at / 64, a.tiles)) = word;
  };
#pragma unroll
  for (int i = 0; i < kKeep; ++i)
    if ((i * TPR + t / 32 * 32) * kUnit < a.cols) write((i * TPR + t) * kUnit, held[i]);
  for (int i = kKeep; i < turns; ++i) {
    if ((i * TPR + t / 32 * 32) * kUnit >= a.cols) break;
    Held<T> h;
    load(h, i);
    write((i * TPR + t) * kUnit, h);
  }
}

// ------------------------------------------------------------------ back
struct DequantArgs {
  const uint8_t *q, *scales;
  const float* row_scale;
  void* x;
  int64_t ldq, ldx;
  uint32_t units;       // of 16 columns, of rows from `first` on
  Divide per;           // of a row
  int64_t first;
  int rows, cols, tiles, wide, mx;
};

template <typename T, int kN>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const __grid_constant__ DequantArgs a) {
  __shared__ float room[kThreads / 32][kExchange];
  pdl_wait();
  pdl_trigger();
  const uint32_t u0 = blockIdx.x * (kThreads * kN) + threadIdx.x;
  uint2 w[kN];
  uint32_t byte[kN], row[kN];
  float t[kN];
  int at[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const uint32_t u = u0 + i * kThreads;
    row[i] = u < a.units ? u / a.per : 0;
    at[i] = u < a.units ? static_cast<int>(u - row[i] * a.per.d) * kUnit : a.cols;
    const int from = at[i] < a.cols ? at[i] : 0;
    w[i] = *reinterpret_cast<const uint2*>(a.q + row[i] * a.ldq + from / 2);
    const int block = from / (a.mx ? 32 : 16);
    byte[i] = a.scales[fp4_scale_at(a.first + row[i], block / 4, a.tiles) + block % 4];
    t[i] = a.row_scale ? a.row_scale[row[i]] : 1.f;
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const float s = a.mx ? e8m0_value(byte[i]) : e4m3_value(byte[i]);
    float f[kUnit];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t p[4];
      eight_values(h == 0 ? w[i].x : w[i].y, p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 v = __fmul2_rn(__fmul2_rn(__half22float2(*reinterpret_cast<const __half2*>(&p[e])), make_float2(s, s)), make_float2(t[i], t[i]));
        f[8 * h + 2 * e] = v.x, f[8 * h + 2 * e + 1] = v.y;
      }
    }
    T* row_at = static_cast<T*>(a.x) + row[i] * a.ldx;
    if (!a.wide) {
      const int tile = at[i] < a.cols ? at[i] / 128 * 128 : a.cols / 128 * 128;
      // a group of eight lanes has one tile, and none of them has one past the last unit
      store_apart<8>(f, row_at + tile, u0 + i * kThreads < a.units ? a.cols - tile : 0, room[threadIdx.x >> 5]);
      continue;
    }
    if (at[i] >= a.cols) continue;
    T* to = row_at + at[i];
    const int left = a.cols - at[i];
    if (a.wide == 32 && left >= kUnit) {
      uint32_t o[8];
#pragma unroll
      for (int h = 0; h < static_cast<int>(sizeof(T)) / 2; ++h) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = sizeof(T) == 4 ? __float_as_uint(f[8 * h + e]) : pack_bf16x2(f[2 * e], f[2 * e + 1]);
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + 8 * h), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]),
                     "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7])
                     : "memory");
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float g[8] = {f[8 * h], f[8 * h + 1], f[8 * h + 2], f[8 * h + 3], f[8 * h + 4], f[8 * h + 5], f[8 * h + 6], f[8 * h + 7]};
        store8(to + 8 * h, left - 8 * h, true, g);
      }
    }
  }
}

bool at_bytes(const void* p, int n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool format_ok(int f) { return f == OSCARS_MXFP4 || f == OSCARS_NVFP4; }
bool sizes_ok(int rows, int cols, int format) {
  return rows >= 0 && rows <= kFp4MaxSide && cols >= 1 && cols <= kFp4MaxSide && format_ok(format);
}
int wide_rows(const void* p, int64_t ld, int size) {
  return at_bytes(p, 32) && ld * size % 32 == 0 ? 32 : at_bytes(p, 16) && ld * size % 16 == 0 ? 16 : 0;
}
// f(first row, rows) over pieces of a matrix that have up to 2^30 units (a row has up to 2^26)
template <typename F>
cudaError_t by_rows(int rows, int per, F&& f) {
  const int64_t most = (int64_t(1) << 30) / per;
  for (int64_t r = 0; r < rows; r += most) {
    const cudaError_t e = f(r, static_cast<int>(rows - r < most ? rows - r : most));
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

// Units of a thread: several where there are enough of them for every SM all the same (1000 x 1000 bf16: one 2.1 us, four 3.2;
// 8192 x 4096: one 18.9, four 12.3)
template <typename T, typename F>
cudaError_t by_units(uint32_t units, F&& f) {
  constexpr int kMany = sizeof(T) == 4 ? 2 : 4;
  if (units >= 152u * 8 * kThreads * kMany) return f(std::integral_constant<int, kMany>());
  return f(std::integral_constant<int, 1>());
}

template <typename T>
cudaError_t quantize(const QuantArgs& a, int format, cudaStream_t s) {
  if (format == OSCARS_MXFP4) {
    const int per = a.tiles * 8;
    return by_rows(a.rows, per, [&](int64_t r, int rows) {
      QuantArgs p = a;
      p.x = static_cast<const T*>(a.x) + r * a.ldx;
      p.q += r * a.ldq;
      p.first = r;
      p.rows = rows;
      p.units = static_cast<uint32_t>(rows) * per;
      p.per = divide_by(per);
      return by_units<T>(p.units, [&](auto n) {
        return launch_dependent(quantize_mx_kernel<T, n()>, dim3((p.units + kThreads * n() - 1) / (kThreads * n())), kThreads, 0, s, p);
      });
    });
  }
  auto rows = [&](auto tpr) {
    constexpr int kRows = kThreads / tpr();
    return launch_dependent(quantize_nv_kernel<T, tpr()>, dim3((a.rows + kRows - 1) / kRows), kRows * tpr(), 0, s, a);
  };
  // the least whole warps that keep a row in registers
  const int warps = (a.cols + 32 * kUnit * kKeep - 1) / (32 * kUnit * kKeep);
  if (warps <= 1) return rows(std::integral_constant<int, 32>());
  if (warps <= 2) return rows(std::integral_constant<int, 64>());
  if (warps <= 4) return rows(std::integral_constant<int, 128>());
  if (warps <= 6) return rows(std::integral_constant<int, 192>());
  return rows(std::integral_constant<int, 256>());
}

template <typename T>
cudaError_t dequantize(const DequantArgs& a, cudaStream_t s) {
  const int per = a.wide ? (a.cols + kUnit - 1) / kUnit : (a.cols + 127) / 128 * 8;   // whole tiles where lanes exchange values
  return by_rows(a.rows, per, [&](int64_t r, int rows) {
    DequantArgs p = a;
    p.x = static_cast<T*>(a.x) + r * a.ldx;
    p.q += r * a.ldq;
    p.first = r;
    if (a.row_scale) p.row_scale += r;
    p.rows = rows;
    p.units = static_cast<uint32_t>(rows) * per;
    p.per = divide_by(per);
    return by_units<T>(p.units, [&](auto n) {
      return launch_dependent(dequantize_kernel<T, n()>, dim3((p.units + kThreads * n() - 1) / (kThreads * n())), kThreads, 0, s, p);
    });
  });
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
  const uint8_t* end = static_cast<const uint8_t*>(x) + ((rows - 1) * ldx + cols) * size;
  QuantArgs a{x, end, q, scales, row_scale, ldx, ldq, 0, {}, 0, rows, cols, fp4_tiles(cols, format), wide_rows(x, ldx, size)};
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
  DequantArgs a{q, scales, row_scale, x, ldq, ldx, 0, {}, 0, rows, cols, fp4_tiles(cols, format), wide_rows(x, ldx, size), format == OSCARS_MXFP4};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == OSCARS_F32 ? dequantize<float>(a, s) : dequantize<__nv_bfloat16>(a, s);
  return e == cudaSuccess ? OSCARS_OK : OSCARS_ECUDA;
}

}  // extern "C"
