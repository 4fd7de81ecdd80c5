// Rows of fp32 or bf16 read eight elements a thread, and launches that depend on
// the previous kernel of their stream.
#pragma once

#include "common.cuh"

namespace oscars {

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// 8 elements of a row; `vec`: 16-byte loads, all 8 inside
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, bool vec, float (&v)[8]) {
  if (vec && n >= 8) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(p);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}

// Eight elements of a row held as they were read (bf16 in half the registers).
template <typename T>
struct Held8 {
  float v[8];
  __device__ __forceinline__ void load(const T* p, int n, bool vec) { load8(p, n, vec, v); }
  __device__ __forceinline__ void get(float (&to)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i] = v[i];
  }
};
template <>
struct Held8<__nv_bfloat16> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int n, bool vec) {
    if (vec && n >= 8) {
      const uint4 a = *reinterpret_cast<const uint4*>(p);
      w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    } else {
      const unsigned short* u = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (2 * i < n ? u[2 * i] : 0u) | (2 * i + 1 < n ? static_cast<uint32_t>(u[2 * i + 1]) << 16 : 0u);
    }
  }
  __device__ __forceinline__ void get(float (&to)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      to[2 * i] = __uint_as_float(w[i] << 16);
      to[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};

// 8 values of a row; `vec`: 16-byte stores
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, bool vec, const float (&v)[8]) {
  if (vec && n >= 8) {
    if constexpr (sizeof(T) == 4) {
      reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = static_cast<T>(v[i]);
  }
}

// Sums of squares over the whole range of fp32, in fp32 (the card's fp64 rate is 1/64 of it): of values whose squares
// neither overflow nor underflow, of larger ones times 2^-80 and of smaller ones times 2^80.
struct Squares {
  float mid = 0.f, big = 0.f, small = 0.f;

  template <int N>
  __device__ __forceinline__ void add(const float (&v)[N]) {
    float s = 0.f, m = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s = fmaf(v[i], v[i], s);
      m = fmaxf(m, fabsf(v[i]));
    }
    if ((s > 1e-20f && s < 1e25f) || m == 0.f) {   // m is 0 for zeros, and for NaN alone, which s carries on
      mid += s;
    } else {
      const float by = m > 1.f ? 0x1p-80f : 0x1p80f;
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) t = fmaf(v[i] * by, v[i] * by, t);
      (m > 1.f ? big : small) += t;
    }
  }
  __device__ __forceinline__ void add(const Squares& o) { mid += o.mid, big += o.big, small += o.small; }
  __device__ __forceinline__ void warp_sum() {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      mid += __shfl_xor_sync(0xffffffffu, mid, o);
      big += __shfl_xor_sync(0xffffffffu, big, o);
      small += __shfl_xor_sync(0xffffffffu, small, o);
    }
  }
  // sum over the block in a fixed order, in thread 0 (`part`: one entry a warp)
  __device__ __forceinline__ void block_sum(Squares* part) {
    warp_sum();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = *this;
    __syncthreads();
    if (threadIdx.x == 0)
      for (int i = 1; i < static_cast<int>(blockDim.x) / 32; ++i) add(part[i]);
  }
  __device__ __forceinline__ double total() const {
    return static_cast<double>(mid) + static_cast<double>(big) * 0x1p160 + static_cast<double>(small) * 0x1p-160;
  }
};

// 1 / (norm + eps) = power x factor of a sum of squares, each a normal fp32 number: norm + eps lies between 2^-149 and 2^145,
// further from 1 than the reciprocal of a power of two can follow it, so `power` stops at 2^125 and 2^-126 and `factor` has the
// rest.  (With all of it in `power`, zeros under an eps of 2^-129 came out as 0 x infinity.)
__device__ __forceinline__ void inverse_norm(double squares, float eps, float& power, float& factor) {
  int e;
  const double m = frexp(sqrt(squares) + static_cast<double>(eps), &e);
  const int in_power = min(max(e, -125), 126);
  factor = static_cast<float>(ldexp(1.0 / m, in_power - e));
  power = isinf(squares) ? 0.f : ldexpf(1.f, -in_power);
}

// A launch whose set-up may run while the previous kernel on the stream ends: the
// kernel calls pdl_wait() before it touches global memory.
template <typename... P, typename... A>
cudaError_t launch_dependent(void (*kernel)(P...), dim3 grid, int block, size_t smem, cudaStream_t s, A... args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace oscars
