// Activations of 16 bytes as fp32 values and back.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "common.cuh"

namespace flare {

template <typename T>
struct Piece;  // 16 bytes of elements as floats
template <>
struct Piece<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void load(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 store(const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void load(const uint4& u, float* x) {
    x[0] = __uint_as_float(u.x);
    x[1] = __uint_as_float(u.y);
    x[2] = __uint_as_float(u.z);
    x[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 store(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                      __float_as_uint(x[3]));
  }
};

// Eight elements as four packed pairs (f2 of common.cuh) and back.
template <typename T>
__device__ __forceinline__ void load_pairs(const uint4* u, uint64_t (&x)[4]);
template <>
__device__ __forceinline__ void load_pairs<__nv_bfloat16>(const uint4* u, uint64_t (&x)[4]) {
  const uint32_t w[4] = {u->x, u->y, u->z, u->w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
template <>
__device__ __forceinline__ void load_pairs<float>(const uint4* u, uint64_t (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[2 * i] = f2(__uint_as_float(u[i].x), __uint_as_float(u[i].y));
    x[2 * i + 1] = f2(__uint_as_float(u[i].z), __uint_as_float(u[i].w));
  }
}

template <typename T>
__device__ __forceinline__ void store_pairs(T* p, const uint64_t (&x)[4]) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) f2_split(x[i], f[2 * i], f[2 * i + 1]);
#pragma unroll
  for (int i = 0; i < 8 / Piece<T>::N; ++i)
    reinterpret_cast<uint4*>(p)[i] = Piece<T>::store(f + i * Piece<T>::N);
}

}  // namespace flare
