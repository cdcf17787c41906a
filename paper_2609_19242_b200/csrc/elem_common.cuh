// Vectors of elements in memory as fp32 in registers, for the bandwidth-bound kernels that take several element types.
#pragma once
#include <cuda_fp16.h>

#include <type_traits>

#include "../../include/bdlm_dtypes.h"
#include "bdlm_common.cuh"

namespace bdlm {

using bf16_t = __nv_bfloat16;

// V elements of type T as they lie in memory: 16-byte vectors, one of 8 bytes, or one element.
template <class T, int V>
struct Raw {
  static constexpr int WORDS = V * (int)sizeof(T) / 4;
  static_assert(WORDS % 4 == 0 || WORDS == 2, "16- or 8-byte vectors");
  using Vec = typename std::conditional<WORDS == 2, uint2, uint4>::type;
  static constexpr int N = WORDS * 4 / (int)sizeof(Vec);
  Vec q[N];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = reinterpret_cast<const Vec*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < N; ++i) reinterpret_cast<Vec*>(p)[i] = q[i];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = Vec{};
  }
  __device__ __forceinline__ void get(float (&f)[V]) const {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(q);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        if constexpr (std::is_same<T, bf16_t>::value) {
          f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
          const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
          f[2 * i] = v.x; f[2 * i + 1] = v.y;
        }
      }
    }
  }
  __device__ __forceinline__ void put(const float (&f)[V]) {
    uint32_t* w = reinterpret_cast<uint32_t*>(q);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        if constexpr (std::is_same<T, bf16_t>::value) {
          w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
        } else {
          const __half2 v = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t*>(&v);
        }
      }
    }
  }
};
template <class T>
struct Raw<T, 1> {
  T e;
  __device__ __forceinline__ void load(const T* p) { e = *p; }
  __device__ __forceinline__ void store(T* p) const { *p = e; }
  __device__ __forceinline__ void clear() { e = T(0.f); }
  __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = (float)e; }
  __device__ __forceinline__ void put(const float (&f)[1]) { e = T(f[0]); }
};

}  // namespace bdlm
