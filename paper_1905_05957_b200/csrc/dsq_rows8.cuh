// Eight neighbouring entries of a row, as floats.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "dsq_internal.h"

namespace dsq {

template <class T>
__device__ __forceinline__ float to_float(T v) {
  if constexpr (std::is_same<T, float>::value) return v;
  else if constexpr (std::is_same<T, __half>::value) return __half2float(v);
  else return __bfloat162float(v);
}
template <class T>
__device__ __forceinline__ T from_float(float v) {
  if constexpr (std::is_same<T, float>::value) return v;
  else if constexpr (std::is_same<T, __half>::value) return __float2half_rn(v);
  else return __float2bfloat16_rn(v);
}
template <class T>
__device__ __forceinline__ void unpack8(const uint4 (&q)[sizeof(T) / 2], float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    v[0] = __uint_as_float(q[0].x), v[1] = __uint_as_float(q[0].y), v[2] = __uint_as_float(q[0].z), v[3] = __uint_as_float(q[0].w);
    v[4] = __uint_as_float(q[1].x), v[5] = __uint_as_float(q[1].y), v[6] = __uint_as_float(q[1].z), v[7] = __uint_as_float(q[1].w);
  } else {
    const uint32_t w[4] = {q[0].x, q[0].y, q[0].z, q[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
      }
    }
  }
}
// Entries behind the row's end are 0.
template <class T>
__device__ __forceinline__ void load8(const void* base, uint64_t at, uint32_t c, uint32_t cols, bool vec, float (&v)[8]) {
  const T* p = static_cast<const T*>(base) + at + c;
  if (vec && c + 8 <= cols) {
    uint4 q[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = ld_plain(reinterpret_cast<const uint4*>(p) + i);
    unpack8<T>(q, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? to_float(ld_plain(p + j)) : 0.f;
  }
}
template <class T>
__device__ __forceinline__ void store8(void* base, uint64_t at, uint32_t c, uint32_t cols, bool vec, const float (&v)[8]) {
  T* p = static_cast<T*>(base) + at + c;
  if (vec && c + 8 <= cols) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      T t[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) t[j] = from_float<T>(v[j]);
      *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(t);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < cols) p[j] = from_float<T>(v[j]);
  }
}

}  // namespace dsq
