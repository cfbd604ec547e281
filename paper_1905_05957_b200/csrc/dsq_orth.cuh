// Shared pieces of the orthogonalised update: its numbers' scale, the momentum, and the form for small matrices.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dsq_internal.h"

namespace dsq {

constexpr float kUp = 1024.f, kDown = 1.f / 1024.f;   // the fixed scale of the 16-bit matrices

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

__device__ __forceinline__ void load4(float (&o)[4], const float* p) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  o[0] = v.x, o[1] = v.y, o[2] = v.z, o[3] = v.w;
}
template <class T16>
__device__ __forceinline__ void load4(float (&o)[4], const T16* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  const T16* e = reinterpret_cast<const T16*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = to_f32(e[i]);
}

// X kUp = (u first) then.  The sum of squares is in 64 bits; where the norm or kUp / norm would leave 32 bits, u is brought into
// range by a power of two.  (A norm of 0 without eps, or one that is not a number, makes X NaN.)
struct NormFactor {
  float first, then;
  __device__ __forceinline__ NormFactor(double sum, float eps) : then(1.f) {
    const double root = sqrt(sum);
    const float norm = (float)root + eps;
    first = kUp / norm;
    if (!(norm > 1e-30f && norm < 1e30f)) {
      const double wide = root + (double)eps;
      if (wide > 0 && wide < 1e60) {
        first = wide < 1 ? 0x1p100f : 0x1p-100f;
        then = (float)((double)kUp / (wide * (double)first));
      }
    }
  }
  __device__ __forceinline__ float operator()(float u) const { return __fmul_rn(__fmul_rn(u, first), then); }
};

struct Momentum {
  const void* g;
  float* buf;        // NULL: u = g
  uint64_t stride;   // elements between matrices of g and buf
  float mu;
  int nesterov;
  __device__ __forceinline__ float update(float g, float b) const {   // the new buf
    return __fadd_rn(__fmul_rn(mu, b), g);
  }
  __device__ __forceinline__ float direction(float g, float b) const {   // u from the new buf
    return nesterov ? __fadd_rn(g, __fmul_rn(mu, b)) : b;
  }
};

// Where a finished update goes.
struct OrthOut {
  void* out;          // NULL or contiguous [batch, rows, cols]
  int dtype;          // DS_F32 or DS_BF16
  float* x;           // NULL or the model: x = keep x - rate X
  uint64_t x_stride;
  float keep, rate;
};

// Matrices whose shorter side is at most 64 and whose longer side is not too long: one cluster of CTAs a matrix, everything in one launch
// (dsq_orth_small.cu).  Returns the CTAs a matrix takes, 0 where the general form is taken.
uint32_t orth_small_ctas(uint32_t m, uint32_t n, uint32_t batch);
cudaError_t launch_orth_small(const ds_orth_config& c, uint32_t ctas, const Momentum& mo, int g_dtype, const OrthOut& o, cudaStream_t st);

}  // namespace dsq
