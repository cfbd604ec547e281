// Products of 16-bit matrices with bias, activation and residual in their epilogue:
//
//   z_mn = sum_k a_mk b_nk + bias_n,   out_mn = act(z_mn) + residual_mn        (sums and epilogue in 32 bits, rounded once)
//
// A layer's forward product takes x and W as they lie; the gradient of its inputs dz and W across K; that of its weights dz
// and x, both across K.  dsq_product16*.cu hold the forms, one file each so that they compile side by side.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dsq_mma.cuh"

namespace dsq {

// ---- numbers --------------------------------------------------------------------------------------------

__device__ __forceinline__ float half_at(uint32_t w, int hi, bool bf16) {      // the low or the high half of a word
  if (bf16) return __uint_as_float(hi ? w & 0xFFFF0000u : w << 16);
  const __half2 h = *reinterpret_cast<const __half2*>(&w);
  return hi ? __high2float(h) : __low2float(h);
}
__device__ __forceinline__ uint32_t halves_of(float a, float b, bool bf16) {
  if (bf16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint16_t half_of(float a, bool bf16) {
  if (bf16) return __bfloat16_as_ushort(__float2bfloat16_rn(a));
  return __half_as_ushort(__float2half_rn(a));
}
__device__ __forceinline__ float from_half(uint16_t w, bool bf16) {
  return bf16 ? __uint_as_float((uint32_t)w << 16) : __half2float(__ushort_as_half(w));
}

// Powers of two and reciprocals by the special function unit, good to a few units of 2^-23; numbers below 2^-126 count as 0.
__device__ __forceinline__ float exp2_of(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float reciprocal(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
constexpr float kLog2E = 1.44269504f, kSqrtHalf = 0.70710678f, kSqrt2OverPi = 0.79788456f, kGeluCubic = 0.044715f, kInvSqrt2Pi = 0.39894228f;
// 1 / (1 + exp(-v)) of v = scaled / log2(e)
__device__ __forceinline__ float sigmoid2(float scaled) { return reciprocal(1.f + exp2_of(-scaled)); }
// The normal distribution's Phi(z), and exp(-z^2 / 2): Phi(-|z|) = exp(-z^2 / 2) t P(t) with t = 1 / (1 + 0.3 |z|) and a P of eight terms, fitted for this so that the largest
// relative error over 0 <= |z| <= 13.3 (where the power of two ends) is least: 1.3e-7.  Evaluated as below it is 2^-20 for |z| up to 4 and grows with the rounding of
// z^2, to 2^-17 at 13: no cancellation for negative z.  (Five terms of a polynomial with a bounded absolute error were off by 0.16 % of Phi at -5 and 1 % at -8.)  An
// unrolled run of 32 values is what an epilogue fetches once a block, so that erff's length costs more than its work (4096^3 in training, forward: 107 us by erff, 98 by
// five terms, 101 by these).
__device__ __forceinline__ float phi_of(float z, float& e) {
  const float t = reciprocal(__fmaf_rn(0.3f, fabsf(z), 1.f));
  e = exp2_of(z * z * (-0.5f * kLog2E));
  float q = __fmaf_rn(t, 0.0360361804f, -0.158713128f);
  q = __fmaf_rn(t, q, 0.208963799f);
  q = __fmaf_rn(t, q, -0.056095186f);
  q = __fmaf_rn(t, q, 0.129843065f);
  q = __fmaf_rn(t, q, 0.099523166f);
  q = __fmaf_rn(t, q, 0.120816876f);
  q = __fmaf_rn(t, q, 0.119625167f) * t * e;
  return z < 0.f ? q : 1.f - q;
}

template <int ACT>
__device__ __forceinline__ float act_of(float z) {
  if constexpr (ACT == DS_ACT_RELU) return z < 0.f ? 0.f : z;
  if constexpr (ACT == DS_ACT_GELU) {
    float e;
    return z * phi_of(z, e);
  }
  if constexpr (ACT == DS_ACT_GELU_TANH) return z * sigmoid2(2.f * kSqrt2OverPi * kLog2E * __fmaf_rn(kGeluCubic * z * z, z, z));   // (1 + tanh u) / 2 = sigmoid(2 u)
  if constexpr (ACT == DS_ACT_SILU) return z * sigmoid2(kLog2E * z);
  return z;
}
// act'(z).  Beyond |z| = 100 the slopes are 0 and 1 in 32 bits; kept there so that no inf meets a zero.
template <int ACT>
__device__ __forceinline__ float slope_of(float z) {
  if constexpr (ACT == DS_ACT_RELU) return z > 0.f ? 1.f : z == z ? 0.f : z;
  const float c = fabsf(z) > 100.f ? copysignf(100.f, z) : z;
  if constexpr (ACT == DS_ACT_GELU) {
    float e;
    const float p = phi_of(c, e);
    return __fmaf_rn(c * kInvSqrt2Pi, e, p);
  }
  if constexpr (ACT == DS_ACT_GELU_TANH) {
    const float s = sigmoid2(2.f * kSqrt2OverPi * kLog2E * __fmaf_rn(kGeluCubic * c * c, c, c));
    return __fmaf_rn(c * s * (1.f - s), 2.f * kSqrt2OverPi * __fmaf_rn(3.f * kGeluCubic * c, c, 1.f), s);
  }
  if constexpr (ACT == DS_ACT_SILU) {
    const float s = sigmoid2(kLog2E * c);
    return s * __fmaf_rn(c, 1.f - s, 1.f);
  }
  return 1.f;
}
// One branch for a run of values, not one a value.
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  switch (act) {
    case DS_ACT_RELU: f(std::integral_constant<int, DS_ACT_RELU>()); break;
    case DS_ACT_GELU: f(std::integral_constant<int, DS_ACT_GELU>()); break;
    case DS_ACT_GELU_TANH: f(std::integral_constant<int, DS_ACT_GELU_TANH>()); break;
    case DS_ACT_SILU: f(std::integral_constant<int, DS_ACT_SILU>()); break;
    default: break;
  }
}

// What every form of the epilogue works on.
struct Out16 {
  const float* bias;           // or NULL
  const uint16_t* residual;    // or NULL
  uint16_t* z;                 // or NULL
  void* out;
  uint64_t ldr, ldz, ldo;
  uint32_t m, n;
  int act;
  int bf16;                    // type of residual, z and a 16-bit out
  int f32;                     // out holds floats
};

// ---- epilogues ------------------------------------------------------------------------------------------

// Rows of residual, z and out start and end on 16-byte boundaries and out has 16 bits: blocks of 32 x 32 pass through shared memory
// by TMA (whose stores leave out rows and columns outside the matrix, but columns 16 bytes at a time).  OUTS 2: z leaves, too.
template <int OUTS>
struct EpiBlocks {
  static constexpr int kIn = 1, kOut = OUTS;
  struct Pre {};
  CUtensorMap map_r, map_y, map_z;
  Out16 o;
  int bias_vec;                // bias starts on a 16-byte boundary
  __device__ __forceinline__ const CUtensorMap* in(int) const { return o.residual ? &map_r : nullptr; }
  __device__ __forceinline__ const CUtensorMap* out(int i) const { return i ? &map_z : &map_y; }
  __device__ __forceinline__ Pre load(uint32_t, uint32_t, uint32_t) const { return {}; }
  __device__ __forceinline__ void put(uint32_t block, int lane, const float (&v)[32]) const {
    uint32_t w[16];
    if (o.bf16) {
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = halves_of(v[2 * j], v[2 * j + 1], true);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = halves_of(v[2 * j], v[2 * j + 1], false);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row_chunk(block, lane, q)), "r"(w[4 * q]), "r"(w[4 * q + 1]), "r"(w[4 * q + 2]),
                   "r"(w[4 * q + 3])
                   : "memory");
  }
  __device__ __forceinline__ void apply(const Pre&, const uint32_t (&acc)[32], uint32_t, uint32_t col0, uint32_t, uint32_t block, int lane) const {
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(acc[j]);
    if (o.bias) {
      if (bias_vec && col0 + 32 <= o.n) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float4 c = ld_plain(reinterpret_cast<const float4*>(o.bias + col0) + q);
          v[4 * q] += c.x, v[4 * q + 1] += c.y, v[4 * q + 2] += c.z, v[4 * q + 3] += c.w;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (col0 + j < o.n) v[j] += ld_plain(o.bias + col0 + j);
      }
    }
    if constexpr (OUTS > 1) put(block + kBlockBytes, lane, v);
    with_act(o.act, [&](auto a) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = act_of<decltype(a)::value>(v[j]);
    });
    if (o.residual) {
      uint32_t w[16];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[4 * q]), "=r"(w[4 * q + 1]), "=r"(w[4 * q + 2]), "=r"(w[4 * q + 3])
                     : "r"(row_chunk(block, lane, q))
                     : "memory");
      if (o.bf16) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] += half_at(w[j / 2], j & 1, true);
      } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] += half_at(w[j / 2], j & 1, false);
      }
    }
    put(block, lane, v);
  }
};

// Floats on 32-byte rows and nothing but the product (gradients of weights, straight into a row of a step's gradients).
struct EpiFloats {
  static constexpr int kIn = 0, kOut = 0;
  struct Pre {};
  float* out;
  uint64_t ld;
  uint32_t m, n;
  __device__ __forceinline__ Pre load(uint32_t, uint32_t, uint32_t) const { return {}; }
  __device__ __forceinline__ void apply(const Pre&, const uint32_t (&acc)[32], uint32_t row, uint32_t col0, uint32_t) const {
    if (row >= m) return;
    float* o = out + row * ld + col0;
    if (col0 + 32 <= n) {
#pragma unroll
      for (int i = 0; i < 4; ++i) st_b32(o + 8 * i, acc + 8 * i);
    } else {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (col0 + j < n) o[j] = __uint_as_float(acc[j]);
    }
  }
};

// Everything else, with the operands' places exchanged: rows of the product are columns of out, so that lanes hold consecutive
// entries of it.  For outputs on no boundary, and for few rows of out, so that a tile fills with weights.  Its instructions are what such a product waits for where K is short:
// types and whole blocks are told apart once a block, two entries are rounded by one instruction (8095 x 1037 -> 3647 with z, fp16: 130 us with both a value).
struct EpiTurned {
  static constexpr int kIn = 0, kOut = 0;
  struct Pre {
    float c;
  };
  Out16 o;       // m, n: of out
  __device__ __forceinline__ Pre load(uint32_t row, uint32_t, uint32_t) const { return {o.bias && row < o.n ? ld_plain(o.bias + row) : 0.f}; }
  template <bool BF16>
  static __device__ __forceinline__ void put16(uint16_t* to, uint64_t ld, const float (&v)[32], uint32_t rows) {
    if (rows >= 32) {
#pragma unroll
      for (int j = 0; j < 32; j += 2) {
        const uint32_t w = halves_of(v[j], v[j + 1], BF16);
        to[0] = (uint16_t)w;
        to[ld] = (uint16_t)(w >> 16);
        to += 2 * ld;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (j < rows) to[j * ld] = half_of(v[j], BF16);
    }
  }
  static __device__ __forceinline__ void put(uint16_t* to, uint64_t ld, const float (&v)[32], uint32_t rows, bool bf16) {
    if (bf16)
      put16<true>(to, ld, v, rows);
    else
      put16<false>(to, ld, v, rows);
  }
  __device__ __forceinline__ void apply(const Pre& p, const uint32_t (&acc)[32], uint32_t col, uint32_t row0, uint32_t) const {
    if (col >= o.n) return;
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(acc[j]) + p.c;
    const uint32_t rows = o.m - row0;      // at least one
    if (o.z) put(o.z + row0 * o.ldz + col, o.ldz, v, rows, o.bf16);
    with_act(o.act, [&](auto a) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = act_of<decltype(a)::value>(v[j]);
    });
    if (o.residual) {
      const uint16_t* from = o.residual + row0 * o.ldr + col;
      uint16_t r[32];
      if (rows >= 32) {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          r[j] = ld_plain(from);
          from += o.ldr;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) r[j] = j < rows ? ld_plain(from + j * o.ldr) : (uint16_t)0;
      }
      if (o.bf16) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] += from_half(r[j], true);
      } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] += from_half(r[j], false);
      }
    }
    if (o.f32) {
      float* to = static_cast<float*>(o.out) + row0 * o.ldo + col;
      if (rows >= 32) {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          *to = v[j];
          to += o.ldo;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (j < rows) to[j * o.ldo] = v[j];
      }
    } else {
      put(static_cast<uint16_t*>(o.out) + row0 * o.ldo + col, o.ldo, v, rows, o.bf16);
    }
  }
};

// ---- host side ------------------------------------------------------------------------------------------

// An operand on 16-byte rows: [rows, k] along K, or [k, rows] across it.
struct Operand16 {
  const void* p;
  uint64_t ld;
  uint32_t rows;
  bool across;
};
inline cudaError_t operand_map(CUtensorMap* map, const Operand16& o, uint32_t k, uint32_t box_rows) {
  return o.across ? make_tensor_map(map, kMmaHalf, o.p, o.rows, k, 1, o.ld, o.ld * k, 64, 64)
                  : make_tensor_map(map, kMmaHalf, o.p, k, o.rows, 1, o.ld, o.ld * o.rows, 64, box_rows);
}

// C = A B^T by the form that `plan` names; A_MODE and B_MODE as the operands lie.
template <int A_MODE, int B_MODE, class Epi>
cudaError_t product16(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const Epi& epi, cudaStream_t st) {
  CUtensorMap ma, mb;
  cudaError_t e = operand_map(&ma, a, s.k, kMmaRows);
  if (e == cudaSuccess) e = operand_map(&mb, b, s.k, plan.box_rows());
  if (e != cudaSuccess) return e;
  return launch_mma<kMmaHalf, A_MODE, B_MODE>(plan, ma, mb, mb, s, epi, st);
}

// The forms, by how the operands lie.  forward: both along K; inputs: B across; weights: both across.
cudaError_t product16_forward(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const EpiBlocks<1>& epi, cudaStream_t st);
cudaError_t product16_forward_z(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const EpiBlocks<2>& epi, cudaStream_t st);
cudaError_t product16_gradient(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const EpiBlocks<1>& epi, cudaStream_t st);
cudaError_t product16_floats(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const EpiFloats& epi, cudaStream_t st);
cudaError_t product16_turned(const MmaPlan& plan, const Operand16& a, const Operand16& b, const MmaShape& s, const EpiTurned& epi, cudaStream_t st);

}  // namespace dsq
