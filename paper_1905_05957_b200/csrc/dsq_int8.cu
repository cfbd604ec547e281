// Layer products in 8-bit integers with one scale per row of either operand.
//
//   s_r = max_c |x_rc| / 127,  q_rc = round(x_rc / s_r)              (quantise: by rows, by columns, or both at once)
//   y_mn = (sum_k qa_mk qb_nk) sa_m sb_n + bias_n                      (product: the sum is exact in 32-bit integers)
//
// A linear layer's forward product takes the rows of x and of W; the gradient of its inputs the rows of dY and the columns of
// W; the gradient of its weights the columns of dY and of x.  Column codes are stored transposed, so that all three are
// the same product of two matrices laid out along K.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "dsq_mma.cuh"

using namespace dsq;

namespace {

constexpr float kInv127 = 1.f / 127.f;
constexpr uint32_t kInfBits = 0x7F800000u;

// Scale and its reciprocal from the bits of the largest magnitude (an inf or a NaN has larger bits than any number and wins
// the maximum: the line's scale is then NaN and its codes 0).  A line whose scale would be subnormal is a line of zeros.
__device__ __forceinline__ void scale_of(uint32_t amax_bits, float& s, float& inv) {
  s = __fmul_rn(__uint_as_float(amax_bits), kInv127);
  inv = 0.f;
  if (amax_bits >= kInfBits)
    s = __uint_as_float(0x7FC00000u);
  else if (s < 1.17549435e-38f)
    s = 0.f;
  else
    inv = __frcp_rn(s);
}
__device__ __forceinline__ int code_of(float v, float inv) { return __float2int_rn(__fmul_rn(v, inv)); }   // a NaN gives 0
__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

// 16 bytes of x as floats.
template <class T>
struct Vec {
  static constexpr int kN = 16 / sizeof(T);
  uint4 raw;
  __device__ __forceinline__ float at(int i) const { return to_f32(reinterpret_cast<const T*>(&raw)[i]); }
};

// ---- by rows: one CTA a row, one reading ----
// The row stays in registers between its maximum and its codes (up to kKeep vectors a thread; the rest of a longer row is read
// again, from cache).  Codes from `cols` up to the next multiple of 16 are written as 0.
constexpr int kKeep = 4;

template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_i8_rows(const T* x, uint64_t ld, uint32_t cols, int8_t* q, uint64_t ldq, float* scale) {
  pdl_prologue();
  constexpr int N = VEC ? Vec<T>::kN : 4;
  const T* row = x + (uint64_t)blockIdx.x * ld;
  int8_t* out = q + (uint64_t)blockIdx.x * ldq;
  const uint32_t nv = (cols + N - 1) / N, nv_out = (cols + 15) / 16 * 16 / N;
  auto fetch = [&](uint32_t v, float (&f)[N]) {
    if (VEC && (v + 1) * N <= cols) {
      Vec<T> r;
      r.raw = *reinterpret_cast<const uint4*>(row + (uint64_t)v * N);
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = r.at(i);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = v * N + i < cols ? to_f32(row[(uint64_t)v * N + i]) : 0.f;
    }
  };
  float keep[kKeep][N];
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < kKeep; ++k) {
    const uint32_t v = threadIdx.x + k * blockDim.x;
    if (v < nv) {
      fetch(v, keep[k]);
#pragma unroll
      for (int i = 0; i < N; ++i) top = max(top, mag_bits(keep[k][i]));
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) keep[k][i] = 0.f;
    }
  }
  for (uint32_t v = threadIdx.x + kKeep * blockDim.x; v < nv; v += blockDim.x) {
    float f[N];
    fetch(v, f);
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, mag_bits(f[i]));
  }
  __shared__ uint32_t tops[8];
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
  for (uint32_t i = 0; i < blockDim.x / 32; ++i) top = max(top, tops[i]);
  float s, inv;
  scale_of(top, s, inv);
  if (threadIdx.x == 0) scale[blockIdx.x] = s;
  auto emit = [&](uint32_t v, const float (&f)[N]) {
    uint32_t w[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      w[i] = pack4(code_of(f[4 * i], inv), code_of(f[4 * i + 1], inv), code_of(f[4 * i + 2], inv), code_of(f[4 * i + 3], inv));
    if constexpr (N == 8)
      *reinterpret_cast<uint2*>(out + v * N) = make_uint2(w[0], w[1]);
    else
      *reinterpret_cast<uint32_t*>(out + v * N) = w[0];
  };
#pragma unroll
  for (int k = 0; k < kKeep; ++k) {
    const uint32_t v = threadIdx.x + k * blockDim.x;
    if (v < nv_out) emit(v, keep[k]);
  }
  for (uint32_t v = threadIdx.x + kKeep * blockDim.x; v < nv_out; v += blockDim.x) {
    float f[N];
    fetch(v, f);
    emit(v, f);
  }
}

// ---- by columns, or by rows and columns at once ----
// First reading: the largest magnitude of every row and column (as bits, by atomic maxima: the same whatever the order) and,
// for the gradient of a bias, the column sums of each block of kAmaxRows rows.
constexpr int kAmaxRows = 64;

template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_i8_amax(const T* x, uint64_t ld, uint32_t rows, uint32_t cols, uint32_t* row_top,
                                                 uint32_t* col_top, float* sums) {
  pdl_prologue();
  constexpr int N = Vec<T>::kN;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t c = (blockIdx.x * 32 + lane) * N, r0 = blockIdx.y * kAmaxRows;
  uint32_t top[N];
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) top[i] = 0, sum[i] = 0.f;
#pragma unroll
  for (int k = 0; k < kAmaxRows / 8; ++k) {
    const uint32_t r = r0 + warp + 8 * k;
    uint32_t mine = 0;
    if (r < rows && c < cols) {
      float f[N];
      if (VEC && c + N <= cols) {
        Vec<T> v;
        v.raw = __ldg(reinterpret_cast<const uint4*>(x + r * ld + c));
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = v.at(i);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = c + i < cols ? to_f32(x[r * ld + c + i]) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint32_t b = mag_bits(f[i]);
        mine = max(mine, b);
        top[i] = max(top[i], b);
        sum[i] += f[i];
      }
    }
    mine = __reduce_max_sync(0xFFFFFFFFu, mine);
    if (row_top && lane == 0 && r < rows && mine) atomicMax(row_top + r, mine);
  }
  __shared__ uint32_t tops[8][32 * N];
  __shared__ float part[8][32 * N];
#pragma unroll
  for (int i = 0; i < N; ++i) tops[warp][lane + 32 * i] = top[i], part[warp][lane + 32 * i] = sum[i];
  __syncthreads();
  for (int t = threadIdx.x; t < 32 * N; t += 256) {
    uint32_t m = 0;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, tops[w][t]), s += part[w][t];
    const uint32_t col = (blockIdx.x * 32 + t % 32) * N + t / 32;
    if (col < cols) {
      if (col_top && m) atomicMax(col_top + col, m);
      if (sums) sums[(uint64_t)blockIdx.y * cols + col] = s;
    }
  }
}

// Second reading: the codes.  A tile is 128 rows x 64 columns; a thread takes blocks of 4 x 4, writes their rows straight and
// their columns through shared memory, so that a column's 128 codes leave as one line.
template <class T, bool VEC>
__global__ void __launch_bounds__(256)
    k_i8_codes(const T* x, uint64_t ld, uint32_t rows, uint32_t cols, const uint32_t* row_top, const uint32_t* col_top, const float* sums,
               int8_t* q, uint64_t ldq, float* scale, int8_t* qt, uint64_t ldqt, float* scale_t, float* col_sum) {
  pdl_prologue();
  __shared__ float rinv[128], cinv[64];
  __shared__ uint32_t turned[64][33];
  const uint32_t r0 = blockIdx.y * 128, c0 = blockIdx.x * 64, tid = threadIdx.x;
  if (tid < 128) {
    const uint32_t r = r0 + tid;
    if (q && r < rows) {
      float s, inv;
      scale_of(row_top[r], s, inv);
      rinv[tid] = inv;
      if (blockIdx.x == 0) scale[r] = s;
    }
  } else if (tid < 192) {
    const uint32_t c = c0 + tid - 128;
    if (c < cols) {
      if (qt) {
        float s, inv;
        scale_of(col_top[c], s, inv);
        cinv[tid - 128] = inv;
        if (blockIdx.y == 0) scale_t[c] = s;
      }
      if (col_sum && blockIdx.y == 0) {
        float s = 0.f;
        for (uint32_t k = 0; k < (rows + kAmaxRows - 1) / kAmaxRows; ++k) s += sums[(uint64_t)k * cols + c];
        col_sum[c] = s;
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const uint32_t lc = tid % 16 * 4, lr = (tid / 16 + 16 * half) * 4, c = c0 + lc;
    float f[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t r = r0 + lr + i;
      const T* p = x + r * ld + c;
      if (VEC && r < rows && c + 4 <= cols) {
        if constexpr (sizeof(T) == 4) {
          const float4 v = __ldg(reinterpret_cast<const float4*>(p));
          f[i][0] = v.x, f[i][1] = v.y, f[i][2] = v.z, f[i][3] = v.w;
        } else {
          const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
#pragma unroll
          for (int j = 0; j < 4; ++j) f[i][j] = to_f32(reinterpret_cast<const T*>(&v)[j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[i][j] = r < rows && c + j < cols ? to_f32(p[j]) : 0.f;
      }
    }
    if (q) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t r = r0 + lr + i;
        const float v = rinv[lr + i];
        if (r < rows && c < ldq)
          *reinterpret_cast<uint32_t*>(q + r * ldq + c) =
              pack4(code_of(f[i][0], v), code_of(f[i][1], v), code_of(f[i][2], v), code_of(f[i][3], v));
      }
    }
    if (qt) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float v = c + j < cols ? cinv[lc + j] : 0.f;
        turned[lc + j][lr / 4] = pack4(code_of(f[0][j], v), code_of(f[1][j], v), code_of(f[2][j], v), code_of(f[3][j], v));
      }
    }
  }
  if (!qt) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t lc = tid / 32 + 8 * k, w = tid % 32;
    if (c0 + lc < cols && r0 + 4 * w < ldqt) *reinterpret_cast<uint32_t*>(qt + (uint64_t)(c0 + lc) * ldqt + r0 + 4 * w) = turned[lc][w];
  }
}

// ---- the product's epilogue ----

__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store1(__half* p, float v) { *p = __float2half_rn(v); }

template <class T>
struct EpiScale {
  struct Pre {
    float s;
  };
  const float *sa, *sb, *bias;
  T* out;
  uint64_t ld;
  uint32_t m, n;
  int vec;   // rows of out, sb and bias start on 16-byte boundaries
  __device__ __forceinline__ Pre load(uint32_t row, uint32_t, uint32_t) const { return {row < m ? __ldg(sa + row) : 0.f}; }
  __device__ __forceinline__ void apply(const Pre& p, const uint32_t (&acc)[32], uint32_t row, uint32_t col0, uint32_t) const {
    if (row >= m) return;
    T* o = out + row * ld + col0;
    if (vec && col0 + 32 <= n) {
#pragma unroll
      for (int i = 0; i < 32; i += 16 / sizeof(T)) {
        T t[16 / sizeof(T)];
#pragma unroll
        for (int j = 0; j < 16 / (int)sizeof(T); j += 4) {
          const float4 s = __ldg(reinterpret_cast<const float4*>(sb + col0 + i + j));
          float4 c = make_float4(0.f, 0.f, 0.f, 0.f);
          if (bias) c = __ldg(reinterpret_cast<const float4*>(bias + col0 + i + j));
          store1(t + j, __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[i + j], p.s), s.x), c.x));
          store1(t + j + 1, __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[i + j + 1], p.s), s.y), c.y));
          store1(t + j + 2, __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[i + j + 2], p.s), s.z), c.z));
          store1(t + j + 3, __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[i + j + 3], p.s), s.w), c.w));
        }
        *reinterpret_cast<uint4*>(o + i) = *reinterpret_cast<uint4*>(t);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (col0 + j < n)
          store1(o + j, __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[j], p.s), __ldg(sb + col0 + j)), bias ? __ldg(bias + col0 + j) : 0.f));
    }
  }
};

// An empty sum (K = 0): the bias alone.
template <class T>
__global__ void __launch_bounds__(kThreads) k_i8_empty(T* out, uint64_t ld, uint32_t n, const float* bias) {
  pdl_prologue();
  for (uint32_t c = threadIdx.x; c < n; c += kThreads) store1(out + blockIdx.x * ld + c, bias ? bias[c] : 0.f);
}

inline uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }
inline bool aligned(const void* p, uint64_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline uint32_t size_of(int dtype) { return dtype == DS_F32 ? 4 : 2; }
inline bool dtype_ok(int t) { return t == DS_F32 || t == DS_BF16 || t == DS_F16; }
constexpr uint64_t kMaxLen = 1ull << 30;

template <class T>
cudaError_t product(const int8_t* a, uint64_t lda, const float* sa, const int8_t* b, uint64_t ldb, const float* sb, const float* bias,
                    uint32_t m, uint32_t n, uint32_t k, T* out, uint64_t ldo, uint32_t* dev_status, cudaStream_t st) {
  if (k == 0) {
    launch_pdl(k_i8_empty<T>, dim3(m), dim3(kThreads), st, out, ldo, n, bias);
    count_launches(1);
    return cudaGetLastError();
  }
  const MmaShape s{m, n, k, 1, 0, dev_status};
  const EpiScale<T> epi{sa, sb, bias, out, ldo, m, n,
                        aligned(out, 16) && ldo * sizeof(T) % 16 == 0 && aligned(sb, 16) && (!bias || aligned(bias, 16))};
  const int bn = pick_bn(s, sm_count());
  CUtensorMap ma, mb;
  cudaError_t e = make_tensor_map(&ma, kMmaI8, a, k, m, 1, lda, lda * m, 128, kMmaRows);
  if (e == cudaSuccess) e = make_tensor_map(&mb, kMmaI8, b, k, n, 1, ldb, ldb * n, 128, bn);
  if (e != cudaSuccess) return e;
  switch (bn) {
    case 256: return launch_mma_bn<kMmaI8, 256, false>(ma, mb, s, epi, st);
    case 192: return launch_mma_bn<kMmaI8, 192, false>(ma, mb, s, epi, st);
    case 128: return launch_mma_bn<kMmaI8, 128, false>(ma, mb, s, epi, st);
    default: return launch_mma_bn<kMmaI8, 64, false>(ma, mb, s, epi, st);
  }
}

template <class T>
cudaError_t quantize(const T* x, uint32_t rows, uint32_t cols, uint64_t ld, int8_t* q, uint64_t ldq, float* scale, int8_t* qt, uint64_t ldqt,
                     float* scale_t, float* col_sum, uint8_t* ws, cudaStream_t st) {
  const bool vec = aligned(x, 16) && ld * sizeof(T) % 16 == 0;
  if (!qt && !col_sum) {
    // as many threads as the row has vectors for two each, at most 256
    const uint32_t nv = (cols + 15) / 16 * 16 / (vec ? Vec<T>::kN : 4);
    const uint32_t want = (uint32_t)round_up((nv + 1) / 2, 32), bs = want < 32 ? 32 : want > 256 ? 256 : want;
    if (vec)
      launch_pdl(k_i8_rows<T, true>, dim3(rows), dim3(bs), st, x, ld, cols, q, ldq, scale);
    else
      launch_pdl(k_i8_rows<T, false>, dim3(rows), dim3(bs), st, x, ld, cols, q, ldq, scale);
    count_launches(1);
    return cudaGetLastError();
  }
  uint32_t* row_top = reinterpret_cast<uint32_t*>(ws);
  uint32_t* col_top = row_top + round_up(rows, 64);
  float* sums = col_sum ? reinterpret_cast<float*>(col_top + round_up(cols, 64)) : nullptr;
  cudaError_t e = cudaMemsetAsync(ws, 0, 4 * (round_up(rows, 64) + round_up(cols, 64)), st);
  if (e != cudaSuccess) return e;
  const dim3 g1((cols + 32 * Vec<T>::kN - 1) / (32 * Vec<T>::kN), (rows + kAmaxRows - 1) / kAmaxRows), g2((cols + 63) / 64, (rows + 127) / 128);
  uint32_t *rt = q ? row_top : nullptr, *ct = qt ? col_top : nullptr;
  if (vec) {
    launch_pdl(k_i8_amax<T, true>, g1, dim3(256), st, x, ld, rows, cols, rt, ct, sums);
    launch_pdl(k_i8_codes<T, true>, g2, dim3(256), st, x, ld, rows, cols, (const uint32_t*)rt, (const uint32_t*)ct, (const float*)sums, q,
               ldq, scale, qt, ldqt, scale_t, col_sum);
  } else {
    launch_pdl(k_i8_amax<T, false>, g1, dim3(256), st, x, ld, rows, cols, rt, ct, sums);
    launch_pdl(k_i8_codes<T, false>, g2, dim3(256), st, x, ld, rows, cols, (const uint32_t*)rt, (const uint32_t*)ct, (const float*)sums, q,
               ldq, scale, qt, ldqt, scale_t, col_sum);
  }
  count_launches(2);
  return cudaGetLastError();
}

// Shared checks of an 8-bit matrix: rows on 16-byte boundaries.
int check_codes(const void* q, uint64_t ld, uint64_t cols) {
  if (!q) return DS_ERR_INVALID_ARG;
  if (ld < cols) return DS_ERR_INVALID_ARG;
  if (!aligned(q, 16) || ld % 16) return DS_ERR_ALIGN;
  return DS_OK;
}

}  // namespace

extern "C" {

uint64_t ds_i8_quantize_workspace(uint64_t rows, uint64_t cols, int with_col_sum) {
  return 4 * (round_up(rows, 64) + round_up(cols, 64)) + (with_col_sum ? 4 * ((rows + kAmaxRows - 1) / kAmaxRows) * cols : 0);
}

int ds_i8_quantize(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int8_t* q, uint64_t ldq, float* scale,
                   int8_t* qt, uint64_t ldqt, float* scale_t, float* col_sum, void* workspace, size_t workspace_bytes,
                   void* cuda_stream) {
  if (!dtype_ok(dtype) || rows > kMaxLen || cols > kMaxLen || ld < cols) return DS_ERR_INVALID_ARG;
  if (!aligned(x, size_of(dtype)) || !aligned(scale, 4) || !aligned(scale_t, 4) || !aligned(col_sum, 4)) return DS_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (rows == 0 || cols == 0) {   // no codes; scales and sums of empty lines are 0
    cudaError_t e = cudaSuccess;
    if (scale && rows) e = cudaMemsetAsync(scale, 0, 4 * rows, st);
    if (e == cudaSuccess && scale_t && cols) e = cudaMemsetAsync(scale_t, 0, 4 * cols, st);
    if (e == cudaSuccess && col_sum && cols) e = cudaMemsetAsync(col_sum, 0, 4 * cols, st);
    return e == cudaSuccess ? DS_OK : cuda_fail(e, "clearing scales");
  }
  if ((!q != !scale) || (!qt != !scale_t) || (!q && !qt && !col_sum)) return DS_ERR_INVALID_ARG;
  int rc;
  if (q && (rc = check_codes(q, ldq, cols)) != DS_OK) return rc;
  if (qt && (rc = check_codes(qt, ldqt, rows)) != DS_OK) return rc;
  if (!x) return DS_ERR_INVALID_ARG;
  if (qt || col_sum) {
    if (!workspace || !aligned(workspace, 16)) return workspace ? DS_ERR_ALIGN : DS_ERR_INVALID_ARG;
    if (workspace_bytes < ds_i8_quantize_workspace(rows, cols, col_sum != nullptr)) return DS_ERR_BUFFER_TOO_SMALL;
    if (rows > 65535ull * kAmaxRows) return DS_ERR_UNSUPPORTED;   // rows of blocks in one launch
  }
  const uint32_t r = (uint32_t)rows, c = (uint32_t)cols;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const cudaError_t e =
      dtype == DS_F32    ? quantize(static_cast<const float*>(x), r, c, ld, q, ldq, scale, qt, ldqt, scale_t, col_sum, ws, st)
      : dtype == DS_BF16 ? quantize(static_cast<const __nv_bfloat16*>(x), r, c, ld, q, ldq, scale, qt, ldqt, scale_t, col_sum, ws, st)
                         : quantize(static_cast<const __half*>(x), r, c, ld, q, ldq, scale, qt, ldqt, scale_t, col_sum, ws, st);
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "8-bit quantiser");
}

int ds_i8_matmul(const int8_t* a, uint64_t lda, const float* sa, const int8_t* b, uint64_t ldb, const float* sb, const float* bias,
                 uint64_t m, uint64_t n, uint64_t k, void* out, int out_dtype, uint64_t ldo, uint32_t* dev_status, void* cuda_stream) {
  if (!dtype_ok(out_dtype) || m > kMaxLen || n > kMaxLen || ldo < n) return DS_ERR_INVALID_ARG;
  if (k > DS_I8_MAX_K) return DS_ERR_UNSUPPORTED;
  if (m == 0 || n == 0) return DS_OK;
  if (!sa || !sb || !out) return DS_ERR_INVALID_ARG;
  int rc;
  if (k && ((rc = check_codes(a, lda, k)) != DS_OK || (rc = check_codes(b, ldb, k)) != DS_OK)) return rc;
  if (!aligned(sa, 4) || !aligned(sb, 4) || !aligned(bias, 4) || !aligned(out, size_of(out_dtype)) || !aligned(dev_status, 4))
    return DS_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const uint32_t M = (uint32_t)m, N = (uint32_t)n, K = (uint32_t)k;
  const cudaError_t e =
      out_dtype == DS_F32    ? product(a, lda, sa, b, ldb, sb, bias, M, N, K, static_cast<float*>(out), ldo, dev_status, st)
      : out_dtype == DS_BF16 ? product(a, lda, sa, b, ldb, sb, bias, M, N, K, static_cast<__nv_bfloat16*>(out), ldo, dev_status, st)
                             : product(a, lda, sa, b, ldb, sb, bias, M, N, K, static_cast<__half*>(out), ldo, dev_status, st);
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "8-bit product");
}

uint64_t ds_i8_linear_workspace(uint64_t rows, uint64_t k) { return rows * round_up(k, 16) + 4 * round_up(rows, 64); }

int ds_i8_linear(const void* x, int dtype, uint64_t rows, uint64_t k, uint64_t ldx, const int8_t* w, uint64_t ldw, const float* sw,
                 const float* bias, uint64_t n, void* out, int out_dtype, uint64_t ldo, void* workspace, size_t workspace_bytes,
                 uint32_t* dev_status, void* cuda_stream) {
  if (rows > kMaxLen || k > DS_I8_MAX_K) return rows > kMaxLen ? DS_ERR_INVALID_ARG : DS_ERR_UNSUPPORTED;
  if (rows == 0 || n == 0) return dtype_ok(dtype) && dtype_ok(out_dtype) ? DS_OK : DS_ERR_INVALID_ARG;
  if (!workspace) return DS_ERR_INVALID_ARG;
  if (!aligned(workspace, 16)) return DS_ERR_ALIGN;
  if (workspace_bytes < ds_i8_linear_workspace(rows, k)) return DS_ERR_BUFFER_TOO_SMALL;
  const uint64_t ldq = round_up(k, 16);
  float* s = static_cast<float*>(workspace);
  int8_t* q = static_cast<int8_t*>(workspace) + 4 * round_up(rows, 64);
  const int rc = ds_i8_quantize(x, dtype, rows, k, ldx, q, ldq, s, nullptr, 0, nullptr, nullptr, nullptr, 0, cuda_stream);
  if (rc != DS_OK) return rc;
  return ds_i8_matmul(q, ldq, s, w, ldw, sw, bias, rows, n, k, out, out_dtype, ldo, dev_status, cuda_stream);
}

}  // extern "C"
