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
#include <type_traits>

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
// round(v * inv) in the low byte: adding 1.5 * 2^23 rounds to the nearest whole number, ties to even, and leaves it in the low
// bits (conversions run at a fraction of the rate of additions).  Of a line with inv = 0 the codes are masked: v may be inf or NaN.
__device__ __forceinline__ uint32_t code_of(float v, float inv) { return __float_as_uint(__fadd_rn(__fmul_rn(v, inv), 12582912.f)); }
__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  const uint32_t w = pack4(code_of(a, inv), code_of(b, inv), code_of(c, inv), code_of(d, inv));
  return inv != 0.f ? w : 0u;
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

// 16 bytes of x as floats.
template <class T>
struct Vec {
  static constexpr int kN = 16 / sizeof(T);
  uint4 raw;
  __device__ __forceinline__ float at(int i) const {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {   // the upper half of a float: one instruction, where an extraction takes two
      const uint32_t w = reinterpret_cast<const uint32_t*>(&raw)[i >> 1];
      return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
    } else {
      return to_f32(reinterpret_cast<const T*>(&raw)[i]);
    }
  }
  __device__ __forceinline__ void set(int i, T t) { reinterpret_cast<T*>(&raw)[i] = t; }
};

// ---- by rows: one CTA a row, one reading ----
// WHOLE: the row is whole vectors of 16 bytes on 16-byte boundaries, at most kKeep of them a thread: they are fetched together
// and stay in registers between the row's maximum and its codes.  Else entry by entry, from cache the second time.  Codes from
// `cols` up to the next multiple of 16 are written as 0.
constexpr int kKeep = 8;

template <class T, bool WHOLE>
__global__ void __launch_bounds__(256) k_i8_rows(const T* x, uint64_t ld, uint32_t cols, int8_t* q, uint64_t ldq, float* scale) {
  pdl_prologue();
  constexpr int N = Vec<T>::kN;
  const T* row = x + (uint64_t)blockIdx.x * ld;
  int8_t* out = q + (uint64_t)blockIdx.x * ldq;
  const uint32_t nv = cols / N;
  Vec<T> keep[WHOLE ? kKeep : 1];
  uint32_t top = 0;
  if constexpr (WHOLE) {
#pragma unroll
    for (int k = 0; k < kKeep; ++k) {
      const uint32_t v = threadIdx.x + k * blockDim.x;
      keep[k].raw = v < nv ? ld_plain(reinterpret_cast<const uint4*>(row) + v) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kKeep; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) top = max(top, mag_bits(keep[k].at(i)));
  } else {
#pragma unroll 4
    for (uint32_t c = threadIdx.x; c < cols; c += blockDim.x) top = max(top, mag_bits(to_f32(row[c])));
  }
  __shared__ uint32_t tops[8];
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
  for (uint32_t i = 0; i < blockDim.x / 32; ++i) top = max(top, tops[i]);
  float s, inv;
  scale_of(top, s, inv);
  if (threadIdx.x == 0) scale[blockIdx.x] = s;
  if constexpr (WHOLE) {
#pragma unroll
    for (int k = 0; k < kKeep; ++k) {
      const uint32_t v = threadIdx.x + k * blockDim.x;
      if (v >= nv) break;
      uint32_t w[N / 4];
#pragma unroll
      for (int i = 0; i < N / 4; ++i)
        w[i] = codes4(keep[k].at(4 * i), keep[k].at(4 * i + 1), keep[k].at(4 * i + 2), keep[k].at(4 * i + 3), inv);
      if constexpr (N == 8)
        *reinterpret_cast<uint2*>(out + v * N) = make_uint2(w[0], w[1]);
      else
        *reinterpret_cast<uint32_t*>(out + v * N) = w[0];
    }
    if (threadIdx.x < 16 && cols + threadIdx.x < (cols + 15) / 16 * 16) out[cols + threadIdx.x] = 0;
  } else {
#pragma unroll 2
    for (uint32_t c = threadIdx.x * 4; c < (cols + 15) / 16 * 16; c += blockDim.x * 4) {
      float f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = c + i < cols ? to_f32(row[c + i]) : 0.f;
      *reinterpret_cast<uint32_t*>(out + c) = codes4(f[0], f[1], f[2], f[3], inv);
    }
  }
}

// ---- by columns, or by rows and columns at once ----
// First reading: the largest magnitude of every row and column (as bits, by atomic maxima: the same whatever the order) and,
// for the gradient of a bias, the column sums of each block of kAmaxRows rows.
constexpr int kAmaxRows = 64;

template <class T, bool VEC, bool SUMS>
__global__ void __launch_bounds__(256) k_i8_amax(const T* x, uint64_t ld, uint32_t rows, uint32_t cols, uint32_t* row_top,
                                                 uint32_t* col_top, float* sums) {
  pdl_prologue();
  constexpr int N = Vec<T>::kN, kRows = kAmaxRows / 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // a lane's columns: a vector's, or (rows on no boundary) every 32nd, so that a warp reads consecutive entries
  const uint32_t c0 = blockIdx.x * 32 * N, r0 = blockIdx.y * kAmaxRows;
  auto col = [&](int i) { return c0 + (VEC ? lane * N + i : lane + 32 * i); };
  uint32_t top[N];
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) top[i] = 0, sum[i] = 0.f;
  Vec<T> v[kRows];
  if (VEC && c0 + 32 * N <= cols && r0 + kAmaxRows <= rows) {   // inside
#pragma unroll
    for (int k = 0; k < kRows; ++k) v[k].raw = ld_plain(reinterpret_cast<const uint4*>(x + (uint64_t)(r0 + warp + 8 * k) * ld + col(0)));
  } else {
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const uint32_t r = r0 + warp + 8 * k;
      v[k].raw = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (r < rows && col(i) < cols) v[k].set(i, x[(uint64_t)r * ld + col(i)]);
    }
  }
  uint32_t row_max = 0;      // of row k in lane k: one atomic instruction for the warp's eight rows
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float f = v[k].at(i);
      const uint32_t b = mag_bits(f);
      mine = max(mine, b);
      top[i] = max(top[i], b);
      if constexpr (SUMS) sum[i] += f;
    }
    mine = __reduce_max_sync(0xFFFFFFFFu, mine);
    if (lane == k) row_max = mine;
  }
  if (row_top && row_max && r0 + warp + 8 * lane < rows) atomicMax(row_top + r0 + warp + 8 * lane, row_max);
  __shared__ uint32_t tops[8][32 * N];
  __shared__ float part[SUMS ? 8 : 1][SUMS ? 32 * N : 1];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    tops[warp][lane + 32 * i] = top[i];
    if constexpr (SUMS) part[warp][lane + 32 * i] = sum[i];
  }
  __syncthreads();
  for (int t = threadIdx.x; t < 32 * N; t += 256) {
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, tops[w][t]);
    const uint32_t at = c0 + (VEC ? t % 32 * N + t / 32 : t);
    if (at < cols) {
      if (col_top && m) atomicMax(col_top + at, m);
      if constexpr (SUMS) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += part[w][t];
        sums[(uint64_t)blockIdx.y * cols + at] = s;
      }
    }
  }
}

// Codes of a line end on the next multiple of 16, whatever lies between that and the next line: it may be another matrix.
__device__ __forceinline__ uint32_t padded(uint32_t n) { return (n + 15) / 16 * 16; }

// Second reading: the codes.  A tile is 128 x 128; a thread takes blocks of 4 rows x 8 columns, writes their rows straight and
// their columns through shared memory, so that a column's 128 codes leave as one line.
template <class T>
__global__ void __launch_bounds__(256)
    k_i8_codes(const T* x, uint64_t ld, uint32_t rows, uint32_t cols, const uint32_t* row_top, const uint32_t* col_top, const float* sums,
               int8_t* q, uint64_t ldq, float* scale, int8_t* qt, uint64_t ldqt, float* scale_t, float* col_sum) {
  pdl_prologue();
  constexpr int N = Vec<T>::kN, V = 8 / N;     // vectors of 16 bytes in 8 columns
  __shared__ float rinv[128], cinv[128];
  // a column's 32 words in pieces of 16 bytes, exchanged by the column's number: writes of a warp meet two to a bank, reads none
  __shared__ __align__(16) uint32_t turned[128][32];
  const uint32_t r0 = blockIdx.y * 128, c0 = blockIdx.x * 128, tid = threadIdx.x;
  const bool inside = r0 + 128 <= rows && c0 + 128 <= cols;
  const uint32_t lc = tid % 16 * 8, c = c0 + lc;
  Vec<T> v[4][V];
  auto fetch = [&](int half) {
    const uint32_t r = r0 + (tid / 16 + 16 * half) * 4;
    if (inside) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) v[i][j].raw = ld_plain(reinterpret_cast<const uint4*>(x + (uint64_t)(r + i) * ld + c) + j);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (j % N == 0) v[i][j / N].raw = make_uint4(0, 0, 0, 0);
          if (r + i < rows && c + j < cols) v[i][j / N].set(j % N, x[(uint64_t)(r + i) * ld + c + j]);
        }
    }
  };
  fetch(0);
  if (tid < 128) {
    const uint32_t r = r0 + tid;
    float s = 0.f, inv = 0.f;
    if (q && r < rows) {
      scale_of(row_top[r], s, inv);
      if (blockIdx.x == 0) scale[r] = s;
    }
    rinv[tid] = inv;
  } else {
    const uint32_t k = c0 + tid - 128;
    float s = 0.f, inv = 0.f;
    if (qt && k < cols) {
      scale_of(col_top[k], s, inv);
      if (blockIdx.y == 0) scale_t[k] = s;
    }
    cinv[tid - 128] = inv;
    if (col_sum && blockIdx.y == 0 && k < cols) {
      float t = 0.f;
#pragma unroll 4
      for (uint32_t b = 0; b < (rows + kAmaxRows - 1) / kAmaxRows; ++b) t += sums[(uint64_t)b * cols + k];
      col_sum[k] = t;
    }
  }
  __syncthreads();
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const uint32_t lr = (tid / 16 + 16 * half) * 4;
    if (half) fetch(1);
    auto at = [&](int i, int j) { return v[i][j / N].at(j % N); };
    if (q) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t r = r0 + lr + i;
        const float f = rinv[lr + i];
        const uint32_t w0 = codes4(at(i, 0), at(i, 1), at(i, 2), at(i, 3), f), w1 = codes4(at(i, 4), at(i, 5), at(i, 6), at(i, 7), f);
        if (r < rows && c < padded(cols)) *reinterpret_cast<uint2*>(q + (uint64_t)r * ldq + c) = make_uint2(w0, w1);
      }
    }
    if (qt) {
#pragma unroll
      for (int j = 0; j < 8; ++j) turned[lc + j][((lr / 16) ^ ((lc + j) / 8 & 7)) * 4 + lr / 4 % 4] = codes4(at(0, j), at(1, j), at(2, j), at(3, j), cinv[lc + j]);
    }
  }
  if (!qt) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t l = tid / 8 + 32 * k, piece = tid % 8;
    if (c0 + l < cols && r0 + 16 * piece < padded(rows))
      *reinterpret_cast<uint4*>(qt + (uint64_t)(c0 + l) * ldqt + r0 + 16 * piece) =
          *reinterpret_cast<const uint4*>(&turned[l][(piece ^ (l / 8 & 7)) * 4]);
  }
}

// The same where rows start on no boundary of 16 bytes: tiles of 64 x 64, read entry by entry along the rows and handed to their
// threads through shared memory (straight reads of 4 x 8 blocks took twice as long: 1999 x 1153 floats 9.2 us, now 6.1).
template <class T>
__global__ void __launch_bounds__(256)
    k_i8_codes_odd(const T* x, uint64_t ld, uint32_t rows, uint32_t cols, const uint32_t* row_top, const uint32_t* col_top, const float* sums,
                   int8_t* q, uint64_t ldq, float* scale, int8_t* qt, uint64_t ldqt, float* scale_t, float* col_sum) {
  pdl_prologue();
  __shared__ float rinv[64], cinv[64], tile[64][65];
  __shared__ uint32_t turned[64][17];
  const uint32_t r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, tid = threadIdx.x;
  float v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t r = r0 + tid / 64 + 4 * i, c = c0 + tid % 64;
    v[i] = r < rows && c < cols ? to_f32(x[(uint64_t)r * ld + c]) : 0.f;
  }
  if (tid < 64) {
    float s = 0.f, inv = 0.f;
    if (q && r0 + tid < rows) {
      scale_of(row_top[r0 + tid], s, inv);
      if (blockIdx.x == 0) scale[r0 + tid] = s;
    }
    rinv[tid] = inv;
  } else if (tid < 128) {
    const uint32_t k = c0 + tid - 64;
    float s = 0.f, inv = 0.f;
    if (qt && k < cols) {
      scale_of(col_top[k], s, inv);
      if (blockIdx.y == 0) scale_t[k] = s;
    }
    cinv[tid - 64] = inv;
  } else if (tid < 192) {
    const uint32_t k = c0 + tid - 128;
    if (col_sum && blockIdx.y == 0 && k < cols) {
      float t = 0.f;
#pragma unroll 4
      for (uint32_t b = 0; b < (rows + kAmaxRows - 1) / kAmaxRows; ++b) t += sums[(uint64_t)b * cols + k];
      col_sum[k] = t;
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) tile[tid / 64 + 4 * i][tid % 64] = v[i];
  __syncthreads();
  const uint32_t lc = tid % 16 * 4, lr = tid / 16 * 4, c = c0 + lc;
  float f[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) f[i][j] = tile[lr + i][lc + j];
  if (q) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (r0 + lr + i < rows && c < padded(cols))
        *reinterpret_cast<uint32_t*>(q + (uint64_t)(r0 + lr + i) * ldq + c) = codes4(f[i][0], f[i][1], f[i][2], f[i][3], rinv[lr + i]);
  }
  if (!qt) return;
#pragma unroll
  for (int j = 0; j < 4; ++j) turned[lc + j][lr / 4] = codes4(f[0][j], f[1][j], f[2][j], f[3][j], cinv[lc + j]);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t l = tid / 16 + 16 * k, w = tid % 16;
    if (c0 + l < cols && r0 + 4 * w < padded(rows)) *reinterpret_cast<uint32_t*>(qt + (uint64_t)(c0 + l) * ldqt + r0 + 4 * w) = turned[l][w];
  }
}

// Both readings in one launch, for matrices so small that launches are what they cost: a CTA looks its tile's rows and columns
// through from end to end for their largest magnitudes (the matrix lies in L2; 512 x 768: 16 MB of reads in all), then encodes
// the tile, 64 x 64.  512 x 768 in bf16: 7.6 us, and one launch for the host instead of three.
// Warps 0..7 hold the tile and look through its rows, warps 8..15 through its columns.
template <class T>
__global__ void __launch_bounds__(512)
    k_i8_small(const T* x, uint64_t ld, uint32_t rows, uint32_t cols, int8_t* q, uint64_t ldq, float* scale, int8_t* qt, uint64_t ldqt,
               float* scale_t, float* col_sum) {
  pdl_prologue();
  constexpr int N = Vec<T>::kN, kLanes = 64 / N, kStep = 256 / kLanes;    // lanes across 64 columns; rows that eight warps take at once
  __shared__ float rinv[64], cinv[64];
  __shared__ uint32_t tops[kStep][64 + 1], turned[64][17];
  __shared__ float part[kStep][64 + 1];
  const uint32_t r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, tid = threadIdx.x & 255, warp = tid >> 5, lane = tid & 31;
  auto vec_at = [&](uint32_t r, uint32_t c) { return ld_plain(reinterpret_cast<const uint4*>(x + (uint64_t)r * ld + c)); };   // c < cols, a multiple of N
  const uint32_t lc = tid % 16 * 4, lr = tid / 16 * 4, c = c0 + lc;        // 4 x 4 blocks of the tile
  float f[4][4];
  if (threadIdx.x < 256) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = r0 + lr + i < rows && c < cols;     // cols is a multiple of 4
      const T* p = x + (uint64_t)(r0 + lr + i) * ld + c;
      if constexpr (sizeof(T) == 4) {
        const float4 v = in ? ld_plain(reinterpret_cast<const float4*>(p)) : make_float4(0.f, 0.f, 0.f, 0.f);
        f[i][0] = v.x, f[i][1] = v.y, f[i][2] = v.z, f[i][3] = v.w;
      } else {
        const uint2 v = in ? ld_plain(reinterpret_cast<const uint2*>(p)) : make_uint2(0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[i][j] = to_f32(reinterpret_cast<const T*>(&v)[j]);
      }
    }
    uint32_t top[8] = {};      // eight rows a warp
    if (q)
      for (uint32_t k = lane * N; k < cols; k += 32 * N) {
        Vec<T> v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i].raw = r0 + warp * 8 + i < rows ? vec_at(r0 + warp * 8 + i, k) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int j = 0; j < N; ++j) top[i] = max(top[i], mag_bits(v[i].at(j)));
      }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, top[i]);
      if (lane == i && q) {
        float s, inv;
        scale_of(m, s, inv);
        rinv[warp * 8 + i] = inv;
        if (blockIdx.x == 0 && r0 + warp * 8 + i < rows) scale[r0 + warp * 8 + i] = s;
      }
    }
  } else if (qt || col_sum) {
    const uint32_t k = c0 + tid % kLanes * N, first = tid / kLanes;
    uint32_t top[N] = {};
    float sum[N] = {};
    if (k < cols) {
      for (uint32_t r = first; r < rows; r += 8 * kStep) {
        Vec<T> v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i].raw = r + i * kStep < rows ? vec_at(r + i * kStep, k) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < N; ++j) {
#pragma unroll
          for (int i = 0; i < 8; ++i) top[j] = max(top[j], mag_bits(v[i].at(j)));
          sum[j] += ((v[0].at(j) + v[1].at(j)) + (v[2].at(j) + v[3].at(j))) + ((v[4].at(j) + v[5].at(j)) + (v[6].at(j) + v[7].at(j)));
        }
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) tops[first][tid % kLanes * N + j] = top[j], part[first][tid % kLanes * N + j] = sum[j];
    // the eight warps of the columns alone
    asm volatile("bar.sync 1, 256;" ::: "memory");
    if (tid < 64) {
      uint32_t m = 0;
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < kStep; i += 4) {
        m = max(max(m, tops[i][tid]), max(tops[i + 1][tid], max(tops[i + 2][tid], tops[i + 3][tid])));
        t += (part[i][tid] + part[i + 1][tid]) + (part[i + 2][tid] + part[i + 3][tid]);
      }
      float s, inv;
      scale_of(m, s, inv);
      cinv[tid] = inv;
      if (blockIdx.y == 0 && c0 + tid < cols) {
        if (qt) scale_t[c0 + tid] = s;
        if (col_sum) col_sum[c0 + tid] = t;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x < 256) {
    if (q) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (r0 + lr + i < rows && c < padded(cols))
          *reinterpret_cast<uint32_t*>(q + (uint64_t)(r0 + lr + i) * ldq + c) = codes4(f[i][0], f[i][1], f[i][2], f[i][3], rinv[lr + i]);
    }
    if (qt) {
#pragma unroll
      for (int j = 0; j < 4; ++j) turned[lc + j][lr / 4] = codes4(f[0][j], f[1][j], f[2][j], f[3][j], cinv[lc + j]);
    }
  }
  if (!qt) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t l = threadIdx.x / 16 + 32 * k, w = threadIdx.x % 16;
    if (c0 + l < cols && r0 + 4 * w < padded(rows)) *reinterpret_cast<uint32_t*>(qt + (uint64_t)(c0 + l) * ldqt + r0 + 4 * w) = turned[l][w];
  }
}

// ---- the product's epilogue ----

__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store1(__half* p, float v) { *p = __float2half_rn(v); }

template <class T>
__device__ __forceinline__ void pack4f(uint32_t* w, float a, float b, float c, float d) {
  if constexpr (sizeof(T) == 4) {
    w[0] = __float_as_uint(a), w[1] = __float_as_uint(b), w[2] = __float_as_uint(c), w[3] = __float_as_uint(d);
  } else if constexpr (std::is_same<T, __half>::value) {
    const __half2 x = __floats2half2_rn(a, b), y = __floats2half2_rn(c, d);
    w[0] = *reinterpret_cast<const uint32_t*>(&x), w[1] = *reinterpret_cast<const uint32_t*>(&y);
  } else {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b), y = __floats2bfloat162_rn(c, d);
    w[0] = *reinterpret_cast<const uint32_t*>(&x), w[1] = *reinterpret_cast<const uint32_t*>(&y);
  }
}

// Rows of out start on 32-byte boundaries, sb and bias on 16.
template <class T>
struct EpiScale {
  static constexpr int kIn = 0, kOut = 0;
  struct Pre {
    float s;
  };
  const float *sa, *sb, *bias;
  T* out;
  uint64_t ld;
  uint32_t m, n;
  __device__ __forceinline__ Pre load(uint32_t row, uint32_t, uint32_t) const { return {row < m ? ld_plain(sa + row) : 0.f}; }
  __device__ __forceinline__ void apply(const Pre& p, const uint32_t (&acc)[32], uint32_t row, uint32_t col0, uint32_t) const {
    if (row >= m) return;
    T* o = out + row * ld + col0;
    if (col0 + 32 <= n) {
      uint32_t piece[sizeof(T)][8];      // all of them before the first store: loads are not moved ahead of stores
#pragma unroll
      for (int i = 0; i < 32; i += 4) {
        const float4 s = ld_plain(reinterpret_cast<const float4*>(sb + col0 + i));
        float4 c = make_float4(0.f, 0.f, 0.f, 0.f);
        if (bias) c = ld_plain(reinterpret_cast<const float4*>(bias + col0 + i));
        const float v0 = __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[i], p.s), s.x), c.x);
        const float v1 = __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[i + 1], p.s), s.y), c.y);
        const float v2 = __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[i + 2], p.s), s.z), c.z);
        const float v3 = __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[i + 3], p.s), s.w), c.w);
        pack4f<T>(&piece[i * sizeof(T) / 32][i * sizeof(T) / 4 % 8], v0, v1, v2, v3);
      }
#pragma unroll
      for (int i = 0; i < (int)sizeof(T); ++i) st_b32(o + 32 / sizeof(T) * i, piece[i]);
    } else {
      float s[32], c[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        s[j] = col0 + j < n ? ld_plain(sb + col0 + j) : 0.f;
        c[j] = bias && col0 + j < n ? ld_plain(bias + col0 + j) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (col0 + j < n) store1(o + j, __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[j], p.s), s[j]), c[j]));
    }
  }
};

// The same with the operands' places exchanged: rows of the product are output channels, its columns tokens.  Lanes hold
// consecutive channels, so a token's outputs leave as 64 or 128 consecutive bytes.
template <class T>
struct EpiScaleTurned {
  static constexpr int kIn = 0, kOut = 0;
  struct Pre {
    float s, c, token;             // of this lane's channel, and the scale of token col0 + lane
  };
  const float *sa, *sb, *bias;   // of tokens, of channels
  T* out;
  uint64_t ld;
  uint32_t m, n;                 // channels, tokens
  __device__ __forceinline__ Pre load(uint32_t row, uint32_t col0, uint32_t) const {
    const uint32_t token = col0 + (row & 31);
    return {row < m ? ld_plain(sb + row) : 0.f, row < m && bias ? ld_plain(bias + row) : 0.f, token < n ? ld_plain(sa + token) : 0.f};
  }
  __device__ __forceinline__ void apply(const Pre& p, const uint32_t (&acc)[32], uint32_t row, uint32_t col0, uint32_t) const {
    T* o = out + col0 * ld + row;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const float s = __shfl_sync(0xFFFFFFFFu, p.token, j);
      if (row < m && col0 + j < n) store1(o + j * ld, __fadd_rn(__fmul_rn(__fmul_rn((float)(int)acc[j], s), p.s), p.c));
    }
  }
};

// An empty sum (K = 0): the bias alone.
template <class T>
__global__ void __launch_bounds__(kThreads) k_i8_empty(T* out, uint64_t ld, uint32_t n, const float* bias) {
  pdl_prologue();
  for (uint32_t c = threadIdx.x; c < n; c += kThreads) store1(out + blockIdx.x * ld + c, bias ? bias[c] : 0.f);
}

// ---- few tokens ----
// The weights' bytes are all that counts.  A CTA takes 16 or 32 rows of W; each of its eight warps has an eighth of K, which it
// reads in chunks of 64 codes a row, four chunks ahead, straight into the registers of m16n8k32 instructions (tokens are the 8
// columns; the warp instruction is enough, the loop waits for memory).  A sum of whole numbers may be taken in any order, so
// k is dealt to the instructions' places as it arrives: lane t of a group of four loads 16 consecutive codes of its rows and
// tokens and feeds them as two instructions' worth.  The warps' sums meet in shared memory.
//
// Short inputs are quantised within, by every CTA for itself, under the first loads of W (x stays in L2): a decode step is then
// one launch, which spares the host more than it costs the device (16 tokens through 4096 x 4096: 9 us a call against 15).
// Above kFewCodes codes of W a launch of TMA-fed tiles is faster than this one.
constexpr uint32_t kFewFusedEntries = 16384, kFewFusedMost = 36864;   // entries of x up to which it is quantised within: by any
                                                                      // number of CTAs, by as many as run at once
constexpr uint32_t kFewMost = 16;              // tokens
constexpr uint64_t kFewCodes = 48u << 20;
constexpr size_t kFewSmem = 72 * 1024;         // codes of x in shared memory: 16 tokens in pitches of up to 64 bytes more than K

struct FewParams {
  const void* x;          // tokens: values of type T, or codes
  uint64_t ldx;
  const float* sx;        // scales of the tokens (codes only)
  const int8_t* w;
  uint64_t ldw;
  const float *sw, *bias;
  void* out;
  uint64_t ldo;
  uint32_t m, n, k;
  int vec;                // rows of x start on 16-byte boundaries
};

// 16 codes from k0 on; behind the end of a row nothing is read and zeros stand.  (The end is rare: kept small, since the
// loops' length in instructions counts where a warp lives for a few microseconds.)
__device__ __forceinline__ uint4 load_codes16(const int8_t* row, uint32_t k0, uint32_t k) {
  if (k0 + 16 <= k) return ld_plain(reinterpret_cast<const uint4*>(row + k0));
  unsigned long long v[2] = {0, 0};
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll 1
    for (uint32_t i = k0 + 8 * h; i < k && i < k0 + 8 * h + 8; ++i) v[h] |= (unsigned long long)(uint8_t)row[i] << (8 * (i & 7));
  return make_uint4((uint32_t)v[0], (uint32_t)(v[0] >> 32), (uint32_t)v[1], (uint32_t)(v[1] >> 32));
}

__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 values of one token from k0 on, as codes.
template <class T>
__device__ __forceinline__ uint4 encode16(const T* row, uint32_t k0, uint32_t k, float inv, int vec) {
  if (vec && k0 + 16 <= k) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 16 / Vec<T>::kN; ++i) {
      Vec<T> v;
      v.raw = ld_plain(reinterpret_cast<const uint4*>(row + k0) + i);
#pragma unroll
      for (int j = 0; j < Vec<T>::kN / 4; ++j)
        w[i * (Vec<T>::kN / 4) + j] =
            codes4(v.at(4 * j), v.at(4 * j + 1), v.at(4 * j + 2), v.at(4 * j + 3), inv);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  unsigned long long v[2] = {0, 0};
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll 1
    for (uint32_t i = k0 + 8 * h; i < k && i < k0 + 8 * h + 8; ++i)
      v[h] |= (unsigned long long)(inv != 0.f ? code_of(to_f32(row[i]), inv) & 0xFFu : 0u) << (8 * (i & 7));
  return make_uint4((uint32_t)v[0], (uint32_t)(v[0] >> 32), (uint32_t)v[1], (uint32_t)(v[1] >> 32));
}

// Bytes between tokens in shared memory: whole chunks, and an odd number of 64 bytes, which spreads a quarter warp's 16-byte
// reads (two tokens, 64 bytes of each) over all banks.
__host__ __device__ inline uint32_t few_pitch(uint32_t k) {
  const uint32_t c = (k + 63) / 64;
  return 64 * (c | 1);
}

// X: type of x (int8_t: codes), O: type of out, NT: groups of 8 tokens, RB: blocks of 16 rows of W.
template <class X, class O, int NT, int RB>
__global__ void __launch_bounds__(256, 2) k_i8_few(const FewParams p) {
  constexpr bool kCodes = sizeof(X) == 1;
  constexpr int kAhead = 4;
  extern __shared__ __align__(16) uint8_t xs[];     // the codes of tokens that are quantised here
  __shared__ int part[8][RB * 16][NT * 8 + 1];
  __shared__ uint32_t tops[NT][8];
  __shared__ float scale[NT * 8], inverse[NT * 8];
  pdl_prologue();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t row0 = blockIdx.x * (16 * RB);
  const uint32_t chunks = p.k / 64, per = (chunks + 7) / 8, pitch = few_pitch(p.k);
  const uint32_t first = warp * per, end = min(first + per, chunks);
  const int8_t *wrow[2 * RB], *xrow[NT];            // rows and tokens past the end: one that is there, not stored
#pragma unroll
  for (int i = 0; i < 2 * RB; ++i) wrow[i] = p.w + (uint64_t)min(row0 + g + 8 * i, p.n - 1) * p.ldw;
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const uint32_t token = min(8u * j + g, p.m - 1);
    xrow[j] = kCodes ? static_cast<const int8_t*>(p.x) + token * p.ldx : reinterpret_cast<const int8_t*>(xs) + token * pitch;
  }
  // whole chunks in a loop without a branch but its own; the rest of K, if any, is the last warp's
  uint4 w[kAhead][2 * RB], xc[kAhead][NT];
  auto fetch = [&](uint32_t c, uint4 (&to)[2 * RB], uint4 (&xt)[NT]) {
    if (c >= end) return;
    const uint32_t k0 = c * 64 + t * 16;
#pragma unroll
    for (int i = 0; i < 2 * RB; ++i) to[i] = ld_plain(reinterpret_cast<const uint4*>(wrow[i] + k0));
    if constexpr (kCodes) {
#pragma unroll
      for (int j = 0; j < NT; ++j) xt[j] = ld_plain(reinterpret_cast<const uint4*>(xrow[j] + k0));
    }
  };
#pragma unroll
  for (int a = 0; a < kAhead; ++a) fetch(first + a, w[a], xc[a]);

  if constexpr (!kCodes) {
    // scales: 8 / 2^ceil(log2 m) warps to a token, at least one
    const int shift = p.m <= 1 ? 3 : p.m <= 2 ? 2 : p.m <= 4 ? 1 : 0;
    const uint32_t share = warp & ((1 << shift) - 1), lanes = 32u << shift;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const uint32_t token = 8 * j + (warp >> shift);
      uint32_t top = 0;
      if (token < p.m) {
        const X* row = static_cast<const X*>(p.x) + token * p.ldx;
        const uint32_t at = share * 32 + lane;
        constexpr int N = Vec<X>::kN;
        const uint32_t nv = p.vec ? p.k / N : 0;
#pragma unroll 4
        for (uint32_t v = at; v < nv; v += lanes) {
          Vec<X> r;
          r.raw = ld_plain(reinterpret_cast<const uint4*>(row) + v);
#pragma unroll
          for (int i = 0; i < N; ++i) top = max(top, mag_bits(r.at(i)));
        }
#pragma unroll 1
        for (uint32_t k = nv * N + at; k < p.k; k += lanes) top = max(top, mag_bits(to_f32(row[k])));
      }
      top = __reduce_max_sync(0xFFFFFFFFu, top);
      if (lane == 0) tops[j][warp] = top;
    }
    __syncthreads();
    if (threadIdx.x < 8 * NT) {
      const uint32_t tok = threadIdx.x % 8, j = threadIdx.x / 8;
      uint32_t m = 0;
      for (uint32_t i = 0; i < (1u << shift); ++i)
        if ((tok << shift) + i < 8) m = max(m, tops[j][(tok << shift) + i]);
      float s, v;
      scale_of(m, s, v);
      scale[threadIdx.x] = s;
      inverse[threadIdx.x] = v;
    }
    __syncthreads();
    const uint32_t pieces = (p.k + 15) / 16;
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < p.m * pieces; i += 256) {
      const uint32_t tok = i / pieces, k0 = (i - tok * pieces) * 16;
      *reinterpret_cast<uint4*>(xs + tok * pitch + k0) =
          encode16(static_cast<const X*>(p.x) + tok * p.ldx, k0, p.k, inverse[tok], p.vec);
    }
    __syncthreads();
  } else {
    if (threadIdx.x < NT * 8) scale[threadIdx.x] = threadIdx.x < p.m ? p.sx[threadIdx.x] : 0.f;
  }

  int acc[RB][NT][4];
#pragma unroll
  for (int r = 0; r < RB; ++r)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[r][j][i] = 0;
  auto multiply = [&](const uint4 (&wc)[2 * RB], const uint4 (&x)[NT]) {
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const uint4 lo = wc[2 * r], hi = wc[2 * r + 1];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        mma_s8(acc[r][j], lo.x, hi.x, lo.y, hi.y, x[j].x, x[j].y);
        mma_s8(acc[r][j], lo.z, hi.z, lo.w, hi.w, x[j].z, x[j].w);
      }
    }
  };
  for (uint32_t c0 = first; c0 < end; c0 += kAhead) {
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const uint32_t c = c0 + a;
      if (c >= end) break;
      if constexpr (!kCodes) {
#pragma unroll
        for (int j = 0; j < NT; ++j) xc[a][j] = *reinterpret_cast<const uint4*>(xrow[j] + c * 64 + t * 16);
      }
      multiply(w[a], xc[a]);
      fetch(c + kAhead, w[a], xc[a]);
    }
  }
  if (warp == 7 && (p.k & 63)) {
    const uint32_t k0 = chunks * 64 + t * 16;
    uint4 we[2 * RB], xe[NT];
#pragma unroll
    for (int i = 0; i < 2 * RB; ++i) we[i] = load_codes16(wrow[i], k0, p.k);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      if constexpr (kCodes)
        xe[j] = load_codes16(xrow[j], k0, p.k);
      else
        xe[j] = k0 < p.k ? *reinterpret_cast<const uint4*>(xrow[j] + k0) : make_uint4(0, 0, 0, 0);
    }
    multiply(we, xe);
  }
#pragma unroll
  for (int r = 0; r < RB; ++r)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[warp][16 * r + g + 8 * (i >> 1)][8 * j + 2 * t + (i & 1)] = acc[r][j][i];
  __syncthreads();
  for (uint32_t o = threadIdx.x; o < RB * 16 * p.m; o += 256) {
    const uint32_t token = o / (RB * 16), r = o % (RB * 16), row = row0 + r;
    int s = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) s += part[q][r][token];
    if (row < p.n)
      store1(static_cast<O*>(p.out) + token * p.ldo + row,
             __fadd_rn(__fmul_rn(__fmul_rn((float)s, scale[token]), ld_plain(p.sw + row)), p.bias ? ld_plain(p.bias + row) : 0.f));
  }
}

template <class X, class O, int NT>
cudaError_t launch_few(const FewParams& p, cudaStream_t st) {
  // 32 rows a CTA halve what the tokens' codes cost; where that leaves SMs without a CTA, 16
  const size_t smem = sizeof(X) > 1 ? (size_t)p.m * few_pitch(p.k) : 0;
  auto go = [&](auto kernel, uint32_t rows) {
    launch_pdl_dyn(kernel, dim3((p.n + rows - 1) / rows), dim3(256), smem, st, p);
    count_launches(1);
    return cudaGetLastError();
  };
  if ((p.n + 31) / 32 >= 2 * (uint32_t)sm_count()) {
    if (smem) allow_smem_for<k_i8_few<X, O, NT, 2>>(kFewSmem);
    return go(k_i8_few<X, O, NT, 2>, 32);
  }
  if (smem) allow_smem_for<k_i8_few<X, O, NT, 1>>(kFewSmem);
  return go(k_i8_few<X, O, NT, 1>, 16);
}
template <class X, int NT>
cudaError_t launch_few_fused(const FewParams& p, int out_dtype, cudaStream_t st) {
  return out_dtype == DS_F32    ? launch_few<X, float, NT>(p, st)
         : out_dtype == DS_BF16 ? launch_few<X, __nv_bfloat16, NT>(p, st)
                                : launch_few<X, __half, NT>(p, st);
}
inline bool few_fused(uint64_t rows, uint64_t n, uint64_t k) {
  if (rows > kFewMost || n * k > kFewCodes) return false;
  return rows * k <= kFewFusedEntries || (rows * k <= kFewFusedMost && (n + 15) / 16 <= 2 * (uint64_t)sm_count());
}

inline uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }
inline bool aligned(const void* p, uint64_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline uint32_t size_of(int dtype) { return dtype == DS_F32 ? 4 : 2; }
inline bool dtype_ok(int t) { return t == DS_F32 || t == DS_BF16 || t == DS_F16; }
constexpr uint64_t kMaxLen = 1ull << 30;
constexpr uint32_t kTurnedMost = 64;

// CTAs that share a tile's K, for few tokens: as many as run at once with at least four steps each.
inline uint32_t few_parts(uint32_t tiles, uint32_t k) {
  uint32_t p = 1;
  while (p < 8 && tiles <= (uint32_t)cluster_count(2 * p) && (k + 127) / 128 >= 8 * p) p *= 2;
  return p;
}

template <class T>
cudaError_t product(const int8_t* a, uint64_t lda, const float* sa, const int8_t* b, uint64_t ldb, const float* sb, const float* bias,
                    uint32_t m, uint32_t n, uint32_t k, T* out, uint64_t ldo, uint32_t* dev_status, cudaStream_t st) {
  if (k == 0) {
    launch_pdl(k_i8_empty<T>, dim3(m), dim3(kThreads), st, out, ldo, n, bias);
    count_launches(1);
    return cudaGetLastError();
  }
  if (m <= kFewMost && (uint64_t)n * k <= kFewCodes) {
    const FewParams p{a, lda, sa, b, ldb, sb, bias, out, ldo, m, n, k, 1};
    return m <= 8 ? launch_few<int8_t, T, 1>(p, st) : launch_few<int8_t, T, 2>(p, st);
  }
  // Turned: tiles of 128 output channels by so many tokens.  For few tokens, so that shared memory fills with weights and not
  // with rows that are not there; and where rows of out are on no boundary, since lanes then hold consecutive entries.
  const bool vec = aligned(out, 32) && ldo * sizeof(T) % 32 == 0 && aligned(sb, 16) && (!bias || aligned(bias, 16));
  if (m <= kTurnedMost || !vec) {
    const MmaShape s{n, m, k, 1, 1, 0, 0, dev_status};
    const EpiScaleTurned<T> epi{sa, sb, bias, out, ldo, n, m};
    const bool narrow = m <= 32;
    MmaPlan plan = plan_mma(s);
    if (narrow) {
      plan.pair = false;
      plan.bn = 32;
      const TileWalk w(s, 32);
      plan.parts = few_parts(w.total, k);
    }
    CUtensorMap mw, mx;
    cudaError_t e = make_tensor_map(&mw, kMmaI8, b, k, n, 1, ldb, ldb * n, 128, kMmaRows);
    if (e == cudaSuccess) e = make_tensor_map(&mx, kMmaI8, a, k, m, 1, lda, lda * m, 128, plan.box_rows());
    if (e != cudaSuccess) return e;
    if (!narrow) return launch_mma<kMmaI8, kAlong, kAlong>(plan, mw, mx, mx, s, epi, st);
    return plan.parts > 1 ? launch_mma_split<kMmaI8, 32, kAlong, kAlong>(plan.parts, mw, mx, mx, s, epi, st)
                          : launch_mma_bn<kMmaI8, 32, kAlong, kAlong>(mw, mx, mx, s, epi, st);
  }
  const MmaShape s{m, n, k, 1, 1, 0, 0, dev_status};
  const EpiScale<T> epi{sa, sb, bias, out, ldo, m, n};
  const MmaPlan plan = plan_mma(s);
  CUtensorMap ma, mb;
  cudaError_t e = make_tensor_map(&ma, kMmaI8, a, k, m, 1, lda, lda * m, 128, kMmaRows);
  if (e == cudaSuccess) e = make_tensor_map(&mb, kMmaI8, b, k, n, 1, ldb, ldb * n, 128, plan.box_rows());
  if (e != cudaSuccess) return e;
  return launch_mma<kMmaI8, kAlong, kAlong>(plan, ma, mb, mb, s, epi, st);
}

template <class T>
cudaError_t quantize(const T* x, uint32_t rows, uint32_t cols, uint64_t ld, int8_t* q, uint64_t ldq, float* scale, int8_t* qt, uint64_t ldqt,
                     float* scale_t, float* col_sum, uint8_t* ws, cudaStream_t st) {
  const bool vec = aligned(x, 16) && ld * sizeof(T) % 16 == 0;
  if (!qt && !col_sum) {
    const uint32_t nv = cols / Vec<T>::kN;
    if (vec && cols % Vec<T>::kN == 0 && nv <= 256 * kKeep) {
      // With rows enough to fill the device, as many vectors a thread as it can keep (8192 rows of 16 KB: 46 us with four, 40 with
      // eight); with few rows, two: the row's latency is what counts.
      const uint32_t each = rows >= 8 * (uint32_t)sm_count() ? kKeep : 2;
      const uint32_t want = (uint32_t)round_up((nv + each - 1) / each, 32), bs = want < 32 ? 32 : want > 256 ? 256 : want;
      launch_pdl(k_i8_rows<T, true>, dim3(rows), dim3(bs), st, x, ld, cols, q, ldq, scale);
    } else {
      launch_pdl(k_i8_rows<T, false>, dim3(rows), dim3(256), st, x, ld, cols, q, ldq, scale);
    }
    count_launches(1);
    return cudaGetLastError();
  }
  // One launch where a CTA's reading stays under 200 KB and all CTAs' under 64 MB (512 x 768 in bf16, 164 KB: 7.5 us; 768 x 768
  // floats, 393 KB, would be 10 against 8); rows of whole vectors only.
  const uint64_t reads = ((uint64_t)rows + cols) * 64 * sizeof(T), ctas = (uint64_t)((rows + 63) / 64) * ((cols + 63) / 64);
  if (vec && cols % Vec<T>::kN == 0 && reads <= 200 * 1024 && reads * ctas <= (64u << 20)) {
    launch_pdl(k_i8_small<T>, dim3((cols + 63) / 64, (rows + 63) / 64), dim3(512), st, x, ld, rows, cols, q, ldq, scale, qt, ldqt, scale_t, col_sum);
    count_launches(1);
    return cudaGetLastError();
  }
  uint32_t* row_top = reinterpret_cast<uint32_t*>(ws);
  uint32_t* col_top = row_top + round_up(rows, 64);
  float* sums = col_sum ? reinterpret_cast<float*>(col_top + round_up(cols, 64)) : nullptr;
  cudaError_t e = cudaMemsetAsync(ws, 0, 4 * (round_up(rows, 64) + round_up(cols, 64)), st);
  if (e != cudaSuccess) return e;
  const dim3 g1((cols + 32 * Vec<T>::kN - 1) / (32 * Vec<T>::kN), (rows + kAmaxRows - 1) / kAmaxRows), g2((cols + 127) / 128, (rows + 127) / 128);
  uint32_t *rt = q ? row_top : nullptr, *ct = qt ? col_top : nullptr;
  auto amax = [&](auto kernel) { launch_pdl(kernel, g1, dim3(256), st, x, ld, rows, cols, rt, ct, sums); };
  if (sums)
    vec ? amax(k_i8_amax<T, true, true>) : amax(k_i8_amax<T, false, true>);
  else
    vec ? amax(k_i8_amax<T, true, false>) : amax(k_i8_amax<T, false, false>);
  auto codes = [&](auto kernel, dim3 grid) {
    launch_pdl(kernel, grid, dim3(256), st, x, ld, rows, cols, (const uint32_t*)rt, (const uint32_t*)ct, (const float*)sums, q, ldq, scale, qt, ldqt,
               scale_t, col_sum);
  };
  vec ? codes(k_i8_codes<T>, g2) : codes(k_i8_codes_odd<T>, dim3((cols + 63) / 64, (rows + 63) / 64));
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

uint64_t ds_i8_linear_workspace(uint64_t rows, uint64_t k, uint64_t n) {
  return few_fused(rows, n, k) ? 0 : rows * round_up(k, 16) + 4 * round_up(rows, 64);
}

int ds_i8_linear(const void* x, int dtype, uint64_t rows, uint64_t k, uint64_t ldx, const int8_t* w, uint64_t ldw, const float* sw,
                 const float* bias, uint64_t n, void* out, int out_dtype, uint64_t ldo, void* workspace, size_t workspace_bytes,
                 uint32_t* dev_status, void* cuda_stream) {
  if (rows > kMaxLen || k > DS_I8_MAX_K) return rows > kMaxLen ? DS_ERR_INVALID_ARG : DS_ERR_UNSUPPORTED;
  if (rows == 0 || n == 0) return dtype_ok(dtype) && dtype_ok(out_dtype) ? DS_OK : DS_ERR_INVALID_ARG;
  if (k == 0)
    return dtype_ok(dtype) ? ds_i8_matmul(nullptr, 0, sw, nullptr, 0, sw, bias, rows, n, 0, out, out_dtype, ldo, dev_status, cuda_stream)
                           : DS_ERR_INVALID_ARG;
  // all refusals come before the first launch
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype) || n > kMaxLen || ldx < k || ldo < n || !x || !sw || !out) return DS_ERR_INVALID_ARG;
  int rc = check_codes(w, ldw, k);
  if (rc != DS_OK) return rc;
  if (!aligned(x, size_of(dtype)) || !aligned(sw, 4) || !aligned(bias, 4) || !aligned(out, size_of(out_dtype)) || !aligned(dev_status, 4))
    return DS_ERR_ALIGN;
  if (few_fused(rows, n, k)) {
    const FewParams p{x, ldx, nullptr, w, ldw, sw, bias, out, ldo, (uint32_t)rows, (uint32_t)n, (uint32_t)k,
                      aligned(x, 16) && ldx * size_of(dtype) % 16 == 0};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    auto go = [&](auto tokens) {
      constexpr int kGroups = decltype(tokens)::value;
      return dtype == DS_F32    ? launch_few_fused<float, kGroups>(p, out_dtype, st)
             : dtype == DS_BF16 ? launch_few_fused<__nv_bfloat16, kGroups>(p, out_dtype, st)
                                : launch_few_fused<__half, kGroups>(p, out_dtype, st);
    };
    const cudaError_t e = rows <= 8 ? go(std::integral_constant<int, 1>()) : go(std::integral_constant<int, 2>());
    return e == cudaSuccess ? DS_OK : cuda_fail(e, "8-bit product");
  }
  if (!workspace) return DS_ERR_INVALID_ARG;
  if (!aligned(workspace, 16)) return DS_ERR_ALIGN;
  if (workspace_bytes < ds_i8_linear_workspace(rows, k, n)) return DS_ERR_BUFFER_TOO_SMALL;
  const uint64_t ldq = round_up(k, 16);
  float* s = static_cast<float*>(workspace);
  int8_t* q = static_cast<int8_t*>(workspace) + 4 * round_up(rows, 64);
  rc = ds_i8_quantize(x, dtype, rows, k, ldx, q, ldq, s, nullptr, 0, nullptr, nullptr, nullptr, 0, cuda_stream);
  if (rc != DS_OK) return rc;
  return ds_i8_matmul(q, ldq, s, w, ldw, sw, bias, rows, n, k, out, out_dtype, ldo, dev_status, cuda_stream);
}

}  // extern "C"
