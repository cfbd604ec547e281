// Orthogonalised update: momentum, then Newton-Schulz products that bring the singular values of the update near one.
//
//   buf = mu buf + g;   u = g + mu buf (Nesterov) or buf;   X = u / (||u||_F + eps)
//   `steps` times:  A = X X^T,  B = b A + c A A,  X = a X + B X         (over the shorter side: X is [m, n], m <= n)
//   out = X;  optionally x = (1 - gamma decay) x - gamma scale X
//
// Numbers.  Products run on 16-bit floats with 11 bits of significand (same rate as the 8-bit-significand format, whose error
// would be eight times as large) and add up in 32 bits.  The entries of X, A and B are bounded (|X| <= 1.3, |A| <= 1.5, |B| <= 8 for
// the usual coefficients), so they are held times 2^10, which keeps small entries out of the subnormals; entries from 64 on are inf.  Three things
// would otherwise lose bits that later steps multiply by a = 3.4 each:
//  - X is carried in two halves (hi + lo, 22 bits), of which aX takes both.  With hi alone, updates whose energy sits in few
//    directions came out 0.6 % to 2 % off.
//  - The diagonals of A and B, which hold most of their size when rows are nearly orthogonal, stay in 32 bits: A = D + O and
//    B = E + F with F off-diagonal:  F = b O + c (O O)_off + c (d_i + d_j) O_ij,  E_ii = b d_i + c d_i^2 + c (O O)_ii,
//    X = a X + E X + F X.  Row scalings cost nothing in the epilogues.  (0.1 % to 0.2 % off without it on such inputs.)
//  - E and F have to take the same X while errors can still grow.  B maps the left null space of X to zero, but only as E + F: with E (hi + lo)
//    + F hi something of the size of lo stays in directions where X is zero, and each later step multiplies it by a.  (In
//    all five steps: updates of 2 live rows of rank 1 were 4 % off, the gradient of one sample 4 %.)  So the first two steps take E hi + F hi,
//    which leaves out B lo where X is not zero, and that does not grow; the last two take E (hi + lo) + F hi, whose errors have one step left
//    to grow in; those between take both halves in both terms, F lo by a second pass over K.
// What is left is 0.02 % to 0.1 % of ordinary updates; at most 0.7 % where few rows are not zero or all entries are alike, so that the
// roundings of O and F are alike too (the worst of 1500 such inputs, and of 30000 under the same roundings emulated; median 0.1 %).
#include <cmath>
#include <cstring>
#include <new>

#include "dsq_mma.cuh"
#include "dsq_orth.cuh"

using namespace dsq;

namespace {

// ---- momentum and norm: one pass over g and buf ----
// Bound by memory: 4 (or 2) + 4 bytes read and 4 written an entry.  Squares add up in 64 bits, each thread over its own
// entries, then in a fixed order; the next kernel adds the CTAs' sums.  (A ticket for the last CTA to add them held every CTA's
// place for the two microseconds of its atomic: 19 us instead of 15 for three 512 x 4608.)
constexpr int kNormCtas = 512;

template <class T>
__global__ void __launch_bounds__(kThreads) k_orth_momentum(const Momentum mo, uint64_t count, int vec, double* partial) {
  pdl_prologue();
  const uint64_t off = (uint64_t)blockIdx.y * mo.stride;
  const T* g = static_cast<const T*>(mo.g) + off;
  float* buf = mo.buf ? mo.buf + off : nullptr;
  double sum = 0;
  const uint64_t first = (uint64_t)blockIdx.x * kThreads + threadIdx.x, step = (uint64_t)gridDim.x * kThreads;
  if (vec) {
    // four vectors of four at once: their loads go ahead of the stores that might alias them
    for (uint64_t i0 = first * 4; i0 < count; i0 += step * 16) {
      float gv[4][4], bv[4][4], part = 0.f, lead = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint64_t i = i0 + q * step * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) gv[q][j] = bv[q][j] = 0.f;
        if (i < count) {
          load4(gv[q], g + i);
          if (buf) load4(bv[q], buf + i);
        }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint64_t i = i0 + q * step * 4;
        float u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u[j] = gv[q][j];
          if (buf) bv[q][j] = mo.update(gv[q][j], bv[q][j]), u[j] = mo.direction(gv[q][j], bv[q][j]);
        }
        if (buf && i < count) *reinterpret_cast<float4*>(buf + i) = make_float4(bv[q][0], bv[q][1], bv[q][2], bv[q][3]);
#pragma unroll
        for (int j = 0; j < 4; ++j) lead = fmaxf(lead, fabsf(u[j])), part = fmaf(u[j], u[j], part);
      }
      // Sixteen squares in 32 bits, then on in 64; where they might leave the range of 32 bits, in 64 throughout.
      if (lead < 1e18f && lead > 1e-18f) {
        sum += (double)part;
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float u = buf ? mo.direction(gv[q][j], bv[q][j]) : gv[q][j];
            sum += (double)u * (double)u;
          }
      }
    }
  } else {
    for (uint64_t i = first; i < count; i += step) {
      const float gv = to_f32(g[i]);
      float u = gv;
      if (buf) {
        const float bv = mo.update(gv, buf[i]);
        buf[i] = bv;
        u = mo.direction(gv, bv);
      }
      sum += (double)u * (double)u;
    }
  }
  __shared__ double warp_sum[kThreads / 32];
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0;
    for (int i = 0; i < kThreads / 32; ++i) s += warp_sum[i];
    partial[(uint64_t)blockIdx.y * kNormCtas + blockIdx.x] = s;
  }
}

// ---- X = u / norm in two halves, transposed where the matrix is taller than wide ----
// A CTA takes a tile of 64 x 64 and adds the norm up for itself; the tile goes through shared memory when it is transposed.
struct Halves {
  __half *hi, *lo;
  uint32_t ld;       // elements between rows (a multiple of 16)
  uint64_t stride;   // elements between matrices
};

template <class T, bool TALL>
__global__ void __launch_bounds__(kThreads) k_orth_split(const Momentum mo, uint32_t rows, uint32_t cols, int vec, const double* partial,
                                                         uint32_t parts, float eps, const Halves x) {
  pdl_prologue();
  __shared__ float tile[TALL ? 64 : 1][TALL ? 65 : 1];
  __shared__ double warp_sum[kThreads / 32];
  // from the end: what the pass before touched last is still in L2
  const uint32_t b = gridDim.z - 1 - blockIdx.z, r0 = (gridDim.y - 1 - blockIdx.y) * 64, c0 = (gridDim.x - 1 - blockIdx.x) * 64;
  const uint64_t off = (uint64_t)b * mo.stride;
  const T* g = static_cast<const T*>(mo.g) + off;
  const float* buf = mo.buf ? mo.buf + off : nullptr;
  auto put = [&](uint32_t r, uint32_t c, const float (&v)[4]) {   // c a multiple of 4 below ld
    __half h[4], l[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = __float2half_rn(v[j]), l[j] = __float2half_rn(v[j] - __half2float(h[j]));
    const uint64_t at = (uint64_t)b * x.stride + (uint64_t)r * x.ld + c;
    *reinterpret_cast<uint2*>(x.hi + at) = *reinterpret_cast<uint2*>(h);
    *reinterpret_cast<uint2*>(x.lo + at) = *reinterpret_cast<uint2*>(l);
  };
  // the norm's parts are asked for before the tile, and added in the same order in every CTA
  static_assert(kNormCtas == 2 * kThreads, "two parts a thread");
  double sum = 0, second = 0;
  if (threadIdx.x < parts) sum = ld_plain(partial + (uint64_t)b * kNormCtas + threadIdx.x);
  if (threadIdx.x + kThreads < parts) second = ld_plain(partial + (uint64_t)b * kNormCtas + threadIdx.x + kThreads);
  float gv[4][4], bv[4][4], v[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lr = threadIdx.x / 16 + 16 * i, lc = threadIdx.x % 16 * 4, r = r0 + lr, c = c0 + lc;
#pragma unroll
    for (int j = 0; j < 4; ++j) gv[i][j] = bv[i][j] = 0.f;
    if (r < rows && c < cols) {
      const uint64_t at = (uint64_t)r * cols + c;
      if (vec) {
        load4(gv[i], g + at);
        if (buf) load4(bv[i], buf + at);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c + j < cols) {
            gv[i][j] = to_f32(g[at + j]);
            if (buf) bv[i][j] = buf[at + j];
          }
      }
    }
  }
  sum += second;
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  sum = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) sum += warp_sum[i];
  const NormFactor f(sum, eps);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lr = threadIdx.x / 16 + 16 * i, lc = threadIdx.x % 16 * 4, r = r0 + lr, c = c0 + lc;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i][j] = f(buf ? mo.direction(gv[i][j], bv[i][j]) : gv[i][j]);
    if constexpr (TALL) {
#pragma unroll
      for (int j = 0; j < 4; ++j) tile[lr][lc + j] = v[i][j];
    } else {
      if (r < rows && c < x.ld) put(r, c, v[i]);
    }
  }
  if constexpr (TALL) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lr = threadIdx.x / 16 + 16 * i, lc = threadIdx.x % 16 * 4, r = c0 + lr, c = r0 + lc;   // of X = u^T
      float t[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) t[j] = tile[lc + j][lr];
      if (r < cols && c < x.ld) put(r, c, t);
    }
  }
}

// ---- epilogues of the three products ----

struct Half32 {   // 32 consecutive entries of a row, two to a word
  uint32_t w[16];
  __device__ __forceinline__ float2 two(int j) const {   // entries 2j and 2j + 1
    return __half22float2(*reinterpret_cast<const __half2*>(w + j));
  }
  __device__ __forceinline__ void set(int j, float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    w[j] = *reinterpret_cast<const uint32_t*>(&h);
  }
  // this lane's row of a block in shared memory
  __device__ __forceinline__ void get(uint32_t block, int lane) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(w[4 * q]), "=r"(w[4 * q + 1]), "=r"(w[4 * q + 2]), "=r"(w[4 * q + 3])
                   : "r"(row_chunk(block, lane, q))
                   : "memory");
  }
  __device__ __forceinline__ void put(uint32_t block, int lane) const {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row_chunk(block, lane, q)), "r"(w[4 * q]), "r"(w[4 * q + 1]), "r"(w[4 * q + 2]),
                   "r"(w[4 * q + 3])
                   : "memory");
  }
};

// A symmetric matrix in 16 bits without its diagonal, which is held apart; its blocks on and above the diagonal.
struct SymOut {
  __half* off;
  float* diag;
  uint32_t m, ld;
  uint64_t stride, diag_stride;
};

struct EpiGram {   // A = X X^T
  static constexpr int kIn = 0, kOut = 1;
  struct Pre {};
  CUtensorMap a_blocks;
  SymOut a;
  __device__ __forceinline__ const CUtensorMap* out(int) const { return &a_blocks; }
  __device__ __forceinline__ Pre load(uint32_t, uint32_t, uint32_t) const { return {}; }
  __device__ __forceinline__ void apply(const Pre&, const uint32_t (&acc)[32], uint32_t row, uint32_t col0, uint32_t b, uint32_t block, int lane) const {
    Half32 v;
    float d = 0.f, s[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      s[j] = __uint_as_float(acc[j]) * kDown;
      if (col0 + j == row) d = s[j], s[j] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) v.set(j, s[2 * j], s[2 * j + 1]);
    if (row >= col0 && row < col0 + 32 && row < a.m) a.diag[b * a.diag_stride + row] = d * kDown;
    v.put(block, lane);
  }
};

struct EpiPoly {   // B = b A + c A A, the accumulator being O O
  static constexpr int kIn = 1, kOut = 1;
  struct Pre {
    float d;
  };
  CUtensorMap a_blocks, b_blocks;
  SymOut a, b;
  float b1, c1;
  __device__ __forceinline__ const CUtensorMap* in(int) const { return &a_blocks; }
  __device__ __forceinline__ const CUtensorMap* out(int) const { return &b_blocks; }
  __device__ __forceinline__ Pre load(uint32_t row, uint32_t, uint32_t z) const { return {row < a.m ? a.diag[z * a.diag_stride + row] : 0.f}; }
  __device__ __forceinline__ void apply(const Pre& p, const uint32_t (&acc)[32], uint32_t row, uint32_t col0, uint32_t z, uint32_t block, int lane) const {
    Half32 v;
    v.get(block, lane);
    const float4* dj = reinterpret_cast<const float4*>(a.diag + z * a.diag_stride + col0);   // padded to a multiple of 32 entries
    float d = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float4 t = ld_plain(dj + q);
      const float2 o0 = v.two(2 * q), o1 = v.two(2 * q + 1);
      const float dd[4] = {t.x, t.y, t.z, t.w}, o[4] = {o0.x, o0.y, o1.x, o1.y};
      float e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = 4 * q + i;
        const float s = __uint_as_float(acc[j]);
        const bool on = col0 + j == row;
        if (on) d = s;
        e[i] = on || col0 + j >= a.m ? 0.f : fmaf(c1, fmaf(s, kDown, (p.d + dd[i]) * o[i]), b1 * o[i]);
      }
      v.set(2 * q, e[0], e[1]);
      v.set(2 * q + 1, e[2], e[3]);
    }
    if (row >= col0 && row < col0 + 32 && row < a.m)
      b.diag[z * a.diag_stride + row] = fmaf(c1, fmaf(d, kDown * kDown, p.d * p.d), b1 * p.d);
    v.put(block, lane);
  }
};

struct EpiX {   // X = (a + E) X + F X
  static constexpr int kIn = 2, kOut = 2;
  struct Pre {
    float e;
  };
  CUtensorMap blocks[2], next[2];   // X and the next X, hi and lo
  const float* diag;                // E
  uint64_t diag_stride;
  uint32_t m, n;
  float a1;
  int e_hi;                         // E multiplies the high half of X alone
  int last;                         // the last step writes:
  OrthOut to;                       //   in the orientation of the gradient
  int tall, vec;
  __device__ __forceinline__ const CUtensorMap* in(int i) const { return blocks + i; }
  __device__ __forceinline__ const CUtensorMap* out(int i) const { return last ? nullptr : next + i; }
  __device__ __forceinline__ Pre load(uint32_t row, uint32_t, uint32_t b) const { return {row < m ? diag[b * diag_stride + row] : 0.f}; }
  __device__ __forceinline__ void apply(const Pre& p, const uint32_t (&acc)[32], uint32_t row, uint32_t col0, uint32_t b, uint32_t block, int lane) const {
    const float f = e_hi ? a1 : a1 + p.e, f_hi = e_hi ? p.e : 0.f;
    float v[32];
    Half32 h, l;
    h.get(block, lane);
    l.get(block + kBlockBytes, lane);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float2 x = h.two(j), y = l.two(j);
      v[2 * j] = fmaf(f, x.x + y.x, fmaf(f_hi, x.x, __uint_as_float(acc[2 * j]) * kDown));
      v[2 * j + 1] = fmaf(f, x.y + y.y, fmaf(f_hi, x.y, __uint_as_float(acc[2 * j + 1]) * kDown));
    }
    if (!last) {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        h.set(j, v[2 * j], v[2 * j + 1]);
        const float2 r = h.two(j);
        l.set(j, v[2 * j] - r.x, v[2 * j + 1] - r.y);
      }
      h.put(block, lane);
      l.put(block + kBlockBytes, lane);
      return;
    }
    if (row >= m) return;
    // The last step leaves the workspace.  Tall matrices come back transposed: lanes then hold consecutive entries.
    const uint64_t step = tall ? m : 1;
    const uint64_t first = tall ? (uint64_t)col0 * m + row : (uint64_t)row * n + col0, each = (uint64_t)m * n;
    const bool whole = vec && !tall && col0 + 32 <= n;
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] *= kDown;
    if (to.out) {
      const uint64_t at = b * each + first;
      if (to.dtype == DS_BF16) {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(to.out) + at;
        if (whole) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t t[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const __nv_bfloat162 h = __floats2bfloat162_rn(v[16 * q + 2 * j], v[16 * q + 2 * j + 1]);
              t[j] = *reinterpret_cast<const uint32_t*>(&h);
            }
            st_b32(o + 16 * q, t);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (col0 + j < n) o[j * step] = __float2bfloat16_rn(v[j]);
        }
      } else {
        float* o = static_cast<float*>(to.out) + at;
        if (whole) {
#pragma unroll
          for (int q = 0; q < 8; ++q) *reinterpret_cast<float4*>(o + 4 * q) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (col0 + j < n) o[j * step] = v[j];
        }
      }
    }
    if (to.x) {
      float* px = to.x + b * to.x_stride + first;
      if (whole) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          float4 t = *reinterpret_cast<float4*>(px + 4 * q);
          t.x = __fsub_rn(__fmul_rn(to.keep, t.x), __fmul_rn(to.rate, v[4 * q]));
          t.y = __fsub_rn(__fmul_rn(to.keep, t.y), __fmul_rn(to.rate, v[4 * q + 1]));
          t.z = __fsub_rn(__fmul_rn(to.keep, t.z), __fmul_rn(to.rate, v[4 * q + 2]));
          t.w = __fsub_rn(__fmul_rn(to.keep, t.w), __fmul_rn(to.rate, v[4 * q + 3]));
          *reinterpret_cast<float4*>(px + 4 * q) = t;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (col0 + j < n) px[j * step] = __fsub_rn(__fmul_rn(to.keep, px[j * step]), __fmul_rn(to.rate, v[j]));
      }
    }
  }
};

inline uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

// Which halves of X step s takes in E X and in F X (file header).
enum HalvesTaken { kEhiFhi, kEbothFboth, kEbothFhi };
inline HalvesTaken halves_of(uint32_t s, uint32_t steps) { return s + 2 >= steps ? kEbothFhi : s < 2 ? kEhiFhi : kEbothFboth; }

bool orth_config_ok(const ds_orth_config* c) {
  if (!c || c->rows < 1 || c->cols < 1 || c->batch < 1 || c->batch > 65535 || c->rows > (1u << 20) || c->cols > (1u << 20)) return false;
  if (c->steps < 1 || c->steps > 32 || (c->flags & ~DS_ORTH_NESTEROV) || c->reserved) return false;
  if (c->stride && c->stride < (uint64_t)c->rows * c->cols) return false;
  for (float v : {c->a, c->b, c->c, c->momentum, c->eps, c->scale})
    if (!std::isfinite(v)) return false;
  return c->eps >= 0.f;
}

}  // namespace

struct ds_orth_ctx {
  ds_orth_config cfg;
  uint32_t m, n, ldx, ldm;
  uint32_t small;                 // CTAs a matrix takes in the form for small matrices, 0: the products below
  uint64_t xs, ms, ds;            // elements between matrices of X, of A and B, of the diagonals
  __half *hi[2], *lo[2];
  SymOut a, b;
  double* partial;
  uint32_t* dev_status;
  bool mapped;                    // the tensor maps below are made (on the first update: the driver makes them)
  MmaPlan p_gram, p_poly, p_x;
  uint32_t half_a, half_b;        // A and B: log2 of the blocks of which half is there
  CUtensorMap x_rows[2], x_cols_gram[2], x_across[2], lo_across[2], a_sym, b_sym;
  CUtensorMap hi_blocks[2], lo_blocks[2], a_blocks, b_blocks;
};

namespace {

// Carves the workspace; returns its size.
uint64_t orth_plan(ds_orth_ctx* h, uint8_t* ws) {
  const ds_orth_config& c = h->cfg;
  h->m = c.rows < c.cols ? c.rows : c.cols;
  h->n = c.rows < c.cols ? c.cols : c.rows;
  h->ldx = (uint32_t)round_up(h->n, 16);
  h->ldm = (uint32_t)round_up(h->m, 16);
  h->xs = (uint64_t)h->m * h->ldx;
  h->ms = (uint64_t)h->m * h->ldm;
  h->ds = round_up(h->m, 32);
  h->small = orth_small_ctas(h->m, h->n, c.batch);
  if (h->small) return 256;   // works in shared memory
  uint64_t pos = 0;
  auto take = [&](uint64_t bytes) {
    uint8_t* p = ws ? ws + pos : nullptr;
    pos += round_up(bytes, 256);
    return p;
  };
  h->partial = reinterpret_cast<double*>(take(8ull * kNormCtas * c.batch));
  for (int i = 0; i < 2; ++i) {
    h->hi[i] = reinterpret_cast<__half*>(take(2 * h->xs * c.batch));
    h->lo[i] = reinterpret_cast<__half*>(take(2 * h->xs * c.batch));
  }
  for (SymOut* s : {&h->a, &h->b}) {
    s->off = reinterpret_cast<__half*>(take(2 * h->ms * c.batch));
    s->diag = reinterpret_cast<float*>(take(4 * h->ds * c.batch));
    s->m = h->m;
    s->ld = h->ldm;
    s->stride = h->ms;
    s->diag_stride = h->ds;
  }
  return pos;
}

cudaError_t orth_maps(ds_orth_ctx* h) {
  const uint32_t batch = h->cfg.batch;
  // from the last product to the first: how a product is taken says how much of its symmetric operand has to be there
  h->p_x = plan_mma({h->m, h->n, h->m, batch, 2, 0, 0, nullptr});
  h->half_b = h->p_x.pair ? 8 : 7;
  h->p_poly = plan_mma({h->m, h->m, h->m, batch, 2, h->half_b, 0, nullptr}, true);
  // (the epilogue of B = b A + c A A reads of A what it writes of B)
  h->half_a = h->half_b == 8 || h->p_poly.pair || h->p_poly.bn > 128 ? 8 : 7;
  h->p_gram = plan_mma({h->m, h->m, h->n, batch, 2, h->half_a, 0, nullptr});
  cudaError_t e = cudaSuccess;
  auto add = [&](CUtensorMap* map, const void* base, uint64_t cols, uint64_t rows, uint64_t ld, uint64_t stride, uint32_t box_rows) {
    if (e == cudaSuccess) e = make_tensor_map(map, kMmaF16, base, cols, rows, batch, ld, stride, 64, box_rows);
  };
  for (int i = 0; i < 2; ++i) {
    add(&h->x_rows[i], h->hi[i], h->n, h->m, h->ldx, h->xs, kMmaRows);
    add(&h->x_cols_gram[i], h->hi[i], h->n, h->m, h->ldx, h->xs, h->p_gram.box_rows());
    add(&h->x_across[i], h->hi[i], h->n, h->m, h->ldx, h->xs, 64);
    add(&h->lo_across[i], h->lo[i], h->n, h->m, h->ldx, h->xs, 64);
  }
  add(&h->a_sym, h->a.off, h->m, h->m, h->ldm, h->ms, 64);
  add(&h->b_sym, h->b.off, h->m, h->m, h->ldm, h->ms, 64);
  auto add_blocks = [&](CUtensorMap* map, const void* base, uint64_t cols, uint64_t ld, uint64_t stride) {
    if (e == cudaSuccess) e = make_tensor_map(map, kMmaF16, base, cols, h->m, batch, ld, stride, 32, 32, true);
  };
  for (int i = 0; i < 2; ++i) {
    add_blocks(&h->hi_blocks[i], h->hi[i], h->n, h->ldx, h->xs);
    add_blocks(&h->lo_blocks[i], h->lo[i], h->n, h->ldx, h->xs);
  }
  add_blocks(&h->a_blocks, h->a.off, h->m, h->ldm, h->ms);
  add_blocks(&h->b_blocks, h->b.off, h->m, h->ldm, h->ms);
  h->mapped = e == cudaSuccess;
  return e;
}

template <class T>
cudaError_t launch_prepare(const ds_orth_ctx* h, const Momentum& mo, int vec, cudaStream_t st) {
  const ds_orth_config& c = h->cfg;
  const uint64_t count = (uint64_t)c.rows * c.cols;
  const uint64_t want = (count + 16ull * kThreads - 1) / (16ull * kThreads);
  const uint64_t fill = (16ull * sm_count() + c.batch - 1) / c.batch, most = fill < kNormCtas ? fill : kNormCtas;   // one wave
  const uint32_t ctas = (uint32_t)(want < most ? want : most);
  launch_pdl(k_orth_momentum<T>, dim3(ctas, c.batch), dim3(kThreads), st, mo, count, vec, h->partial);
  const Halves x{h->hi[0], h->lo[0], h->ldx, h->xs};
  const dim3 grid((c.cols + 63) / 64, (c.rows + 63) / 64, c.batch);
  if (c.rows > c.cols)
    launch_pdl(k_orth_split<T, true>, grid, dim3(kThreads), st, mo, c.rows, c.cols, vec, (const double*)h->partial, ctas, c.eps, x);
  else
    launch_pdl(k_orth_split<T, false>, grid, dim3(kThreads), st, mo, c.rows, c.cols, vec, (const double*)h->partial, ctas, c.eps, x);
  count_launches(2);
  return cudaGetLastError();
}

}  // namespace

extern "C" {

int ds_orth_create(const ds_orth_config* cfg, void* workspace, size_t* workspace_bytes, uint32_t* dev_status, ds_orth_handle* out) {
  if (!orth_config_ok(cfg) || !workspace_bytes) return DS_ERR_INVALID_ARG;
  ds_orth_ctx tmp;
  memset(&tmp, 0, sizeof tmp);
  tmp.cfg = *cfg;
  const uint64_t need = orth_plan(&tmp, static_cast<uint8_t*>(workspace));
  if (!workspace) {
    *workspace_bytes = need;
    return DS_NEED_BUFFERS;
  }
  if (!dev_status || !out) return DS_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) || (reinterpret_cast<uintptr_t>(dev_status) & 3u)) return DS_ERR_ALIGN;
  if (*workspace_bytes < need) return DS_ERR_BUFFER_TOO_SMALL;
  tmp.dev_status = dev_status;
  ds_orth_ctx* h = new (std::nothrow) ds_orth_ctx(tmp);
  if (!h) return DS_ERR_INVALID_ARG;
  *out = h;
  return DS_OK;
}

int ds_orth_update(ds_orth_handle h, const void* g, int g_dtype, float* momentum, void* out, int out_dtype, float* x, float gamma,
                   float decay, void* cuda_stream) {
  if (!h || !g || (!out && !x)) return DS_ERR_INVALID_ARG;
  if (g_dtype != DS_F32 && g_dtype != DS_BF16 && g_dtype != DS_F16) return DS_ERR_INVALID_ARG;
  if (out && out_dtype != DS_F32 && out_dtype != DS_BF16) return DS_ERR_INVALID_ARG;
  if (x && (!std::isfinite(gamma) || !std::isfinite(decay))) return DS_ERR_INVALID_ARG;
  const ds_orth_config& c = h->cfg;
  const uintptr_t gp = reinterpret_cast<uintptr_t>(g), bp = reinterpret_cast<uintptr_t>(momentum), op = reinterpret_cast<uintptr_t>(out),
                  xp = reinterpret_cast<uintptr_t>(x);
  const uint32_t g_size = g_dtype == DS_F32 ? 4 : 2, out_size = out_dtype == DS_F32 ? 4 : 2;
  if ((gp & (g_size - 1)) || ((bp | xp) & 3u) || (out && (op & (out_size - 1)))) return DS_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  Momentum mo;
  mo.g = g;
  mo.buf = momentum;
  mo.stride = c.stride ? c.stride : (uint64_t)c.rows * c.cols;
  mo.mu = c.momentum;
  mo.nesterov = (c.flags & DS_ORTH_NESTEROV) ? 1 : 0;
  const OrthOut where{out, out_dtype, x, mo.stride, 1.f - gamma * decay, gamma * c.scale};
  if (h->small) {
    const cudaError_t e = launch_orth_small(c, h->small, mo, g_dtype, where, st);
    return e == cudaSuccess ? DS_OK : cuda_fail(e, "orthogonalised update");
  }
  if (!h->mapped) {
    const cudaError_t e = orth_maps(h);
    if (e != cudaSuccess) return cuda_fail(e, "tensor maps");
  }
  // four entries at a time where every matrix, and every row of it, starts on a boundary of four
  const int vec = c.cols % 4 == 0 && mo.stride % 4 == 0 && (gp & (4 * g_size - 1)) == 0 && (bp & 15u) == 0;
  cudaError_t e = g_dtype == DS_F32    ? launch_prepare<float>(h, mo, vec, st)
                  : g_dtype == DS_BF16 ? launch_prepare<__nv_bfloat16>(h, mo, vec, st)
                                       : launch_prepare<__half>(h, mo, vec, st);
  const MmaShape gram{h->m, h->m, h->n, c.batch, 2, h->half_a, 0, h->dev_status}, poly{h->m, h->m, h->m, c.batch, 2, h->half_b, h->half_a, h->dev_status};
  MmaShape full{h->m, h->n, h->m, c.batch, 2, 0, h->half_b, h->dev_status};
  int cur = 0;
  for (uint32_t s = 0; s < c.steps && e == cudaSuccess; ++s, cur ^= 1) {
    e = launch_mma<kMmaF16, kAlong, kAlong>(h->p_gram, h->x_rows[cur], h->x_cols_gram[cur], h->x_cols_gram[cur], gram, EpiGram{h->a_blocks, h->a}, st);
    if (e == cudaSuccess)
      e = launch_mma<kMmaF16, kSym, kSym>(h->p_poly, h->a_sym, h->a_sym, h->a_sym, poly, EpiPoly{h->a_blocks, h->b_blocks, h->a, h->b, c.b, c.c}, st);
    EpiX ex;
    memset(&ex, 0, sizeof ex);
    ex.blocks[0] = h->hi_blocks[cur];
    ex.blocks[1] = h->lo_blocks[cur];
    ex.next[0] = h->hi_blocks[cur ^ 1];
    ex.next[1] = h->lo_blocks[cur ^ 1];
    ex.diag = h->b.diag;
    ex.diag_stride = h->ds;
    ex.m = h->m;
    ex.n = h->n;
    ex.a1 = c.a;
    ex.last = s + 1 == c.steps;
    if (ex.last) {
      ex.to = where;
      ex.tall = c.rows > c.cols;
      ex.vec = c.cols % 16 == 0 && (op & 31u) == 0 && (xp & 15u) == 0 && mo.stride % 4 == 0;
    }
    const HalvesTaken taken = halves_of(s, c.steps);
    ex.e_hi = taken == kEhiFhi;
    full.passes = taken == kEbothFboth ? 2 : 1;
    if (e == cudaSuccess) e = launch_mma<kMmaF16, kSym, kAcross>(h->p_x, h->b_sym, h->x_across[cur], h->lo_across[cur], full, ex, st);
  }
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "orthogonalised update");
}

int ds_orth_destroy(ds_orth_handle h) {
  if (!h) return DS_ERR_INVALID_ARG;
  delete h;
  return DS_OK;
}

}  // extern "C"
