// A linear layer in 16-bit floats: its products (dsq_product16.cuh), the form for a few tokens, the gradient through the
// activation, and copies onto 16-byte rows.
#include <atomic>
#include <type_traits>

#include "dsq_product16.cuh"
#include "dsq_rows8.cuh"

using namespace dsq;

namespace {

inline uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }
inline bool aligned(const void* p, uint64_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline bool half_ok(uint64_t t) { return t == DS_BF16 || t == DS_F16; }
inline bool dtype_ok(uint64_t t) { return t == DS_F32 || t == DS_BF16 || t == DS_F16; }
inline uint32_t size_of(uint64_t dtype) { return dtype == DS_F32 ? 4 : 2; }
constexpr uint64_t kMaxLen = 1ull << 30;

// ---- copies onto 16-byte rows ---------------------------------------------------------------------------
// Bound by memory; a lane takes eight entries of a row.  Entries behind a row's end become 0.
template <class T, class O>
__global__ void __launch_bounds__(kThreads) k_f16_pack(const T* x, uint64_t ld, uint32_t rows, uint32_t cols, O* out, uint64_t ldo) {
  pdl_prologue();
  const uint32_t c = (blockIdx.x * blockDim.x + threadIdx.x) * 8;
  const int lane = threadIdx.x & 31;
  if (c - 8 * lane >= ldo) return;
  for (uint32_t r = blockIdx.y * blockDim.y + threadIdx.y; r < rows; r += gridDim.y * blockDim.y) {
    float v[8];
    load_row8<false>(x + r * ld, c, cols, lane, v);
    store_row8<true>(out + r * ldo, c, (uint32_t)ldo, lane, v);
  }
}

template <class T, class O>
cudaError_t pack_as(const void* x, uint64_t rows, uint64_t cols, uint64_t ld, void* out, uint64_t ldo, cudaStream_t st) {
  const uint32_t warps = (uint32_t)((ldo + 255) / 256), tx = 32 * (warps < 8 ? warps : 8), ty = kThreads / tx, gy = (uint32_t)((rows + ty - 1) / ty);
  launch_pdl(k_f16_pack<T, O>, dim3((warps * 32 + tx - 1) / tx, gy < 32768 ? gy : 32768), dim3(tx, ty), st, static_cast<const T*>(x), ld, (uint32_t)rows, (uint32_t)cols,
             static_cast<O*>(out), ldo);
  count_launches(1);
  return cudaGetLastError();
}
cudaError_t pack(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, void* out, int out_dtype, uint64_t ldo, cudaStream_t st) {
  using B = __nv_bfloat16;
  using H = __half;
  if (out_dtype == DS_BF16)
    return dtype == DS_F32 ? pack_as<float, B>(x, rows, cols, ld, out, ldo, st) : dtype == DS_BF16 ? pack_as<B, B>(x, rows, cols, ld, out, ldo, st)
                                                                                                  : pack_as<H, B>(x, rows, cols, ld, out, ldo, st);
  return dtype == DS_F32 ? pack_as<float, H>(x, rows, cols, ld, out, ldo, st) : dtype == DS_BF16 ? pack_as<B, H>(x, rows, cols, ld, out, ldo, st)
                                                                                                : pack_as<H, H>(x, rows, cols, ld, out, ldo, st);
}

// ---- an empty sum: act(bias) + residual -----------------------------------------------------------------
__global__ void __launch_bounds__(kThreads) k_f16_empty(const Out16 o) {
  pdl_prologue();
  const uint64_t r = blockIdx.x;
  for (uint32_t c = threadIdx.x; c < o.n; c += kThreads) {
    float v = o.bias ? o.bias[c] : 0.f;
    if (o.z) o.z[r * o.ldz + c] = half_of(v, o.bf16);
    with_act(o.act, [&](auto a) { v = act_of<decltype(a)::value>(v); });
    if (o.residual) v += from_half(o.residual[r * o.ldr + c], o.bf16);
    if (o.f32)
      static_cast<float*>(o.out)[r * o.ldo + c] = v;
    else
      static_cast<uint16_t*>(o.out)[r * o.ldo + c] = half_of(v, o.bf16);
  }
}

// ---- few tokens -----------------------------------------------------------------------------------------
// The weights' bytes are all that counts.  A CTA takes 16 or 32 rows of W; each of its eight warps has an eighth of K, which it
// reads in chunks of 32 entries a row, four chunks ahead, straight into the registers of m16n8k16 instructions (tokens are the
// 8 columns; the warp instruction is enough, the loop waits for memory).  K is dealt to the instructions' places as it arrives:
// lane t of a group of four loads 8 consecutive entries of its rows and tokens and feeds them as two instructions' worth.
// The warps' sums meet in shared memory and are added in the order of the warps.
constexpr uint32_t kFewMost = 16, kFewGroup = 8;

struct FewParams16 {
  const uint16_t *x, *w;
  uint64_t ldx, ldw;
  uint32_t k;
  Out16 o;
};

// 8 entries from k0 on; behind the end of a row nothing is read and zeros stand.
__device__ __forceinline__ uint4 load_halves8(const uint16_t* row, uint32_t k0, uint32_t k) {
  if (k0 + 8 <= k) return ld_plain(reinterpret_cast<const uint4*>(row + k0));
  uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    if (k0 + 2 * h < k) v[h] = row[k0 + 2 * h];
    if (k0 + 2 * h + 1 < k) v[h] |= (uint32_t)row[k0 + 2 * h + 1] << 16;
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}

template <bool BF16>
__device__ __forceinline__ void mma_half(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same of a row that starts anywhere; the granules are read that hold something of the row.
__device__ __forceinline__ uint4 load_halves8_anywhere(const uint16_t* row, uint32_t k0, uint32_t k) {
  if (k0 + 8 > k) return load_halves8(row, k0, k);      // entry by entry
  const uint32_t shift = shift_of(row);
  const uint4* at = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(row + k0) - shift);
  const uint4 a = ld_plain(at);
  if (!shift) return a;
  const uint4 b = ld_plain(at + 1);
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  take_from<4>(w, shift);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// NT: groups of 8 tokens, RB: blocks of 16 rows of W.  XVEC: tokens start on 16-byte boundaries (those of W always do).
template <bool BF16, int NT, int RB, bool XVEC>
__global__ void __launch_bounds__(256, 2) k_f16_few(const FewParams16 p) {
  constexpr int kAhead = 4;
  __shared__ float part[8][RB * 16][NT * 8 + 1];
  pdl_prologue();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t row0 = blockIdx.x * (16 * RB);
  const uint32_t chunks = p.k / 32, per = (chunks + 7) / 8;
  const uint32_t first = min(warp * per, chunks), end = min(first + per, chunks);
  const uint16_t *wrow[2 * RB], *xrow[NT];      // rows and tokens past the end: one that is there, not stored
#pragma unroll
  for (int i = 0; i < 2 * RB; ++i) wrow[i] = p.w + (uint64_t)min(row0 + g + 8 * i, p.o.n - 1) * p.ldw;
#pragma unroll
  for (int j = 0; j < NT; ++j) xrow[j] = p.x + min(8u * j + g, p.o.m - 1) * p.ldx;
  uint4 w[kAhead][2 * RB], xc[kAhead][NT];
  auto fetch = [&](uint32_t c, uint4 (&to)[2 * RB], uint4 (&xt)[NT]) {
    if (c >= end) return;
    const uint32_t k0 = c * 32 + t * 8;
#pragma unroll
    for (int i = 0; i < 2 * RB; ++i) to[i] = ld_plain(reinterpret_cast<const uint4*>(wrow[i] + k0));
#pragma unroll
    for (int j = 0; j < NT; ++j) xt[j] = XVEC ? ld_plain(reinterpret_cast<const uint4*>(xrow[j] + k0)) : load_halves8_anywhere(xrow[j], k0, p.k);
  };
#pragma unroll
  for (int a = 0; a < kAhead; ++a) fetch(first + a, w[a], xc[a]);
  float acc[RB][NT][4];
#pragma unroll
  for (int r = 0; r < RB; ++r)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[r][j][i] = 0.f;
  auto multiply = [&](const uint4 (&wc)[2 * RB], const uint4 (&x)[NT]) {
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const uint4 lo = wc[2 * r], hi = wc[2 * r + 1];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        mma_half<BF16>(acc[r][j], lo.x, hi.x, lo.y, hi.y, x[j].x, x[j].y);
        mma_half<BF16>(acc[r][j], lo.z, hi.z, lo.w, hi.w, x[j].z, x[j].w);
      }
    }
  };
  for (uint32_t c0 = first; c0 < end; c0 += kAhead) {
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const uint32_t c = c0 + a;
      if (c >= end) break;
      multiply(w[a], xc[a]);
      fetch(c + kAhead, w[a], xc[a]);
    }
  }
  if (warp == 7 && (p.k & 31)) {      // the rest of K
    const uint32_t k0 = chunks * 32 + t * 8;
    uint4 we[2 * RB], xe[NT];
#pragma unroll
    for (int i = 0; i < 2 * RB; ++i) we[i] = load_halves8(wrow[i], k0, p.k);
#pragma unroll
    for (int j = 0; j < NT; ++j) xe[j] = XVEC ? load_halves8(xrow[j], k0, p.k) : load_halves8_anywhere(xrow[j], k0, p.k);
    multiply(we, xe);
  }
#pragma unroll
  for (int r = 0; r < RB; ++r)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[warp][16 * r + g + 8 * (i >> 1)][8 * j + 2 * t + (i & 1)] = acc[r][j][i];
  __syncthreads();
  const Out16& o = p.o;
  for (uint32_t at = threadIdx.x; at < RB * 16 * o.m; at += 256) {
    const uint32_t token = at / (RB * 16), r = at % (RB * 16), row = row0 + r;
    if (row >= o.n) continue;
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) v += part[q][r][token];
    if (o.bias) v += ld_plain(o.bias + row);
    if (o.z) o.z[token * o.ldz + row] = half_of(v, BF16);
    with_act(o.act, [&](auto a) { v = act_of<decltype(a)::value>(v); });
    if (o.residual) v += from_half(ld_plain(o.residual + token * o.ldr + row), BF16);
    if (o.f32)
      static_cast<float*>(o.out)[token * o.ldo + row] = v;
    else
      static_cast<uint16_t*>(o.out)[token * o.ldo + row] = half_of(v, BF16);
  }
}

// CTAs of a form that an SM holds, asked for once a device.
template <auto KERNEL>
uint32_t ctas_an_sm() {
  constexpr int kMaxDevices = 64;
  static std::atomic<int> known[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 2;
  int n = known[dev].load(std::memory_order_relaxed);
  if (!n) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, KERNEL, 256, 0) != cudaSuccess || n < 1) {
      (void)cudaGetLastError();
      return 2;
    }
    known[dev].store(n, std::memory_order_relaxed);
  }
  return (uint32_t)n;
}
// What an SM goes through: rounds of CTAs, each taking as long as it has rows of W.
template <bool BF16, int NT, int RB, bool XVEC>
uint32_t few_cost(uint32_t n) {
  const uint32_t rows = ctas_an_sm<k_f16_few<BF16, NT, RB, XVEC>>() * 16 * RB, round = rows * (uint32_t)sm_count();
  return (n + round - 1) / round * rows;
}

template <bool BF16, int NT, bool XVEC>
cudaError_t launch_few16(const FewParams16& p, cudaStream_t st) {
  // 16 or 32 rows a CTA, by the rounds that they take (16 and 32, K = 4096, 148 SMs.  Up to 8 tokens three CTAs an SM and two: -> 7104 10.3 and 10.9 us, -> 7680 13.7 and 11.5,
  // -> 11008 16.2 and 17.6, -> 16384 23.1 and 21.7.  9 to 16 tokens, two and two: -> 4608 8.7 and 12.6, -> 6144 14.0 and 13.1, -> 11008 20.7 and 23.2)
  if (few_cost<BF16, NT, 2, XVEC>(p.o.n) <= few_cost<BF16, NT, 1, XVEC>(p.o.n))
    launch_pdl(k_f16_few<BF16, NT, 2, XVEC>, dim3((p.o.n + 31) / 32), dim3(256), st, p);
  else
    launch_pdl(k_f16_few<BF16, NT, 1, XVEC>, dim3((p.o.n + 15) / 16), dim3(256), st, p);
  count_launches(1);
  return cudaGetLastError();
}
template <bool BF16, int NT>
cudaError_t launch_few16(const FewParams16& p, cudaStream_t st) {
  return rows_on_boundary(p.x, p.ldx, p.o.m, 2) ? launch_few16<BF16, NT, true>(p, st) : launch_few16<BF16, NT, false>(p, st);
}

// ---- the gradient through the activation ----------------------------------------------------------------
// dz = dy act'(z) in 16 bits and, from what is not yet rounded, the column sums of each block of kSumRows rows; a second kernel adds
// the blocks in their order.  Bound by memory (4096 x 4096 in bf16: silu 17 us, 5.9 TB/s; gelu, whose instructions count, 23 us, 4.5 TB/s).  A lane has eight columns; a
// CTA's eight warps take every eighth row, four at a time.
// dz is rounded to 16 bits, since the operands of the matrix instructions that follow have as many, and z was kept so: half a step each, which leaves the gradients 1.4 times
// as far from exact ones as their own rounding does.
constexpr uint32_t kSumRows = 32;

// DY, Z: how the rows of dy, and of z and dz lie (what this package's layers keep starts on boundaries, a gradient may not).
template <class T, int ACT, int DY, int Z>
__global__ void __launch_bounds__(256, DY ? 4 : 3) k_f16_slope(const T* dy, uint64_t lddy, const T* z, uint64_t ldz, T* dz, uint64_t lddz, uint32_t rows, uint32_t cols, float* sums) {
  __shared__ float part[8][256];
  pdl_prologue();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t c = blockIdx.x * 256 + lane * 8, r0 = blockIdx.y * kSumRows + warp;
  float s[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] = 0.f;
  constexpr uint32_t kBatch = 4;      // rows in flight
#pragma unroll 1
  for (uint32_t i = 0; i < kSumRows; i += 8 * kBatch) {
    uint32_t g[kBatch][kWords<T> + 4], q[kBatch][kWords<T> + 4];
#pragma unroll
    for (uint32_t b = 0; b < kBatch; ++b) {
      const uint64_t r = r0 + i + 8 * b;
      if (r < rows) {
        load_words8<DY>(dy + r * lddy, c, cols, lane, g[b]);
        if constexpr (ACT != DS_ACT_NONE) load_words8<Z>(z + r * ldz, c, cols, lane, q[b]);
      }
    }
#pragma unroll
    for (uint32_t b = 0; b < kBatch; ++b) {
      const uint64_t r = r0 + i + 8 * b;
      if (r >= rows) break;
      float v[8], t[8];
      entries8<DY>(dy + r * lddy, g[b], c, cols, lane, v);
      if constexpr (ACT != DS_ACT_NONE) entries8<Z>(z + r * ldz, q[b], c, cols, lane, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (ACT != DS_ACT_NONE) v[j] *= slope_of<ACT>(t[j]);
        s[j] += v[j];
      }
      if (dz) store_row8<Z>(dz + r * lddz, c, cols, lane, v);
    }
  }
  if (!sums) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) part[warp][lane * 8 + j] = s[j];
  __syncthreads();
  const uint32_t col = blockIdx.x * 256 + threadIdx.x;
  if (col >= cols) return;
  float v = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) v += part[w][threadIdx.x];
  sums[(uint64_t)blockIdx.y * cols + col] = v;
}

template <class T>
void launch_slope(const ds_f16_slope_args* p, float* sums, dim3 grid, cudaStream_t st) {
  auto on = [&](const void* q, uint64_t ld) { return rows_on_boundary(q, ld, p->rows, 2); };
  const bool z = on(p->z, p->ldz) && on(p->dz, p->lddz), all = z && p->cols % 8 == 0 && on(p->dy, p->lddy);
  auto go = [&](auto kernel) {
    launch_pdl(kernel, grid, dim3(256), st, static_cast<const T*>(p->dy), p->lddy, static_cast<const T*>(p->z), p->ldz, static_cast<T*>(p->dz), p->lddz, (uint32_t)p->rows,
               (uint32_t)p->cols, sums);
  };
  auto by = [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    all ? go(k_f16_slope<T, ACT, kWhole, kWhole>) : z ? go(k_f16_slope<T, ACT, kAnywhere, kAligned>) : go(k_f16_slope<T, ACT, kAnywhere, kAnywhere>);
  };
  switch (p->activation) {
    case DS_ACT_NONE: return by(std::integral_constant<int, DS_ACT_NONE>());
    case DS_ACT_RELU: return by(std::integral_constant<int, DS_ACT_RELU>());
    case DS_ACT_GELU: return by(std::integral_constant<int, DS_ACT_GELU>());
    case DS_ACT_GELU_TANH: return by(std::integral_constant<int, DS_ACT_GELU_TANH>());
    default: return by(std::integral_constant<int, DS_ACT_SILU>());
  }
}

constexpr int kSumThreads = 512;
__global__ void __launch_bounds__(kSumThreads) k_f16_sums(const float* sums, uint32_t blocks, uint32_t cols, void* out, int f32, int bf16) {
  constexpr int kWarps = kSumThreads / 32, kBatch = 8;      // loads in flight
  __shared__ float part[kWarps][32];
  pdl_prologue();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t col = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (col < cols)
    for (uint32_t i = warp; i < blocks; i += kWarps * kBatch) {
      float t[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) t[b] = i + kWarps * b < blocks ? ld_plain(sums + (uint64_t)(i + kWarps * b) * cols + col) : 0.f;
#pragma unroll
      for (int b = 0; b < kBatch; ++b) v += t[b];
    }
  part[warp][lane] = v;
  __syncthreads();
  if (warp || col >= cols) return;
  v = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) v += part[w][lane];
  if (f32)
    static_cast<float*>(out)[col] = v;
  else
    static_cast<uint16_t*>(out)[col] = half_of(v, bf16);
}

// ---- host side ------------------------------------------------------------------------------------------

// Entries that rows of copied operands are a multiple of: whole lines of 128 bytes.  (Rows on other boundaries of 16 bytes span a line more in every step of K:
// 4096 x 4096 x 4104 takes 114 us so, and 88 on lines.)
constexpr uint64_t kLine = 64;

struct Shape16 {
  uint64_t rows_a, cols_a, rows_b, cols_b;      // as they lie in memory
  bool copy_a, copy_b;
  uint64_t bytes_a, bytes_b;
};
// Few tokens are multiplied by k_f16_few, but where TMA-fed tiles are faster: two groups of tokens and more rows of W than two CTAs an SM with 32 rows each take in a
// round (9 tokens, K = 4096, 148 SMs: -> 9472 15.7 and, by tiles, 17.2 us, -> 9504 18.6 and 16.5, -> 16384 26.9 and 24.6), or long rows and no more CTAs than SMs, so
// that a warp's eighth of K takes longer than memory does (8 tokens -> 1024: K = 8192 10.0 and 10.3, 10240 12.1 and 10.8, 16384 18.4 and 13.0; K = 12288 -> 2048 17.4 and
// 14.9, -> 4096 19.0 and 20.7).
constexpr uint64_t kFewLong = 8192;
bool few_tokens(const ds_f16_product* p) {
  const uint64_t sms = (uint64_t)sm_count();
  if (p->layout != DS_F16_FORWARD || p->m > kFewMost || (p->k > kFewLong && p->n <= 16 * sms)) return false;
  return p->m <= kFewGroup || p->n <= 2 * 32 * sms;
}
// Tokens on no boundary are read where they lie while rows are shorter than this, and copied else (a launch of its own and, in Python, memory for it): 8 tokens, K ->
// 2048, K = 512: 3.0 and, copied, 3.7 us, 2048: 6.7 and 5.8, 8192: 21.9 and 13.5; 16 tokens: 3.8 and 3.9, 9.5 and 6.3, 33.7 and 14.4.
constexpr uint64_t kFewWhereTheyLie = 2048;
Shape16 shape_of(const ds_f16_product* p) {
  Shape16 s;
  const bool a_across = p->layout == DS_F16_WEIGHTS, b_across = p->layout != DS_F16_FORWARD;
  s.rows_a = a_across ? p->k : p->m, s.cols_a = a_across ? p->m : p->k;
  s.rows_b = b_across ? p->k : p->n, s.cols_b = b_across ? p->n : p->k;
  // a single row has no pitch
  s.copy_a = (!few_tokens(p) || p->k >= kFewWhereTheyLie) && (!aligned(p->a, 16) || (s.rows_a > 1 && p->lda % 8));
  s.copy_b = !aligned(p->b, 16) || (s.rows_b > 1 && p->ldb % 8);
  s.bytes_a = s.copy_a ? round_up(s.rows_a * round_up(s.cols_a, kLine) * 2, 256) : 0;
  s.bytes_b = s.copy_b ? round_up(s.rows_b * round_up(s.cols_b, kLine) * 2, 256) : 0;
  return s;
}

// CTAs that share a tile's K, for few tokens: as many as run at once with at least four steps each, if that spares a tile 18 steps, which is what the exchange of their sums costs
// (17 tokens, split and not: 1536 -> 1536, 18 spared, 7.1 and 7.6 us; 2048 -> 6144, 16, 9.7 and 9.3; 1024 -> 4096, 12, 7.5 and 6.3; 4096 -> 6144, 32, 13.6 and 14.9).
inline uint32_t few_parts(uint32_t tiles, uint32_t k) {
  const uint32_t steps = (k + 63) / 64;
  uint32_t p = 1;
  while (p < 8 && tiles <= (uint32_t)cluster_count(2 * p) && steps >= 8 * p) p *= 2;
  return steps * (p - 1) >= 18 * p ? p : 1;
}

constexpr uint32_t kTurnedMost = 64;
// Up to 32 tokens have tiles of 32 columns, which plan_mma's times do not know: as good as its plan, and better where that is 64 columns and tokens are fewer than 16
// (10 tokens, 4096 -> 16384 24.5 and 28.3 us, 2048 -> 8192 9.6 and 11.4; 17 tokens 9.7 and 10.6, 4096 -> 8192 15.6 and 15.4).
constexpr uint32_t kNarrow = 32;

cudaError_t multiply(const ds_f16_product* p, const Out16& o, Operand16 a, Operand16 b, cudaStream_t st) {
  const uint32_t m = o.m, n = o.n, k = (uint32_t)p->k;
  if (few_tokens(p)) {
    const FewParams16 f{static_cast<const uint16_t*>(a.p), static_cast<const uint16_t*>(b.p), a.ld, b.ld, k, o};
    if (o.bf16) return m <= kFewGroup ? launch_few16<true, 1>(f, st) : launch_few16<true, 2>(f, st);
    return m <= kFewGroup ? launch_few16<false, 1>(f, st) : launch_few16<false, 2>(f, st);
  }
  const MmaShape s{m, n, k, 1, 2, 0, 0, p->dev_status, 1, (uint32_t)o.bf16};
  const bool bare = !o.residual && !o.z && !o.bias && !o.act;
  // (rows that end inside 16 bytes: a block's store would write the rest of them, which is not the matrix's)
  const bool blocks = !o.f32 && n % 8 == 0 && aligned(o.out, 16) && o.ldo % 8 == 0 && (!o.residual || (aligned(o.residual, 16) && o.ldr % 8 == 0)) &&
                      (!o.z || (aligned(o.z, 16) && o.ldz % 8 == 0)) && (p->layout == DS_F16_FORWARD || bare);
  const bool floats = o.f32 && bare && aligned(o.out, 32) && o.ldo % 8 == 0;
  if (m <= kTurnedMost || !(blocks || floats)) {
    const MmaShape t{n, m, k, 1, 2, 0, 0, p->dev_status, 1, (uint32_t)o.bf16};
    MmaPlan plan = plan_mma(t);
    if (m <= kNarrow && !a.across && !b.across) {
      plan.pair = false;
      plan.bn = 32;
      plan.parts = few_parts(TileWalk(t, 32).total, k);
    }
    return product16_turned(plan, b, a, t, EpiTurned{o}, st);
  }
  const MmaPlan plan = plan_mma(s);
  if (floats) return product16_floats(plan, a, b, s, EpiFloats{static_cast<float*>(o.out), o.ldo, m, n}, st);
  auto maps = [&](auto& epi) {
    cudaError_t e = make_tensor_map(&epi.map_y, kMmaHalf, o.out, n, m, 1, o.ldo, o.ldo * m, 32, 32, true);
    if (e == cudaSuccess && o.residual) e = make_tensor_map(&epi.map_r, kMmaHalf, o.residual, n, m, 1, o.ldr, o.ldr * m, 32, 32, true);
    if (e == cudaSuccess && o.z) e = make_tensor_map(&epi.map_z, kMmaHalf, o.z, n, m, 1, o.ldz, o.ldz * m, 32, 32, true);
    epi.o = o;
    epi.bias_vec = aligned(o.bias, 16);
    return e;
  };
  if (o.z) {
    EpiBlocks<2> epi{};
    const cudaError_t e = maps(epi);
    return e != cudaSuccess ? e : product16_forward_z(plan, a, b, s, epi, st);
  }
  EpiBlocks<1> epi{};
  const cudaError_t e = maps(epi);
  if (e != cudaSuccess) return e;
  return p->layout == DS_F16_FORWARD ? product16_forward(plan, a, b, s, epi, st) : product16_gradient(plan, a, b, s, epi, st);
}

int check_product(const ds_f16_product* p) {
  if (!p || !half_ok(p->dtype) || p->layout > DS_F16_WEIGHTS || p->activation > DS_ACT_SILU) return DS_ERR_INVALID_ARG;
  if (p->out_dtype != DS_F32 && p->out_dtype != p->dtype) return DS_ERR_INVALID_ARG;
  if (p->m > kMaxLen || p->n > kMaxLen || p->k > kMaxLen) return DS_ERR_INVALID_ARG;
  return DS_OK;
}

}  // namespace

extern "C" {

int ds_f16_pack(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, void* out, int out_dtype, uint64_t ldo, void* cuda_stream) {
  if (!dtype_ok(dtype) || !half_ok(out_dtype) || rows > kMaxLen || cols > kMaxLen || ldo > kMaxLen + 8) return DS_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return DS_OK;
  if (!x || !out || (ld < cols && rows > 1) || ldo < cols) return DS_ERR_INVALID_ARG;
  if (!aligned(x, size_of(dtype)) || !aligned(out, 16) || ldo % 8) return DS_ERR_ALIGN;
  if (overlap(span(x, rows, cols, ld, size_of(dtype)), span(out, rows, ldo, ldo, 2))) return DS_ERR_INVALID_ARG;
  const cudaError_t e = pack(x, dtype, rows, cols, ld, out, out_dtype, ldo, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "16-bit copy");
}

uint64_t ds_f16_matmul_workspace(const ds_f16_product* p) {
  if (check_product(p) != DS_OK || !p->m || !p->n || !p->k) return 0;
  const Shape16 s = shape_of(p);
  return s.bytes_a + s.bytes_b;
}

int ds_f16_matmul(const ds_f16_product* p, void* cuda_stream) {
  const int rc = check_product(p);
  if (rc != DS_OK) return rc;
  if (p->m == 0 || p->n == 0) return DS_OK;
  if (!p->out || (p->m > 1 && p->ldo < p->n)) return DS_ERR_INVALID_ARG;
  if ((p->residual && p->m > 1 && p->ldr < p->n) || (p->z && p->m > 1 && p->ldz < p->n)) return DS_ERR_INVALID_ARG;
  if (!aligned(p->out, size_of(p->out_dtype)) || !aligned(p->bias, 4) || !aligned(p->residual, 2) || !aligned(p->z, 2) || !aligned(p->dev_status, 4))
    return DS_ERR_ALIGN;
  const Shape16 s = shape_of(p);
  const Span out = span(p->out, p->m, p->n, p->ldo, size_of(p->out_dtype)), z = span(p->z, p->m, p->n, p->ldz, 2),
             res = span(p->residual, p->m, p->n, p->ldr, 2), bias = span(p->bias, 1, p->n, p->n, 4);
  // the residual may be added to in place
  const bool in_place = p->residual == p->out && (p->ldr == p->ldo || p->m == 1) && p->out_dtype != DS_F32;
  if (overlap(out, z) || overlap(res, z) || (!in_place && overlap(out, res)) || overlap(out, bias) || overlap(z, bias)) return DS_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const Out16 o{p->bias, static_cast<const uint16_t*>(p->residual), static_cast<uint16_t*>(p->z), p->out, p->ldr, p->ldz, p->ldo, (uint32_t)p->m, (uint32_t)p->n,
                (int)p->activation, p->dtype == DS_BF16, p->out_dtype == DS_F32};
  cudaError_t e = cudaSuccess;
  if (p->k == 0) {
    launch_pdl(k_f16_empty, dim3(o.m), dim3(kThreads), st, o);
    count_launches(1);
    e = cudaGetLastError();
    return e == cudaSuccess ? DS_OK : cuda_fail(e, "16-bit product");
  }
  if (!p->a || !p->b || (s.rows_a > 1 && p->lda < s.cols_a) || (s.rows_b > 1 && p->ldb < s.cols_b)) return DS_ERR_INVALID_ARG;
  if (!aligned(p->a, 2) || !aligned(p->b, 2)) return DS_ERR_ALIGN;
  const Span sa = span(p->a, s.rows_a, s.cols_a, p->lda, 2), sb = span(p->b, s.rows_b, s.cols_b, p->ldb, 2);
  if (overlap(out, sa) || overlap(out, sb) || overlap(z, sa) || overlap(z, sb)) return DS_ERR_INVALID_ARG;
  if (s.bytes_a + s.bytes_b) {
    if (!p->workspace) return DS_ERR_INVALID_ARG;
    if (!aligned(p->workspace, 16)) return DS_ERR_ALIGN;
    if (p->workspace_bytes < s.bytes_a + s.bytes_b) return DS_ERR_BUFFER_TOO_SMALL;
    const Span ws = span(p->workspace, 1, s.bytes_a + s.bytes_b, s.bytes_a + s.bytes_b, 1);
    if (overlap(ws, sa) || overlap(ws, sb) || overlap(ws, out) || overlap(ws, z) || overlap(ws, res) || overlap(ws, bias)) return DS_ERR_INVALID_ARG;
  }
  const bool a_across = p->layout == DS_F16_WEIGHTS, b_across = p->layout != DS_F16_FORWARD;
  // a single row's pitch is the caller's word for nothing: one that a tensor map takes
  Operand16 a{p->a, s.rows_a > 1 ? p->lda : round_up(s.cols_a, 8), o.m, a_across}, b{p->b, s.rows_b > 1 ? p->ldb : round_up(s.cols_b, 8), o.n, b_across};
  uint8_t* ws = static_cast<uint8_t*>(p->workspace);
  if (s.copy_a) {
    const uint64_t ld = round_up(s.cols_a, kLine);
    e = pack(p->a, (int)p->dtype, s.rows_a, s.cols_a, p->lda, ws, (int)p->dtype, ld, st);
    a.p = ws, a.ld = ld;
  }
  if (e == cudaSuccess && s.copy_b) {
    const uint64_t ld = round_up(s.cols_b, kLine);
    e = pack(p->b, (int)p->dtype, s.rows_b, s.cols_b, p->ldb, ws + s.bytes_a, (int)p->dtype, ld, st);
    b.p = ws + s.bytes_a, b.ld = ld;
  }
  if (e == cudaSuccess) e = multiply(p, o, a, b, st);
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "16-bit product");
}

uint64_t ds_f16_slope_workspace(uint64_t rows, uint64_t cols) { return 4 * ((rows + kSumRows - 1) / kSumRows) * cols; }

int ds_f16_slope(const ds_f16_slope_args* p, void* cuda_stream) {
  if (!p || !half_ok(p->dtype) || p->activation > DS_ACT_SILU || p->rows > kMaxLen || p->cols > kMaxLen) return DS_ERR_INVALID_ARG;
  if (p->sum && p->sum_dtype != DS_F32 && p->sum_dtype != p->dtype) return DS_ERR_INVALID_ARG;
  if (p->cols == 0) return DS_OK;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (!aligned(p->sum, p->sum ? size_of(p->sum_dtype) : 1)) return DS_ERR_ALIGN;
  if (p->rows == 0) {
    const cudaError_t e = p->sum ? cudaMemsetAsync(p->sum, 0, size_of(p->sum_dtype) * p->cols, st) : cudaSuccess;
    return e == cudaSuccess ? DS_OK : cuda_fail(e, "clearing sums");
  }
  if (!p->dy || (p->activation != DS_ACT_NONE) != (p->z != nullptr) || (!p->dz && !p->sum)) return DS_ERR_INVALID_ARG;
  if (p->rows > 1 && (p->lddy < p->cols || (p->z && p->ldz < p->cols) || (p->dz && p->lddz < p->cols))) return DS_ERR_INVALID_ARG;
  if (!aligned(p->dy, 2) || !aligned(p->z, 2) || !aligned(p->dz, 2)) return DS_ERR_ALIGN;
  const uint64_t blocks = (p->rows + kSumRows - 1) / kSumRows;
  if (blocks > 65535) return DS_ERR_UNSUPPORTED;
  const Span dy = span(p->dy, p->rows, p->cols, p->lddy, 2), z = span(p->z, p->rows, p->cols, p->ldz, 2), dz = span(p->dz, p->rows, p->cols, p->lddz, 2),
             sum = span(p->sum, 1, p->cols, p->cols, p->sum ? size_of(p->sum_dtype) : 0);
  // in place over dy or z, entry by entry
  auto itself = [&](const void* q, uint64_t ld) { return p->dz == q && (p->lddz == ld || p->rows == 1); };
  if ((overlap(dz, dy) && !itself(p->dy, p->lddy)) || (overlap(dz, z) && !itself(p->z, p->ldz)) || overlap(sum, dz) || overlap(sum, dy) || overlap(sum, z))
    return DS_ERR_INVALID_ARG;
  float* sums = nullptr;
  if (p->sum) {
    if (!p->workspace) return DS_ERR_INVALID_ARG;
    if (!aligned(p->workspace, 16)) return DS_ERR_ALIGN;
    if (p->workspace_bytes < ds_f16_slope_workspace(p->rows, p->cols)) return DS_ERR_BUFFER_TOO_SMALL;
    const Span ws = span(p->workspace, 1, ds_f16_slope_workspace(p->rows, p->cols), ds_f16_slope_workspace(p->rows, p->cols), 1);
    if (overlap(ws, dy) || overlap(ws, z) || overlap(ws, dz) || overlap(ws, sum)) return DS_ERR_INVALID_ARG;
    sums = static_cast<float*>(p->workspace);
  }
  const dim3 grid((uint32_t)((p->cols + 255) / 256), (uint32_t)blocks);
  if (p->dtype == DS_BF16)
    launch_slope<__nv_bfloat16>(p, sums, grid, st);
  else
    launch_slope<__half>(p, sums, grid, st);
  count_launches(1);
  if (p->sum) {
    launch_pdl(k_f16_sums, dim3((uint32_t)((p->cols + 31) / 32)), dim3(kSumThreads), st, (const float*)sums, (uint32_t)blocks, (uint32_t)p->cols, p->sum,
               (int)(p->sum_dtype == DS_F32), (int)(p->dtype == DS_BF16));
    count_launches(1);
  }
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "gradient through the activation");
}

}  // extern "C"
