// Dropout by itself, of activations or of their gradients: y = keep ? x * scale : 0 with the mask of dsq_dropout.cuh.  Bound by memory
// where entries have 32 bits (16384 x 8192: 158 us, 6.8 TB/s), near the generator's rate in 16 (twenty 32 x 32-bit products for eight entries: 91 us, 5.9 TB/s).
#include "dsq_dropout.cuh"
#include "dsq_mma.cuh"
#include "dsq_rows8.cuh"

using namespace dsq;

namespace {

// A warp has 256 neighbouring entries of a row, blockDim.x / 32 warps side by side, blockDim.y rows at once; a thread has kBatch rows in flight.  (One
// row a thread: 16384 x 8192 in bf16 124 us.)
constexpr int kBatch = 4;
template <class T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_dropout(const T* x, uint64_t ldx, T* out, uint64_t ldo, uint32_t rows, uint32_t cols, const Drop drop) {
  pdl_prologue();
  const uint32_t c = (blockIdx.x * blockDim.x + threadIdx.x) * 8, step = gridDim.y * blockDim.y;
  const int lane = threadIdx.x & 31;
  if (c - 8 * lane >= cols) return;
  for (uint32_t first = blockIdx.y * blockDim.y + threadIdx.y; first < rows; first += kBatch * step) {
    uint32_t w[kBatch][kWords<T> + 4];
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
      if (first + b * step < rows) load_words8<VEC>(x + (first + b * step) * ldx, c, cols, lane, w[b]);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const uint32_t row = first + b * step;
      if (row >= rows) break;
      float v[8];
      entries8<VEC>(x + row * ldx, w[b], c, cols, lane, v);
      if (drop.threshold) drop8(drop, draw8(drop, row, c), v);
      store_row8<VEC>(out + row * ldo, c, cols, lane, v);
    }
  }
}

// Rows of x and out that start at the same place within 8 entries' bytes, on any boundary of an entry: a thread has the 8 entries between two such boundaries, which no
// neighbour has to hand anything of, and shifts the random words instead, which are those of two groups of columns.  A warp's first lane draws the words that the second one
// lacks, and no more: 31 pieces a warp.  (By pieces of columns, handed over twice: 16384 x 8191 in bf16 215 us.)
template <class T>
__global__ void __launch_bounds__(kThreads) k_dropout_apart(const T* x, uint64_t ldx, T* out, uint64_t ldo, uint32_t rows, uint32_t cols, const Drop drop) {
  constexpr int N = kWords<T>;
  pdl_prologue();
  const int lane = threadIdx.x & 31;
  const uint32_t step = gridDim.y * blockDim.y;
  const int piece = (int)((blockIdx.x * blockDim.x + threadIdx.x) / 32 * 31) + lane - 1;
  for (uint32_t first = blockIdx.y * blockDim.y + threadIdx.y; first < rows; first += kBatch * step) {
    uint32_t w[kBatch][N];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const uint32_t row = first + b * step;
      if (row >= rows) break;
      const T* at = x + row * ldx;
      const uint32_t apart = (uint32_t)(reinterpret_cast<uintptr_t>(at) / sizeof(T)) & 7;      // entries from the boundary to the row's first
      const int c = 8 * piece - (int)apart;
      // a granule is read if it holds something of the row
#pragma unroll
      for (int g = 0; g < N / 4; ++g) {
        uint4 q = make_uint4(0, 0, 0, 0);
        const int from = c + g * (int)(16 / sizeof(T));
        if (lane && from < (int)cols && from + (int)(16 / sizeof(T)) > 0) q = ld_plain(reinterpret_cast<const uint4*>(at + c) + g);
        w[b][4 * g] = q.x, w[b][4 * g + 1] = q.y, w[b][4 * g + 2] = q.z, w[b][4 * g + 3] = q.w;
      }
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const uint32_t row = first + b * step;
      if (row >= rows) break;
      T* to = out + row * ldo;
      const uint32_t apart = (uint32_t)(reinterpret_cast<uintptr_t>(to) / sizeof(T)) & 7;
      const int c = 8 * piece - (int)apart;
      // words of the piece before and of this one: the halves from 8 - apart on
      const uint4 mine = draw8(drop, row, (uint32_t)(8 * piece));
      uint32_t r[8] = {__shfl_up_sync(0xFFFFFFFFu, mine.x, 1), __shfl_up_sync(0xFFFFFFFFu, mine.y, 1), __shfl_up_sync(0xFFFFFFFFu, mine.z, 1),
                       __shfl_up_sync(0xFFFFFFFFu, mine.w, 1), mine.x, mine.y, mine.z, mine.w};
      if (apart)
        take_from<4>(r, 16 - 2 * apart);
      else
        r[0] = mine.x, r[1] = mine.y, r[2] = mine.z, r[3] = mine.w;
      float v[8];
      unpack8<T>(w[b], v);
      drop8(drop, make_uint4(r[0], r[1], r[2], r[3]), v);
      if (!lane || c >= (int)cols || c + 8 <= 0) continue;
      if (c >= 0 && c + 8 <= (int)cols) {
        store_piece8(to + c, v);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j >= 0 && c + j < (int)cols) to[c + j] = from_float<T>(v[j]);
      }
    }
  }
}

inline bool aligned(const void* p, uint64_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <class T>
cudaError_t launch(const void* x, uint64_t ldx, void* out, uint64_t ldo, uint32_t rows, uint32_t cols, const Drop& drop, cudaStream_t st) {
  const bool vec = cols % 8 == 0 && rows_on_boundary(x, ldx, rows, sizeof(T)) && rows_on_boundary(out, ldo, rows, sizeof(T));
  const uint64_t off = reinterpret_cast<uintptr_t>(x) / sizeof(T) - reinterpret_cast<uintptr_t>(out) / sizeof(T);
  const bool same = !vec && drop.threshold && off % 8 == 0 && (rows == 1 || (ldx - ldo) % 8 == 0);
  const uint32_t warps = same ? ((cols + 14) / 8 + 30) / 31 : (cols + 255) / 256;
  const uint32_t tx = 32 * (warps < 8 ? warps : 8), ty = kThreads / tx, gx = (warps * 32 + tx - 1) / tx;
  // kBatch rows a thread where that leaves eight CTAs an SM
  const uint32_t all = (rows + ty - 1) / ty, fewest = (rows + kBatch * ty - 1) / (kBatch * ty), wanted = (8 * (uint32_t)sm_count() + gx - 1) / gx;
  uint32_t gy = wanted < fewest ? fewest : wanted < all ? wanted : all;
  if (gy > 32768) gy = 32768;
  auto kernel = same ? k_dropout_apart<T> : vec ? k_dropout<T, true> : k_dropout<T, false>;
  launch_pdl(kernel, dim3(gx, gy), dim3(tx, ty), st, static_cast<const T*>(x), ldx, static_cast<T*>(out), ldo, rows, cols, drop);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace

extern "C" int ds_dropout(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, void* out, uint64_t ldo, uint32_t threshold, uint64_t seed, uint32_t layer,
                          uint32_t step, void* cuda_stream) {
  if (dtype < DS_F32 || dtype > DS_F16 || rows > (1ull << 30) || cols > (1ull << 30) || threshold > 65535) return DS_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return DS_OK;
  if (!x || !out || (rows > 1 && (ldx < cols || ldo < cols))) return DS_ERR_INVALID_ARG;
  const uint32_t size = dtype == DS_F32 ? 4 : 2;
  if (!aligned(x, size) || !aligned(out, size)) return DS_ERR_ALIGN;
  // over its input only entry by entry
  if (overlap(span(x, rows, cols, ldx, size), span(out, rows, cols, ldo, size)) && !(x == out && (ldx == ldo || rows == 1))) return DS_ERR_INVALID_ARG;
  const Drop drop = make_drop(threshold, seed, layer, step);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == DS_F32    ? launch<float>(x, ldx, out, ldo, (uint32_t)rows, (uint32_t)cols, drop, st)
                        : dtype == DS_BF16 ? launch<__nv_bfloat16>(x, ldx, out, ldo, (uint32_t)rows, (uint32_t)cols, drop, st)
                                           : launch<__half>(x, ldx, out, ldo, (uint32_t)rows, (uint32_t)cols, drop, st);
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "dropout");
}
