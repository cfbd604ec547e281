// Dropout by itself, of activations or of their gradients: y = keep ? x * scale : 0 with the mask of dsq_dropout.cuh.  Bound by memory
// where entries have 32 bits, near the generator's rate in 16 (twenty 32 x 32-bit products for eight entries).
#include "dsq_dropout.cuh"
#include "dsq_rows8.cuh"

using namespace dsq;

namespace {

// A warp has 256 neighbouring entries of a row, blockDim.x / 32 warps side by side, blockDim.y rows at once; two rows in flight a thread.
template <class T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_dropout(const T* x, uint64_t ldx, T* out, uint64_t ldo, uint32_t rows, uint32_t cols, const Drop drop) {
  pdl_prologue();
  const uint32_t c = (blockIdx.x * blockDim.x + threadIdx.x) * 8, step = gridDim.y * blockDim.y;
  const int lane = threadIdx.x & 31;
  if (c - 8 * lane >= cols) return;
  for (uint32_t row = blockIdx.y * blockDim.y + threadIdx.y; row < rows; row += 2 * step) {
    const bool two = row + step < rows;
    float v[8], u[8];
    load_row8<VEC>(x + row * ldx, c, cols, lane, v);
    if (two) load_row8<VEC>(x + (row + step) * ldx, c, cols, lane, u);
    if (drop.threshold) drop8(drop, draw8(drop, row, c), v);
    store_row8<VEC>(out + row * ldo, c, cols, lane, v);
    if (two) {
      if (drop.threshold) drop8(drop, draw8(drop, row + step, c), u);
      store_row8<VEC>(out + (row + step) * ldo, c, cols, lane, u);
    }
  }
}

inline bool aligned(const void* p, uint64_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <class T>
cudaError_t launch(const void* x, uint64_t ldx, void* out, uint64_t ldo, uint32_t rows, uint32_t cols, const Drop& drop, cudaStream_t st) {
  const uint32_t warps = (cols + 255) / 256;
  const uint32_t tx = 32 * (warps < 8 ? warps : 8), ty = kThreads / tx, gx = (warps * 32 + tx - 1) / tx;
  const bool vec = cols % 8 == 0 && rows_on_boundary(x, ldx, rows, sizeof(T)) && rows_on_boundary(out, ldo, rows, sizeof(T));
  const uint32_t gy = (rows + ty - 1) / ty;
  launch_pdl(vec ? k_dropout<T, true> : k_dropout<T, false>, dim3(gx, gy < 32768 ? gy : 32768), dim3(tx, ty), st, static_cast<const T*>(x), ldx, static_cast<T*>(out), ldo,
             rows, cols, drop);
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
  const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(out);
  if (a < b + ((rows - 1) * ldo + cols) * size && b < a + ((rows - 1) * ldx + cols) * size && !(a == b && (ldx == ldo || rows == 1))) return DS_ERR_INVALID_ARG;
  const Drop drop = make_drop(threshold, seed, layer, step);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = dtype == DS_F32    ? launch<float>(x, ldx, out, ldo, (uint32_t)rows, (uint32_t)cols, drop, st)
                        : dtype == DS_BF16 ? launch<__nv_bfloat16>(x, ldx, out, ldo, (uint32_t)rows, (uint32_t)cols, drop, st)
                                           : launch<__half>(x, ldx, out, ldo, (uint32_t)rows, (uint32_t)cols, drop, st);
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "dropout");
}
