// Matrix products on the fifth-generation tensor cores (tcgen05), shared by the orthogonalised update (16-bit
// floating operands) and the 8-bit layer products: C = A B^T with A [M, K] and B [N, K], both laid out along K, or B
// given as [K, N] (16-bit only).
//
// One CTA per SM walks over 128 x BN tiles of C.  Warp 0 fetches operand tiles by TMA into a ring of stages (rows of 128
// bytes, 128-byte swizzle), one thread of warp 1 issues the matrix instructions, and warps 4..11 read the finished
// accumulator out of tensor memory and hand it to an epilogue.  Two accumulators alternate, so the epilogue of a tile
// runs under the products of the next one.
//
// Every wait is bounded (kWaitCycles): a wait that runs out sets DS_DEV_MMA_TIMEOUT in the device status word, and the CTA
// drains its copies, frees its tensor memory and leaves.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dsq_internal.h"

namespace dsq {

constexpr int kMmaThreads = 384;          // 4 warps of plumbing, 8 of epilogue
constexpr int kMmaRows = 128;             // rows of a tile: the lanes of tensor memory
constexpr long long kWaitCycles = 2000000000ll;   // about one second

enum MmaKind : int { kMmaF16 = 0, kMmaI8 = 1 };

// ---- PTX ------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// Waits until the phase of the given parity has completed.  False: another role gave up, or the limit ran out (which
// makes the others give up too).
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
  if (mbar_try(bar, parity)) return true;
  const long long t0 = clock64();
  while (true) {
    for (int i = 0; i < 16; ++i)
      if (mbar_try(bar, parity)) return true;
    if (*gave_up) return false;
    if (clock64() - t0 > kWaitCycles) {
      *gave_up = 1;
      return false;
    }
  }
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
__device__ __forceinline__ void tmem_alloc(uint32_t smem_dst, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <int KIND>
__device__ __forceinline__ void tc_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  if constexpr (KIND == kMmaF16)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 32 consecutive columns of this warp's 32 lanes: register j of lane l is (lane l, column j).
__device__ __forceinline__ void tmem_load32(uint32_t (&r)[32], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Shared-memory descriptor of an operand tile whose rows are 128 bytes, swizzled by 128 bytes (atoms of 8 rows, 1024
// bytes).  Laid out along K: `stride` = bytes between groups of eight rows.  Laid out across K: `stride` = bytes between
// groups of eight k, `lead` = bytes between blocks of 64 columns.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead, uint32_t stride) {
  return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)((lead >> 4) & 0x3FFFu) << 16) | ((uint64_t)((stride >> 4) & 0x3FFFu) << 32) |
         (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: f16 x f16 -> f32, or s8 x s8 -> s32; M = 128.
template <int KIND, int BN, bool B_ACROSS>
__host__ __device__ constexpr uint32_t mma_idesc() {
  const uint32_t types = KIND == kMmaF16 ? (1u << 4) : ((2u << 4) | (1u << 7) | (1u << 10));
  return types | (B_ACROSS ? 1u << 16 : 0u) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(kMmaRows >> 4) << 24);
}

// ---- the product ----------------------------------------------------------------------------------------

struct MmaShape {
  uint32_t m, n, k;        // C is [m, n] per matrix of the batch
  uint32_t batch;
  uint32_t sym;            // 1: C is symmetric; only 32 x 32 blocks on or above the diagonal are handed to the epilogue
  uint32_t* dev_status;
};

template <int BN>
struct MmaTile {
  static constexpr int kStageBytes = (kMmaRows + BN) * 128;
  static constexpr int kStages = BN == 256 ? 4 : BN == 192 ? 5 : BN == 128 ? 6 : 8;
  static constexpr int kTmemCols = BN == 192 ? 512 : 2 * BN;
  static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024;
};

// Tiles of C in the order in which CTAs take them.
struct TileWalk {
  uint32_t mt, nt, per, total, sym, bn;
  __host__ __device__ TileWalk(const MmaShape& s, uint32_t bn_) : sym(s.sym), bn(bn_) {
    mt = (s.m + kMmaRows - 1) / kMmaRows;
    nt = (s.n + bn - 1) / bn;
    if (sym) {
      per = 0;
      for (uint32_t i = 0; i < mt; ++i) per += nt - i * kMmaRows / bn;
    } else {
      per = mt * nt;
    }
    total = per * s.batch;
  }
  __host__ __device__ void at(uint32_t t, uint32_t& b, uint32_t& i, uint32_t& j) const {
    b = t / per;
    t -= b * per;
    if (sym) {
      i = 0;
      while (true) {
        const uint32_t first = i * kMmaRows / bn, c = nt - first;
        if (t < c) {
          j = first + t;
          return;
        }
        t -= c;
        ++i;
      }
    }
    // bands of eight tile rows, column by column: the operands of the tiles in flight stay in L2
    const uint32_t band = 8 * nt, g = t / band, r = t - g * band;
    const uint32_t h = mt - 8 * g < 8 ? mt - 8 * g : 8;
    j = r / h;
    i = 8 * g + r - j * h;
  }
};

// Epi: struct with
//   struct Pre                                      what it reads from global memory for one block of 32 columns
//   Pre load(row, col0, batch) const               (row may be out of range)
//   void apply(pre, acc, row, col0, batch) const   acc: 32 raw accumulators of one row
template <int KIND, int BN, bool B_ACROSS, class Epi>
__global__ void __launch_bounds__(kMmaThreads, 1)
    k_mma(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const MmaShape shape, const Epi epi) {
  using T = MmaTile<BN>;
  constexpr int kBK = KIND == kMmaF16 ? 64 : 128;    // elements of K per stage: 128 bytes
  extern __shared__ uint8_t dyn[];
  __shared__ uint64_t bars[2 * T::kStages + 5];
  __shared__ uint32_t tmem_slot;
  __shared__ int gave_up;
  const uint32_t ring = (smem_u32(dyn) + 1023u) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * T::kStages, tfull = empty + 8 * T::kStages, tempty = tfull + 16,
                 drain = tempty + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    tma_prefetch_map(&map_a);
    tma_prefetch_map(&map_b);
    for (int i = 0; i < T::kStages; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull + 8 * i, 1);
      mbar_init(tempty + 8 * i, 8);
    }
    mbar_init(drain, 1);
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 2) tmem_alloc(smem_u32(&tmem_slot), T::kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  // Only now may the next kernel's CTAs come in: one that took this SM's tensor memory before this CTA had its share would
  // wait for this kernel while this kernel waits for it.
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  const TileWalk walk(shape, BN);
  const uint32_t nk = (shape.k + kBK - 1) / kBK;

  if (warp == 0 && lane == 0) {
    asm volatile("fence.proxy.async.global;" ::: "memory");
    uint32_t stage = 0, phase = 0, issued = 0;
    bool ok = true;
    for (uint32_t t = blockIdx.x; ok && t < walk.total; t += gridDim.x) {
      uint32_t b, i, j;
      walk.at(t, b, i, j);
      for (uint32_t kb = 0; kb < nk; ++kb) {
        if (!(ok = mbar_wait(empty + 8 * stage, phase ^ 1, &gave_up))) break;
        const uint32_t dst = ring + stage * T::kStageBytes;
        mbar_expect_tx(full + 8 * stage, T::kStageBytes);
        tma_load_3d(dst, &map_a, (int)(kb * kBK), (int)(i * kMmaRows), (int)b, full + 8 * stage);
        if constexpr (B_ACROSS) {
#pragma unroll
          for (int c = 0; c < BN / 64; ++c)
            tma_load_3d(dst + kMmaRows * 128 + c * (kBK * 128), &map_b, (int)(j * BN + c * 64), (int)(kb * kBK), (int)b, full + 8 * stage);
        } else {
          tma_load_3d(dst + kMmaRows * 128, &map_b, (int)(kb * kBK), (int)(j * BN), (int)b, full + 8 * stage);
        }
        ++issued;
        if (++stage == T::kStages) {
          stage = 0;
          phase ^= 1;
        }
      }
    }
    if (!ok) {   // copies in flight must have landed before this CTA's shared memory is given away
      const uint32_t last = issued < (uint32_t)T::kStages ? issued : (uint32_t)T::kStages;
      for (uint32_t q = 0; q < last; ++q) {
        stage = stage ? stage - 1 : T::kStages - 1;
        const uint32_t use = (issued - 1 - q) / T::kStages;
        const long long t0 = clock64();
        while (!mbar_try(full + 8 * stage, use & 1) && clock64() - t0 < kWaitCycles) {
        }
      }
    }
  } else if (warp == 1 && lane == 0) {
    constexpr uint32_t idesc = mma_idesc<KIND, BN, B_ACROSS>();
    uint32_t stage = 0, phase = 0, at = 0, aphase = 0;
    bool ok = true;
    for (uint32_t t = blockIdx.x; ok && t < walk.total; t += gridDim.x) {
      if (!(ok = mbar_wait(tempty + 8 * at, aphase ^ 1, &gave_up))) break;
      tc_fence_after();
      const uint32_t d = tmem + at * BN;
      for (uint32_t kb = 0; kb < nk; ++kb) {
        if (!(ok = mbar_wait(full + 8 * stage, phase, &gave_up))) break;
        tc_fence_after();
        const uint32_t sa = ring + stage * T::kStageBytes, sb = sa + kMmaRows * 128;
#pragma unroll
        for (int q = 0; q < 4; ++q) {   // four instructions of 32 bytes of K
          const uint64_t da = smem_desc(sa + 32 * q, 16, 1024);
          const uint64_t db = B_ACROSS ? smem_desc(sb + 2048 * q, kBK * 128, 1024) : smem_desc(sb + 32 * q, 16, 1024);
          tc_mma<KIND>(d, da, db, idesc, (kb | q) != 0);
        }
        tc_commit(empty + 8 * stage);
        if (++stage == T::kStages) {
          stage = 0;
          phase ^= 1;
        }
      }
      if (!ok) break;
      tc_commit(tfull + 8 * at);
      if (++at == 2) {
        at = 0;
        aphase ^= 1;
      }
    }
    if (!ok) {   // products in flight must have ended before the tensor memory is freed
      tc_commit(drain);
      const long long t0 = clock64();
      while (!mbar_try(drain, 0) && clock64() - t0 < kWaitCycles) {
      }
    }
  } else if (warp >= 4) {
    // two groups of four warps; a warp reads the 32 lanes that its rank in the group names
    const uint32_t quarter = warp & 3, group = (warp - 4) >> 2;
    uint32_t at = 0, aphase = 0;
    for (uint32_t t = blockIdx.x; t < walk.total; t += gridDim.x) {
      uint32_t b, i, j;
      walk.at(t, b, i, j);
      const uint32_t row0 = i * kMmaRows + quarter * 32, row = row0 + lane;
      constexpr int kBlocks = BN / 32;
      const uint32_t c_first = j * BN;
      auto wanted = [&](int c) {
        const uint32_t col0 = c_first + 32 * c;
        return row0 < shape.m && col0 < shape.n && (!shape.sym || col0 >= row0);
      };
      int c = (int)group;
      while (c < kBlocks && !wanted(c)) c += 2;
      typename Epi::Pre pre{};
      if (c < kBlocks) pre = epi.load(row, c_first + 32 * c, b);
      const bool ok = mbar_wait(tfull + 8 * at, aphase, &gave_up);
      if (!__all_sync(0xFFFFFFFFu, ok)) break;
      tc_fence_after();
      while (c < kBlocks) {
        uint32_t acc[32];
        tmem_load32(acc, tmem + at * BN + 32 * c + (quarter << 21));
        int cn = c + 2;
        while (cn < kBlocks && !wanted(cn)) cn += 2;
        typename Epi::Pre nxt{};
        if (cn < kBlocks) nxt = epi.load(row, c_first + 32 * cn, b);
        tmem_load_wait();
        if (nk == 0) {   // an empty sum: nothing was written to the accumulator
#pragma unroll
          for (int q = 0; q < 32; ++q) acc[q] = 0;
        }
        epi.apply(pre, acc, row, c_first + 32 * c, b);
        pre = nxt;
        c = cn;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(tempty + 8 * at);
      if (++at == 2) {
        at = 0;
        aphase ^= 1;
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 2) tmem_free(tmem, T::kTmemCols);
  if (threadIdx.x == 0 && gave_up && shape.dev_status) atomicOr(shape.dev_status + DS_DEV_WORD_FLAGS, DS_DEV_MMA_TIMEOUT);
}

// ---- host side ------------------------------------------------------------------------------------------

// A map over `batch` matrices of `rows` rows of `cols` elements (2-byte floats or bytes), `ld` elements apart, read in
// boxes of box_cols x box_rows with 128-byte swizzle; entries outside read as zero.
cudaError_t make_tensor_map(CUtensorMap* map, int kind, const void* base, uint64_t cols, uint64_t rows, uint64_t batch, uint64_t ld,
                            uint64_t batch_stride, uint32_t box_cols, uint32_t box_rows);

int sm_count();

// The width of a tile that ends first: CTAs go through the tiles in rounds, and a round lasts as long as its tile is wide
// plus what a tile costs whatever its width (its first operands and the end of its epilogue, about 24 columns' worth).
inline int pick_bn(const MmaShape& s, int sms) {
  int best = 64;
  double least = 1e300;
  for (int bn : {256, 192, 128, 64}) {
    const TileWalk w(s, bn);
    const double rounds = (double)((w.total + sms - 1) / sms);
    // a tile narrower than 192 columns is held up by shared memory: 128 + bn rows are read for 128 x bn products
    const double width = bn >= 192 ? bn : (128 + bn) * 0.6;
    const double cost = rounds * (width + 24);
    if (cost < least * 0.999) {
      least = cost;
      best = bn;
    }
  }
  return best;
}

template <int KIND, int BN, bool B_ACROSS, class Epi>
cudaError_t launch_mma_bn(const CUtensorMap& a, const CUtensorMap& b, const MmaShape& s, const Epi& epi, cudaStream_t st) {
  const TileWalk w(s, BN);
  const uint32_t grid = w.total < (uint32_t)sm_count() ? w.total : (uint32_t)sm_count();
  if (!grid) return cudaSuccess;
  launch_pdl_smem(k_mma<KIND, BN, B_ACROSS, Epi>, dim3(grid), dim3(kMmaThreads), MmaTile<BN>::kSmem, st, a, b, s, epi);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace dsq
