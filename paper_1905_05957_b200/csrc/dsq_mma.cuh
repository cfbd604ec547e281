// Matrix products on the fifth-generation tensor cores (tcgen05), shared by the orthogonalised update (16-bit
// floating operands) and the 8-bit layer products: C = A B^T with A [M, K] and B [N, K], both laid out along K, or B
// given as [K, N] (16-bit only), or a symmetric operand of which half is there.
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

enum MmaKind : int { kMmaF16 = 0, kMmaI8 = 1, kMmaHalf = 2 };   // kMmaHalf: fp16 or bf16, which of the two the shape says

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
// Waits until the phase of the given parity has completed (a whole warp together).  False: another role gave up, or the limit ran out (which
// makes the others give up too).
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
  if (__all_sync(0xFFFFFFFFu, mbar_try(bar, parity))) return true;
  const long long t0 = clock64();
  while (true) {
    for (int i = 0; i < 16; ++i)
      if (__all_sync(0xFFFFFFFFu, mbar_try(bar, parity))) return true;
    if (__any_sync(0xFFFFFFFFu, *gave_up != 0)) return false;
    if (__any_sync(0xFFFFFFFFu, clock64() - t0 > kWaitCycles)) {
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
  if constexpr (KIND != kMmaI8)
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
// 32 bytes at once (a whole sector: a row's piece written 16 bytes at a time costs twice the transactions), 32-byte aligned.
__device__ __forceinline__ void ld_b32(uint32_t* w, const void* p) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void st_b32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
               "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
// Ends when the loads before have arrived.  The registers pass through it, so that nothing that uses them can be moved ahead.
__device__ __forceinline__ void tmem_load_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]),
                 "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                 "+r"(r[28]), "+r"(r[29])
               :
               : "memory");
  asm volatile("" : "+r"(r[30]), "+r"(r[31])::"memory");
}

// One lane of a converged warp.  The loops around TMA and matrix instructions are run by whole warps, whose loop values the
// compiler can then keep in the uniform registers that these instructions take, and only their issue by one lane: run by a
// single lane altogether, a step of K cost 520 cycles whatever the tile's width.
__device__ __forceinline__ bool elect_one() {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
  return ok != 0;
}

// Shared-memory descriptor of an operand tile whose rows are 128 bytes, swizzled by 128 bytes (atoms of 8 rows, 1024
// bytes).  Laid out along K: `stride` = bytes between groups of eight rows.  Laid out across K: `stride` = bytes between
// groups of eight k, `lead` = bytes between blocks of 64 columns.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead, uint32_t stride) {
  return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)((lead >> 4) & 0x3FFFu) << 16) | ((uint64_t)((stride >> 4) & 0x3FFFu) << 32) |
         (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: f16 x f16 -> f32, bf16 x bf16 -> f32 (kMmaHalf with `bf16`), or s8 x s8 -> s32; `rows` x `cols` of C; whether
// the operands lie across K.
template <int KIND>
__device__ __forceinline__ uint32_t mma_idesc(uint32_t rows, uint32_t cols, bool a_across, bool b_across, bool bf16) {
  uint32_t types = KIND != kMmaI8 ? (1u << 4) : ((2u << 4) | (1u << 7) | (1u << 10));
  if (KIND == kMmaHalf && bf16) types |= (1u << 7) | (1u << 10);
  return types | (a_across ? 1u << 15 : 0u) | (b_across ? 1u << 16 : 0u) | (cols >> 3 << 17) | (rows >> 4 << 24);
}
// The descriptor of instruction q (of four) of a step of 128 bytes of K.
__device__ __forceinline__ uint64_t step_desc(uint32_t tile, int q, bool across) {
  return across ? smem_desc(tile + 2048 * q, 64 * 128, 1024) : smem_desc(tile + 32 * q, 16, 1024);
}

// ---- the product ----------------------------------------------------------------------------------------

// How an operand lies in memory.  kSym: a symmetric matrix of which blocks of 128 x 128 or 256 x 256 on and above the diagonal are
// there (the diagonal ones whole): a piece below the diagonal is fetched from its mirror image and laid across K.  A tile's rows
// of such an operand lie within one block: blocks are 256 wide where pairs or tiles of 256 columns read them, else 128, which
// leaves less to compute below the diagonal.  (Writing the mirror images out instead cost 16 of 216 us of an update of twelve
// 768 x 768.)
enum MmaOperand : int { kAlong = 0, kAcross = 1, kSym = 2 };

struct MmaShape {
  uint32_t m, n, k;        // C is [m, n] per matrix of the batch
  uint32_t batch;
  uint32_t elem;           // bytes of an operand's element
  uint32_t sym;            // 7 or 8: C is symmetric; only its blocks of 2^sym on or above the diagonal go to the epilogue (0: all)
  uint32_t half;           // 7 or 8: blocks of 2^half of the kSym operands are there
  uint32_t* dev_status;
  uint32_t passes = 1;     // 2: C = A B2 + A B, B and B2 across K: K is gone through for B2 first, then for B
  uint32_t bf16 = 0;       // kMmaHalf: the operands are bf16, else fp16
};
// Step kb of all passes as a step of K, and whether it belongs to B2.
template <int B_MODE>
struct PassStep {
  uint32_t k;
  bool second;
  __device__ __forceinline__ PassStep(const MmaShape& s, uint32_t kb, uint32_t steps) : k(kb), second(false) {
    if (B_MODE == kAcross && s.passes > 1) {
      second = kb < steps;
      k = second ? kb : kb - steps;
    }
  }
};

// Fetches a step of an operand: ROWS rows by 128 bytes of K, or their mirror image, 64 columns at a time.
__device__ __forceinline__ bool mirrored(const MmaShape& s, uint32_t k, uint32_t row) { return k >> s.half < row >> s.half; }
template <int MODE, int ROWS>
__device__ __forceinline__ void load_operand(const MmaShape& s, uint32_t dst, const CUtensorMap* map, uint32_t k, uint32_t row, uint32_t b, uint32_t bar) {
  if constexpr (MODE == kAlong) {
    tma_load_3d(dst, map, (int)k, (int)row, (int)b, bar);
  } else {
    const bool across = MODE == kAcross || mirrored(s, k, row);
#pragma unroll
    for (int c = 0; c < ROWS; c += 64)
      tma_load_3d(dst + c * 128, map, (int)(across ? row + c : k), (int)(across ? k : row + c), (int)b, bar);
  }
}

// Epilogues.  A warp hands over blocks of 32 x 32 of C, a row to a lane:
//   struct Pre;  Pre load(row, col0, batch) const;   what it reads from global memory for its row (row may be out of range)
//   void apply(pre, acc, row, col0, batch) const;    acc: 32 raw accumulators of the row
// and, with kIn or kOut above 0, blocks of 32 x 32 halves that pass through shared memory: kIn of them are fetched by TMA, two
// blocks ahead, and kOut are stored by TMA.  A row read or written straight from a lane touches 32 lines an instruction; that
// alone was most of the epilogue of X = a X + B X (1536 x 4608 x 512: 17.6 us, 7.1 without reads and writes).
//   const CUtensorMap* in(i) const;  const CUtensorMap* out(i) const;     (NULL where nothing is read or stored)
//   void apply(pre, acc, row, col0, batch, smem) const;                   smem: this lane's row of the first block (see row_chunk)
constexpr uint32_t kBlockBytes = 2048;     // 32 rows of 64 bytes, 64-byte swizzle
// The 16-byte piece q of a lane's row: pieces are exchanged within a row by the row's number, as TMA lays them.
__device__ __forceinline__ uint32_t row_chunk(uint32_t block, int lane, int q) { return block + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4); }

template <class Epi>
struct Staged {
  static constexpr int kBlocks = Epi::kIn > Epi::kOut ? Epi::kIn : Epi::kOut;
  static constexpr uint32_t kSlot = kBlocks * kBlockBytes;      // a warp has two
  static constexpr uint32_t kBytes = 8 * 2 * kSlot;
};

template <int BN, class Epi>
struct MmaTile {
  static constexpr int kStageBytes = (kMmaRows + BN) * 128;
  static constexpr int kFit = (int)((225 * 1024 - Staged<Epi>::kBytes) / kStageBytes);
  static constexpr int kStages = kFit < 10 ? kFit : 10;
  static constexpr int kTmemCols = BN == 192 ? 512 : 2 * BN;
  static constexpr uint32_t kRing = kStages * kStageBytes;
  static constexpr size_t kSmem = kRing + Staged<Epi>::kBytes + 1024;
};

__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src)
               : "memory");
}

// The epilogue of one warp: its two slots of shared memory, and the barriers on which their loads arrive.
template <class Epi>
struct EpilogueWarp {
  uint32_t slots, bars;      // addresses
  uint32_t slot = 0, phases = 0;
  int lane;
  volatile int* gave_up;

  __device__ __forceinline__ uint32_t at(uint32_t which) const { return slots + which * Staged<Epi>::kSlot; }
  static __device__ __forceinline__ bool reads(const Epi& epi) {
    if constexpr (Epi::kIn > 0) return epi.in(0) != nullptr;
    return false;
  }
  __device__ __forceinline__ void fetch(const Epi& epi, uint32_t which, uint32_t row0, uint32_t col0, uint32_t b) {
    if constexpr (Epi::kIn > 0) {
      if (!epi.in(0)) return;
      if (lane == 0) {
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");    // what this slot last held has left it
        mbar_expect_tx(bars + 8 * which, Epi::kIn * kBlockBytes);
#pragma unroll
        for (int i = 0; i < Epi::kIn; ++i) tma_load_3d(at(which) + i * kBlockBytes, epi.in(i), (int)col0, (int)row0, (int)b, bars + 8 * which);
      }
      __syncwarp();
    }
  }
  // One block.  False: a wait ran out.
  template <class LoadNext>
  __device__ __forceinline__ bool block(const Epi& epi, const typename Epi::Pre& pre, uint32_t tmem_addr, bool empty, uint32_t row0, uint32_t col0,
                                        uint32_t b, LoadNext&& load_next) {
    uint32_t acc[32];
    tmem_load32(acc, tmem_addr);
    load_next();
    tmem_load_wait(acc);
    if (empty) {      // an empty sum: nothing was written to the accumulator
#pragma unroll
      for (int q = 0; q < 32; ++q) acc[q] = 0;
    }
    return finish(epi, pre, acc, row0, col0, b);
  }
  __device__ __forceinline__ bool finish(const Epi& epi, const typename Epi::Pre& pre, const uint32_t (&acc)[32], uint32_t row0, uint32_t col0, uint32_t b) {
    if (Epi::kIn > 0 && reads(epi)) {
      if (!mbar_wait(bars + 8 * slot, (phases >> slot) & 1, gave_up)) return false;
      phases ^= 1u << slot;
    } else if constexpr (Epi::kOut > 0) {
      if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
      __syncwarp();
    }
    if constexpr (Epi::kIn + Epi::kOut > 0) {
      epi.apply(pre, acc, row0 + lane, col0, b, at(slot), lane);
      if constexpr (Epi::kOut > 0) {
        if (epi.out(0)) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
#pragma unroll
            for (int i = 0; i < Epi::kOut; ++i) tma_store_3d(epi.out(i), (int)col0, (int)row0, (int)b, at(slot) + i * kBlockBytes);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        }
      }
      __syncwarp();
      slot ^= 1;
    } else {
      epi.apply(pre, acc, row0 + lane, col0, b);
    }
    return true;
  }
  __device__ __forceinline__ void drain() const {      // stores have been made
    if constexpr (Epi::kOut > 0) {
      if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
      __syncwarp();
    }
  }
  // What is still on its way into this warp's slots when it gives up lands first (`fetched`: loads asked for and not waited for).
  __device__ __forceinline__ void abandon(const Epi& epi, int fetched) {
    if (Epi::kIn > 0 && reads(epi)) {
      for (int i = 0; i < fetched; ++i) {
        const uint32_t which = (slot + i) & 1;
        const long long t0 = clock64();
        while (!mbar_try(bars + 8 * which, (phases >> which) & 1) && clock64() - t0 < kWaitCycles) {
        }
      }
    }
  }
  // All blocks of this warp's part of a tile.  `ready` waits for the accumulator.
  template <class Wanted, class Ready>
  __device__ __forceinline__ bool tile(const Epi& epi, int group, int blocks, uint32_t row0, uint32_t col, uint32_t b, uint32_t tmem_at, bool empty,
                                       Wanted&& wanted, Ready&& ready) {
    auto next = [&](int c) {
      c += 2;
      while (c < blocks && !wanted(c)) c += 2;
      return c;
    };
    int c = next(group - 2), cn = next(c);
    typename Epi::Pre pre{};
    if (c < blocks) {
      fetch(epi, slot, row0, col + 32 * c, b);
      pre = epi.load(row0 + lane, col + 32 * c, b);
    }
    if (cn < blocks) fetch(epi, slot ^ 1, row0, col + 32 * cn, b);
    if (!ready()) {
      abandon(epi, (c < blocks) + (cn < blocks));
      return false;
    }
    tc_fence_after();
    while (c < blocks) {
      const int nn = next(cn);
      const uint32_t used = slot;
      typename Epi::Pre after{};
      if (!block(epi, pre, tmem_at + 32 * c, empty, row0, col + 32 * c, b,
                 [&] { if (cn < blocks) after = epi.load(row0 + lane, col + 32 * cn, b); })) {
        abandon(epi, 1 + (cn < blocks));
        return false;
      }
      if (nn < blocks) fetch(epi, used, row0, col + 32 * nn, b);
      pre = after;
      c = cn;
      cn = nn;
    }
    return true;
  }
};

// Tiles of C in the order in which CTAs take them.
struct TileWalk {
  uint32_t mt, nt, per, total, sym, bn;
  __host__ __device__ TileWalk(const MmaShape& s, uint32_t bn_) : sym(s.sym), bn(bn_) {
    mt = (s.m + kMmaRows - 1) / kMmaRows;
    nt = (s.n + bn - 1) / bn;
    if (sym) {
      per = 0;
      for (uint32_t i = 0; i < mt; ++i) per += nt - first(i);
    } else {
      per = mt * nt;
    }
    total = per * s.batch;
  }
  // the first tile of tile row i that is wanted
  __host__ __device__ uint32_t first(uint32_t i) const { return (i * kMmaRows >> sym << sym) / bn; }
  __host__ __device__ void at(uint32_t t, uint32_t& b, uint32_t& i, uint32_t& j) const {
    b = t / per;
    t -= b * per;
    if (sym) {
      i = 0;
      while (true) {
        const uint32_t f = first(i), c = nt - f;
        if (t < c) {
          j = f + t;
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

template <int KIND, int BN, int A_MODE, int B_MODE, class Epi>
__global__ void __launch_bounds__(kMmaThreads, 1)
    k_mma(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_b2, const MmaShape shape,
          const __grid_constant__ Epi epi) {
  using T = MmaTile<BN, Epi>;
  constexpr int kBK = KIND != kMmaI8 ? 64 : 128;    // elements of K per stage: 128 bytes
  extern __shared__ uint8_t dyn[];
  __shared__ uint64_t bars[2 * T::kStages + 5 + 16];
  __shared__ uint32_t tmem_slot;
  __shared__ int gave_up;
  const uint32_t ring = (smem_u32(dyn) + 1023u) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * T::kStages, tfull = empty + 8 * T::kStages, tempty = tfull + 16,
                 drain = tempty + 16, staged = drain + 8;
  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    tma_prefetch_map(&map_a);
    tma_prefetch_map(&map_b);
    if (B_MODE == kAcross && shape.passes > 1) tma_prefetch_map(&map_b2);
    for (int i = 0; i < T::kStages; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull + 8 * i, 1);
      mbar_init(tempty + 8 * i, 8);
    }
    mbar_init(drain, 1);
    for (int i = 0; i < 16; ++i) mbar_init(staged + 8 * i, 1);
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 2) tmem_alloc(smem_u32(&tmem_slot), T::kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, tmem_slot, 0);
  // Only now may the next kernel's CTAs come in: one that took this SM's tensor memory before this CTA had its share would
  // wait for this kernel while this kernel waits for it.
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("fence.proxy.async.global;" ::: "memory");   // what earlier kernels stored is about to be read by TMA

  const TileWalk walk(shape, BN);
  const uint32_t steps = (shape.k + kBK - 1) / kBK, nk = B_MODE == kAcross ? steps * shape.passes : steps;

  if (warp == 0) {
    const bool one = elect_one();
    uint32_t stage = 0, phase = 0, issued = 0;
    bool ok = true;
    for (uint32_t t = blockIdx.x; ok && t < walk.total; t += gridDim.x) {
      uint32_t b, i, j;
      walk.at(t, b, i, j);
      for (uint32_t kb = 0; kb < nk; ++kb) {
        if (!(ok = mbar_wait(empty + 8 * stage, phase ^ 1, &gave_up))) break;
        const uint32_t dst = ring + stage * T::kStageBytes;
        if (one) {
          mbar_expect_tx(full + 8 * stage, T::kStageBytes);
          const PassStep<B_MODE> at(shape, kb, steps);
          load_operand<A_MODE, kMmaRows>(shape, dst, &map_a, at.k * kBK, i * kMmaRows, b, full + 8 * stage);
          load_operand<B_MODE, BN>(shape, dst + kMmaRows * 128, at.second ? &map_b2 : &map_b, at.k * kBK, j * BN, b, full + 8 * stage);
        }
        __syncwarp();
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
  } else if (warp == 1) {
    const bool one = elect_one();
    uint32_t stage = 0, phase = 0, at = 0, aphase = 0;
    bool ok = true;
    for (uint32_t t = blockIdx.x; ok && t < walk.total; t += gridDim.x) {
      uint32_t b = 0, i = 0, j = 0;
      if constexpr (A_MODE == kSym || B_MODE == kSym) walk.at(t, b, i, j);
      if (!(ok = mbar_wait(tempty + 8 * at, aphase ^ 1, &gave_up))) break;
      tc_fence_after();
      const uint32_t d = tmem + at * BN;
      for (uint32_t kb = 0; kb < nk; ++kb) {
        if (!(ok = mbar_wait(full + 8 * stage, phase, &gave_up))) break;
        tc_fence_after();
        if (one) {
          const uint32_t sa = ring + stage * T::kStageBytes, sb = sa + kMmaRows * 128;
          const uint32_t k0 = PassStep<B_MODE>(shape, kb, steps).k * kBK;
          const bool ta = A_MODE == kAcross || (A_MODE == kSym && mirrored(shape, k0, i * kMmaRows)), tb = B_MODE == kAcross || (B_MODE == kSym && mirrored(shape, k0, j * BN));
          const uint32_t idesc = mma_idesc<KIND>(kMmaRows, BN, ta, tb, shape.bf16);
#pragma unroll
          for (int q = 0; q < 4; ++q)   // four instructions of 32 bytes of K
            tc_mma<KIND>(d, step_desc(sa, q, ta), step_desc(sb, q, tb), idesc, (kb | q) != 0);
          tc_commit(empty + 8 * stage);
        }
        __syncwarp();
        if (++stage == T::kStages) {
          stage = 0;
          phase ^= 1;
        }
      }
      if (!ok) break;
      if (one) tc_commit(tfull + 8 * at);
      __syncwarp();
      if (++at == 2) {
        at = 0;
        aphase ^= 1;
      }
    }
    if (!ok) {   // products in flight must have ended before the tensor memory is freed
      if (one) tc_commit(drain);
      const long long t0 = clock64();
      while (!mbar_try(drain, 0) && clock64() - t0 < kWaitCycles) {
      }
    }
  } else if (warp >= 4) {
    // two groups of four warps; a warp reads the 32 lanes that its rank in the group names
    const uint32_t quarter = warp & 3, group = (warp - 4) >> 2;
    EpilogueWarp<Epi> ew{ring + T::kRing + (warp - 4) * 2 * Staged<Epi>::kSlot, staged + 16 * (warp - 4), 0, 0, lane, &gave_up};
    uint32_t at = 0, aphase = 0;
    for (uint32_t t = blockIdx.x; t < walk.total; t += gridDim.x) {
      uint32_t b, i, j;
      walk.at(t, b, i, j);
      const uint32_t row0 = i * kMmaRows + quarter * 32, col = j * BN;
      auto wanted = [&](int c) {
        const uint32_t col0 = col + 32 * c;
        return row0 < shape.m && col0 < shape.n && (!shape.sym || col0 >> shape.sym >= row0 >> shape.sym);
      };
      if (!ew.tile(epi, (int)group, BN / 32, row0, col, b, tmem + at * BN + (quarter << 21), nk == 0, wanted,
                   [&] { return mbar_wait(tfull + 8 * at, aphase, &gave_up); }))
        break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(tempty + 8 * at);
      if (++at == 2) {
        at = 0;
        aphase ^= 1;
      }
    }
    ew.drain();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 2) tmem_free(tmem, T::kTmemCols);
  if (threadIdx.x == 0 && gave_up && shape.dev_status) atomicOr(shape.dev_status + DS_DEV_WORD_FLAGS, DS_DEV_MMA_TIMEOUT);
}

// ---- the same product by pairs of CTAs ----
// Two CTAs of a cluster work on one 256 x 256 tile (cta_group::2): each fetches 128 rows of A and half of B's rows, each
// tensor core reads both halves of B, and each CTA keeps the accumulator of its own 128 rows.  Per product that is two thirds of
// the shared-memory and L2 traffic of a 128 x 256 tile of one CTA, which is what bounds large products (a 4096^3 product:
// 118 us by single CTAs, 100 by pairs).  The first CTA of the pair issues all matrix instructions.
//
// An item of work is a tile or half of one (256 x 128): the tiles left over after whole rounds are halved where both halves
// of all of them fit into one round.
struct PairWalk {
  uint32_t mt, nt, per, total, whole, items, sym;
  __host__ __device__ PairWalk(const MmaShape& s, uint32_t pairs) : sym(s.sym) {
    mt = (s.m + 255) / 256;
    nt = (s.n + 255) / 256;
    per = sym ? mt * (mt + 1) / 2 : mt * nt;
    total = per * s.batch;
    const uint32_t rest = total % pairs;
    whole = 2 * rest <= pairs ? total - rest : total;
    items = whole + 2 * (total - whole);
  }
  // item -> matrix b, first row of the tile, first column and width of the item
  __host__ __device__ void at(uint32_t t, uint32_t& b, uint32_t& row, uint32_t& col, uint32_t& width) const {
    uint32_t half = 0;
    width = 256;
    if (t >= whole) {
      half = (t - whole) & 1;
      t = whole + ((t - whole) >> 1);
      width = 128;
    }
    b = t / per;
    t -= b * per;
    uint32_t i, j;
    if (sym) {   // columns of the upper triangle one after the other: column j holds the tiles 0..j
      j = (uint32_t)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
      while (j * (j + 1) / 2 > t) --j;
      while ((j + 1) * (j + 2) / 2 <= t) ++j;
      i = t - j * (j + 1) / 2;
    } else {
      const uint32_t band = 4 * nt, g = t / band, r = t - g * band;
      const uint32_t h = mt - 4 * g < 4 ? mt - 4 * g : 4;
      j = r / h;
      i = 4 * g + r - j * h;
    }
    row = i * 256;
    col = j * 256 + half * 128;
  }
};

constexpr int kPairStageBytes = 2 * kMmaRows * 128;   // per CTA: 128 rows of A, 128 of B
template <class Epi>
struct PairTile {
  static constexpr int kStages = (int)((225 * 1024 - Staged<Epi>::kBytes) / kPairStageBytes);
  static constexpr uint32_t kRing = kStages * kPairStageBytes;
  static constexpr size_t kSmem = kRing + Staged<Epi>::kBytes + 1024;
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {   // the same place in a CTA of the cluster
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tc_commit_pair(uint32_t bar) {   // arrives at this place in both CTAs
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
               : "memory");
}
template <int KIND>
__device__ __forceinline__ void tc_mma_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  if constexpr (KIND != kMmaI8)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

template <int KIND, int A_MODE, int B_MODE, class Epi>
__global__ void __launch_bounds__(kMmaThreads, 1) __cluster_dims__(2, 1, 1)
    k_mma_pair(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_b2, const MmaShape shape,
               const __grid_constant__ Epi epi) {
  constexpr int kPairStages = PairTile<Epi>::kStages;
  constexpr int kBK = KIND != kMmaI8 ? 64 : 128;
  extern __shared__ uint8_t dyn[];
  __shared__ uint64_t bars[2 * kPairStages + 5 + 16];
  __shared__ uint32_t tmem_slot;
  __shared__ int gave_up;
  const uint32_t ring = (smem_u32(dyn) + 1023u) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * kPairStages, tfull = empty + 8 * kPairStages, tempty = tfull + 16,
                 drain = tempty + 16, staged = drain + 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();

  if (threadIdx.x == 0) {
    tma_prefetch_map(&map_a);
    tma_prefetch_map(&map_b);
    if (B_MODE == kAcross && shape.passes > 1) tma_prefetch_map(&map_b2);
    for (int i = 0; i < kPairStages; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull + 8 * i, 1);
      mbar_init(tempty + 8 * i, 16);   // the epilogue warps of both CTAs
    }
    mbar_init(drain, 1);
    for (int i = 0; i < 16; ++i) mbar_init(staged + 8 * i, 1);
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  tc_fence_before();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, tmem_slot, 0);
  asm volatile("griddepcontrol.launch_dependents;");   // after the allocation, as above
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("fence.proxy.async.global;" ::: "memory");   // what earlier kernels stored is about to be read by TMA

  const uint32_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const PairWalk walk(shape, pairs);
  const uint32_t steps = (shape.k + kBK - 1) / kBK, nk = B_MODE == kAcross ? steps * shape.passes : steps;
  // an item of which nothing is wanted (outside C, or below the diagonal): every role passes over it
  auto skip = [&](uint32_t row, uint32_t col, uint32_t width) { return col >= shape.n || (shape.sym && col + width <= row); };

  if (warp == 0) {
    const bool one = elect_one();
    uint32_t stage = 0, phase = 0, issued = 0;
    bool ok = true;
    for (uint32_t t = pair; ok && t < walk.items; t += pairs) {
      uint32_t b, row, col, width;
      walk.at(t, b, row, col, width);
      if (skip(row, col, width)) continue;
      const uint32_t mine = width / 2;                 // rows of B that this CTA fetches
      for (uint32_t kb = 0; kb < nk; ++kb) {
        if (!(ok = mbar_wait(empty + 8 * stage, phase ^ 1, &gave_up))) break;
        const uint32_t dst = ring + stage * kPairStageBytes, bar = in_cta(full + 8 * stage, 0);
        if (one) {
          if (rank == 0) mbar_expect_tx(full + 8 * stage, 2 * (kMmaRows + mine) * 128);
          const PassStep<B_MODE> at(shape, kb, steps);
          const uint32_t k0 = at.k * kBK, r0 = row + rank * kMmaRows, n0 = col + rank * mine;
          if constexpr (A_MODE == kAlong) {
            tma_load_3d_pair(dst, &map_a, (int)k0, (int)r0, (int)b, bar);
          } else {
            const bool across = A_MODE == kAcross || mirrored(shape, k0, row);
#pragma unroll
            for (uint32_t c = 0; c < kMmaRows; c += 64)
              tma_load_3d_pair(dst + c * 128, &map_a, (int)(across ? r0 + c : k0), (int)(across ? k0 : r0 + c), (int)b, bar);
          }
          const bool across = B_MODE == kAcross || (B_MODE == kSym && mirrored(shape, k0, col));
          for (uint32_t c = 0; c < mine; c += 64)
            tma_load_3d_pair(dst + (kMmaRows + c) * 128, at.second ? &map_b2 : &map_b, (int)(across ? n0 + c : k0), (int)(across ? k0 : n0 + c), (int)b, bar);
        }
        __syncwarp();
        ++issued;
        if (++stage == kPairStages) {
          stage = 0;
          phase ^= 1;
        }
      }
    }
    if (!ok && rank == 0) {   // copies in flight land before shared memory is given away (their bytes count in this CTA)
      const uint32_t last = issued < (uint32_t)kPairStages ? issued : (uint32_t)kPairStages;
      for (uint32_t q = 0; q < last; ++q) {
        stage = stage ? stage - 1 : kPairStages - 1;
        const uint32_t use = (issued - 1 - q) / kPairStages;
        const long long t0 = clock64();
        while (!mbar_try(full + 8 * stage, use & 1) && clock64() - t0 < kWaitCycles) {
        }
      }
    }
  } else if (warp == 1 && rank == 0) {
    const bool one = elect_one();
    uint32_t stage = 0, phase = 0, at = 0, aphase = 0;
    bool ok = true;
    for (uint32_t t = pair; ok && t < walk.items; t += pairs) {
      uint32_t b, row, col, width;
      walk.at(t, b, row, col, width);
      if (skip(row, col, width)) continue;
      if (!(ok = mbar_wait(tempty + 8 * at, aphase ^ 1, &gave_up))) break;
      tc_fence_after();
      const uint32_t d = tmem + at * 256;
      for (uint32_t kb = 0; kb < nk; ++kb) {
        if (!(ok = mbar_wait(full + 8 * stage, phase, &gave_up))) break;
        tc_fence_after();
        if (one) {
          const uint32_t sa = ring + stage * kPairStageBytes, sb = sa + kMmaRows * 128;
          const uint32_t k0 = PassStep<B_MODE>(shape, kb, steps).k * kBK;
          const bool ta = A_MODE == kAcross || (A_MODE == kSym && mirrored(shape, k0, row)), tb = B_MODE == kAcross || (B_MODE == kSym && mirrored(shape, k0, col));
          const uint32_t idesc = mma_idesc<KIND>(2 * kMmaRows, width, ta, tb, shape.bf16);
#pragma unroll
          for (int q = 0; q < 4; ++q) tc_mma_pair<KIND>(d, step_desc(sa, q, ta), step_desc(sb, q, tb), idesc, (kb | q) != 0);
          tc_commit_pair(empty + 8 * stage);
        }
        __syncwarp();
        if (++stage == kPairStages) {
          stage = 0;
          phase ^= 1;
        }
      }
      if (!ok) break;
      if (one) tc_commit_pair(tfull + 8 * at);
      __syncwarp();
      if (++at == 2) {
        at = 0;
        aphase ^= 1;
      }
    }
    if (!ok) {
      if (one) tc_commit_pair(drain);
      const long long t0 = clock64();
      while (!mbar_try(drain, 0) && clock64() - t0 < kWaitCycles) {
      }
    }
  } else if (warp >= 4) {
    const uint32_t quarter = warp & 3, group = (warp - 4) >> 2;
    EpilogueWarp<Epi> ew{ring + PairTile<Epi>::kRing + (warp - 4) * 2 * Staged<Epi>::kSlot, staged + 16 * (warp - 4), 0, 0, lane, &gave_up};
    uint32_t at = 0, aphase = 0;
    for (uint32_t t = pair; t < walk.items; t += pairs) {
      uint32_t b, row_t, col, width;
      walk.at(t, b, row_t, col, width);
      if (skip(row_t, col, width)) continue;
      const uint32_t row0 = row_t + rank * kMmaRows + quarter * 32;
      auto wanted = [&](int c) {
        const uint32_t col0 = col + 32 * c;
        return row0 < shape.m && col0 < shape.n && (!shape.sym || col0 >> shape.sym >= row0 >> shape.sym);
      };
      if (!ew.tile(epi, (int)group, (int)(width >> 5), row0, col, b, tmem + at * 256 + (quarter << 21), false, wanted,
                   [&] { return mbar_wait(tfull + 8 * at, aphase, &gave_up); }))
        break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(in_cta(tempty + 8 * at, 0));
      if (++at == 2) {
        at = 0;
        aphase ^= 1;
      }
    }
    ew.drain();
  }
  __syncwarp();
  tc_fence_before();
  cluster_sync();   // the other CTA's arrivals and commits name this CTA's shared memory until here
  tc_fence_after();
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
  if (threadIdx.x == 0 && gave_up && shape.dev_status) atomicOr(shape.dev_status + DS_DEV_WORD_FLAGS, DS_DEV_MMA_TIMEOUT);
}

// ---- a long K and few tiles: one tile by a cluster, K split over its CTAs ----
// Each CTA of the cluster sums its share of K; then every 32 x 32 block of the tile gets an owner, the other CTAs write their
// sums of it into the owner's shared memory (the ring, which is idle by then), and the owner adds them in the order of the
// CTAs' ranks, so that results do not depend on timing.  512 x 512 x 4608 by single CTAs: 15.5 us of which 12 are the 72 steps
// of K in a row; on a third of the SMs.
template <int KIND, int BN, int A_MODE, int B_MODE, class Epi>
__global__ void __launch_bounds__(kMmaThreads, 1)
    k_mma_split(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_b2, const MmaShape shape,
                const __grid_constant__ Epi epi,
                const uint32_t parts) {
  using T = MmaTile<BN, Epi>;
  constexpr int kBK = KIND != kMmaI8 ? 64 : 128;
  constexpr int kTmem = BN < 32 ? 32 : BN == 192 ? 256 : BN;
  constexpr int kBlocks = BN / 32;
  extern __shared__ uint8_t dyn[];
  __shared__ uint64_t bars[2 * T::kStages + 1 + 16];
  __shared__ uint32_t tmem_slot;
  __shared__ int gave_up;
  const uint32_t ring = (smem_u32(dyn) + 1023u) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * T::kStages, done = empty + 8 * T::kStages,
                 staged = done + 8;
  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();

  if (threadIdx.x == 0) {
    tma_prefetch_map(&map_a);
    tma_prefetch_map(&map_b);
    if (B_MODE == kAcross && shape.passes > 1) tma_prefetch_map(&map_b2);
    for (int i = 0; i < T::kStages; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    mbar_init(done, 1);
    for (int i = 0; i < 16; ++i) mbar_init(staged + 8 * i, 1);
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 2) tmem_alloc(smem_u32(&tmem_slot), kTmem);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, tmem_slot, 0);
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("fence.proxy.async.global;" ::: "memory");   // what earlier kernels stored is about to be read by TMA

  const TileWalk walk(shape, BN);
  uint32_t b, ti, tj;
  walk.at(blockIdx.x / parts, b, ti, tj);
  const uint32_t steps = (shape.k + kBK - 1) / kBK, nk_all = B_MODE == kAcross ? steps * shape.passes : steps, share = (nk_all + parts - 1) / parts;
  const uint32_t k_first = min(rank * share, nk_all), nk = min(share, nk_all - k_first);

  const uint32_t quarter = warp & 3, group = (warp - 4) >> 2;   // epilogue warps
  const uint32_t row0 = ti * kMmaRows + quarter * 32, c_first = tj * BN;
  auto wanted = [&](int c) {
    const uint32_t col0 = c_first + 32 * c;
    return row0 < shape.m && col0 < shape.n && (!shape.sym || col0 >> shape.sym >= row0 >> shape.sym);
  };
  auto owner = [&](int c) { return (uint32_t)(c * 4 + quarter) % parts; };
  // where in an owner's ring the sums of block (c, quarter) from CTA r lie: 4 KB
  auto slot = [&](int c, uint32_t r) { return ring + (((c * 4 + quarter) / parts) * parts + r) * 4096u; };

  if (warp == 0) {
    const bool one = elect_one();
    uint32_t stage = 0, phase = 0, issued = 0;
    bool ok = true;
    for (uint32_t kb = k_first; kb < k_first + nk; ++kb) {
      if (!(ok = mbar_wait(empty + 8 * stage, phase ^ 1, &gave_up))) break;
      const uint32_t dst = ring + stage * T::kStageBytes;
      if (one) {
        mbar_expect_tx(full + 8 * stage, T::kStageBytes);
        const PassStep<B_MODE> at(shape, kb, steps);
        load_operand<A_MODE, kMmaRows>(shape, dst, &map_a, at.k * kBK, ti * kMmaRows, b, full + 8 * stage);
        load_operand<B_MODE, BN>(shape, dst + kMmaRows * 128, at.second ? &map_b2 : &map_b, at.k * kBK, c_first, b, full + 8 * stage);
      }
      __syncwarp();
      ++issued;
      if (++stage == T::kStages) {
        stage = 0;
        phase ^= 1;
      }
    }
    if (!ok) {
      const uint32_t last = issued < (uint32_t)T::kStages ? issued : (uint32_t)T::kStages;
      for (uint32_t q = 0; q < last; ++q) {
        stage = stage ? stage - 1 : T::kStages - 1;
        const uint32_t use = (issued - 1 - q) / T::kStages;
        const long long t0 = clock64();
        while (!mbar_try(full + 8 * stage, use & 1) && clock64() - t0 < kWaitCycles) {
        }
      }
    }
  } else if (warp == 1) {
    const bool one = elect_one();
    uint32_t stage = 0, phase = 0;
    for (uint32_t kb = 0; kb < nk; ++kb) {
      if (!mbar_wait(full + 8 * stage, phase, &gave_up)) break;
      tc_fence_after();
      if (one) {
        const uint32_t sa = ring + stage * T::kStageBytes, sb = sa + kMmaRows * 128, k0 = PassStep<B_MODE>(shape, k_first + kb, steps).k * kBK;
        const bool ta = A_MODE == kAcross || (A_MODE == kSym && mirrored(shape, k0, ti * kMmaRows)), tb = B_MODE == kAcross || (B_MODE == kSym && mirrored(shape, k0, c_first));
        const uint32_t idesc = mma_idesc<KIND>(kMmaRows, BN, ta, tb, shape.bf16);
#pragma unroll
        for (int q = 0; q < 4; ++q) tc_mma<KIND>(tmem, step_desc(sa, q, ta), step_desc(sb, q, tb), idesc, (kb | q) != 0);
        tc_commit(empty + 8 * stage);
      }
      __syncwarp();
      if (++stage == T::kStages) {
        stage = 0;
        phase ^= 1;
      }
    }
    if (one) tc_commit(done);   // after a wait that ran out, too: it tells that the products in flight have ended
    __syncwarp();
  }
  // every role: this CTA's products have ended, its ring is idle
  (void)mbar_wait(done, 0, &gave_up);
  tc_fence_after();
  cluster_sync();
  if (warp >= 4) {
    for (int c = (int)group; c < kBlocks; c += 2) {
      if (!wanted(c) || owner(c) == rank) continue;
      uint32_t acc[32];
      tmem_load32(acc, tmem + 32 * c + (quarter << 21));
      tmem_load_wait(acc);
      const uint32_t to = in_cta(slot(c, rank), owner(c)) + lane * 16;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + 512 * j), "r"(nk ? acc[4 * j] : 0u),
                     "r"(nk ? acc[4 * j + 1] : 0u), "r"(nk ? acc[4 * j + 2] : 0u), "r"(nk ? acc[4 * j + 3] : 0u)
                     : "memory");
    }
  }
  __syncwarp();
  cluster_sync();
  if (warp >= 4) {
    EpilogueWarp<Epi> ew{ring + T::kRing + (warp - 4) * 2 * Staged<Epi>::kSlot, staged + 16 * (warp - 4), 0, 0, lane, &gave_up};
    for (int c = (int)group; c < kBlocks; c += 2) {
      if (!wanted(c) || owner(c) != rank) continue;
      ew.fetch(epi, ew.slot, row0, c_first + 32 * c, b);
      const typename Epi::Pre pre = epi.load(row0 + lane, c_first + 32 * c, b);
      uint32_t acc[32], own[32];
      tmem_load32(own, tmem + 32 * c + (quarter << 21));
      tmem_load_wait(own);
#pragma unroll
      for (int j = 0; j < 32; ++j) acc[j] = 0;
      for (uint32_t r = 0; r < parts; ++r) {
        const uint32_t from = slot(c, r) + lane * 16;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint32_t v[4];
          if (r != rank)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(from + 512 * j) : "memory");
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = r != rank ? v[i] : nk ? own[4 * j + i] : 0u;
            if constexpr (KIND == kMmaI8)
              acc[4 * j + i] += x;
            else
              acc[4 * j + i] = __float_as_uint(__fadd_rn(__uint_as_float(acc[4 * j + i]), __uint_as_float(x)));
          }
        }
      }
      if (!ew.finish(epi, pre, acc, row0, c_first + 32 * c, b)) {
        ew.abandon(epi, 1);
        break;
      }
    }
    ew.drain();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 2) tmem_free(tmem, kTmem);
  if (threadIdx.x == 0 && gave_up && shape.dev_status) atomicOr(shape.dev_status + DS_DEV_WORD_FLAGS, DS_DEV_MMA_TIMEOUT);
}

// ---- host side ------------------------------------------------------------------------------------------

// A map over `batch` matrices of `rows` rows of `cols` elements (2-byte floats or bytes), `ld` elements apart, read in
// boxes of box_cols x box_rows with 128-byte swizzle (blocks of an epilogue, 64 bytes wide: 64-byte swizzle); entries outside
// read as zero and are not written.
cudaError_t make_tensor_map(CUtensorMap* map, int kind, const void* base, uint64_t cols, uint64_t rows, uint64_t batch, uint64_t ld,
                            uint64_t batch_stride, uint32_t box_cols, uint32_t box_rows, bool block = false);

int sm_count();

// Clusters of `size` (2, 4 or 8) such CTAs that run at once on this device (a cluster stays within a part of the device, which
// may leave SMs over).
int cluster_count(uint32_t size);
inline int pair_count() { return cluster_count(2); }

// How a product is taken.
struct MmaPlan {
  bool pair;
  int bn;             // width of a tile (single CTAs and clusters)
  uint32_t parts;     // CTAs that share a tile's K: 1, or a cluster of 2, 4 or 8
  uint32_t box_rows() const { return pair ? 64 : (uint32_t)bn; }   // rows of a box of B
};

// Which form ends first, from times measured on a B200 in us: `steps` of 128 bytes of K; what a launch costs whatever its size
// (single CTAs 4, pairs 6, clusters that split K 8); a tile's step by its width, with few SMs busy and with all of them (when
// L2 and power bound it); a tile's epilogue, which the next tile's products hide.  Measured and modelled, 16-bit operands:
//   4096^3: 64 columns 162 / 165, 128 116 / 127, 192 107 / 114, 256 116 / 118, pairs 98 / 98
//   2048^3: 38 / 29, 25 / 24, 30 / 28, 22 / 22, 24 / 23;   1024^3: 8.5 / 8.2, 9.9 / 9.0, 11.7 / 11, 14 / 13, 12 / 11
constexpr double kTileEpilogue = 1.0;      // per 64 columns
inline double step_time(int bn, double busy) {
  const double few = bn == 256 ? 0.30 : bn == 192 ? 0.25 : bn == 128 ? 0.18 : 0.16;
  const double all = bn == 256 ? 0.43 : bn == 192 ? 0.335 : bn == 128 ? 0.27 : 0.18;
  return busy >= 1 ? all : busy <= 0.4 ? few : few + (all - few) * (busy - 0.4) / 0.6;
}
inline double rounds_time(double rounds, double main, double epilogue) {
  return rounds <= 0 ? 0 : main + (rounds - 1) * (main > epilogue ? main : epilogue) + epilogue;
}
inline double k_steps(const MmaShape& s) { return s.passes * (s.k * (double)s.elem / 128); }
inline double single_time(const MmaShape& s, int sms, int bn) {
  const TileWalk w(s, bn);
  return 4 + rounds_time((double)((w.total + sms - 1) / sms), step_time(bn, (double)w.total / sms) * k_steps(s),
                         kTileEpilogue * bn / 64);
}
inline double split_time(const MmaShape& s, int sms, int bn, uint32_t parts) {
  const TileWalk w(s, bn);
  if (w.total > (uint32_t)cluster_count(parts) || bn > 128) return 1e300;   // one round: a CTA keeps one tile
  return 8 + step_time(bn, (double)w.total * parts / sms) * k_steps(s) / parts + kTileEpilogue * bn / 64;
}
inline double pair_time(const MmaShape& s, int pairs) {
  const PairWalk w(s, pairs);
  const double rounds = w.whole / pairs + (w.whole % pairs != 0), steps = k_steps(s), epi = 4 * kTileEpilogue;
  const double main = 0.40 * steps;
  double t = 6 + rounds_time(rounds, main, epi);
  if (w.items > w.whole) t += rounds > 0 ? (0.5 * main > epi ? 0.5 * main : epi) - 0.5 * epi : 0.5 * (main + epi);
  return t;
}
inline MmaPlan plan_mma(const MmaShape& s, bool b_sym = false) {   // b_sym: a tile of a symmetric B lies within one of its blocks
  const int sms = sm_count();
  MmaPlan p{false, 64, 1};
  double least = single_time(s, sms, 64);
  for (int bn : {128, 192, 256}) {
    if (b_sym && bn == 192) continue;
    const double t = single_time(s, sms, bn);
    if (t < least) least = t, p = MmaPlan{false, bn, 1};
  }
  for (int bn : {64, 128})
    for (uint32_t parts : {2u, 4u, 8u}) {
      const double t = split_time(s, sms, bn, parts);
      if (t < least) least = t, p = MmaPlan{false, bn, parts};
    }
  const int pairs = pair_count();      // 0: no device that could be asked; the launch then says what is wrong
  if (pairs > 0 && pair_time(s, pairs) < least) p = MmaPlan{true, 256, 1};
  return p;
}

// launch_pdl with `smem` bytes of dynamic shared memory; beyond the 48 KB that a kernel gets by default allow_smem_for has raised its limit.
template <typename... P, typename... A>
inline void launch_pdl_dyn(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, A&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// Shared memory beyond 48 KB is asked for once per kernel and device.
template <auto KERNEL>
inline void allow_smem_for(size_t bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  (void)cudaGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (done.load(std::memory_order_relaxed) & bit) return;
  if (cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess)
    done.fetch_or(bit, std::memory_order_relaxed);
}

template <int KIND, int BN, int A_MODE, int B_MODE, class Epi>
cudaError_t launch_mma_bn(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& b2, const MmaShape& s, const Epi& epi, cudaStream_t st) {
  const TileWalk w(s, BN);
  const uint32_t grid = w.total < (uint32_t)sm_count() ? w.total : (uint32_t)sm_count();
  if (!grid) return cudaSuccess;
  allow_smem_for<k_mma<KIND, BN, A_MODE, B_MODE, Epi>>(MmaTile<BN, Epi>::kSmem);
  launch_pdl_dyn(k_mma<KIND, BN, A_MODE, B_MODE, Epi>, dim3(grid), dim3(kMmaThreads), MmaTile<BN, Epi>::kSmem, st, a, b, b2, s, epi);
  count_launches(1);
  return cudaGetLastError();
}

template <int KIND, int BN, int A_MODE, int B_MODE, class Epi>
cudaError_t launch_mma_split(uint32_t parts, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& b2, const MmaShape& s, const Epi& epi, cudaStream_t st) {
  const TileWalk w(s, BN);
  if (!w.total) return cudaSuccess;
  allow_smem_for<k_mma_split<KIND, BN, A_MODE, B_MODE, Epi>>(MmaTile<BN, Epi>::kSmem);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(w.total * parts);
  cfg.blockDim = dim3(kMmaThreads);
  cfg.dynamicSmemBytes = MmaTile<BN, Epi>::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = parts;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, k_mma_split<KIND, BN, A_MODE, B_MODE, Epi>, a, b, b2, s, epi, parts);
  count_launches(1);
  return cudaGetLastError();
}

template <int KIND, int A_MODE, int B_MODE, class Epi>
cudaError_t launch_mma(const MmaPlan& plan, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& b2, const MmaShape& s, const Epi& epi, cudaStream_t st) {
  if (plan.pair) {
    const PairWalk w(s, pair_count());
    const uint32_t pairs = w.items < (uint32_t)pair_count() ? w.items : (uint32_t)pair_count();
    if (!pairs) return cudaSuccess;
    allow_smem_for<k_mma_pair<KIND, A_MODE, B_MODE, Epi>>(PairTile<Epi>::kSmem);
    launch_pdl_dyn(k_mma_pair<KIND, A_MODE, B_MODE, Epi>, dim3(2 * pairs), dim3(kMmaThreads), PairTile<Epi>::kSmem, st, a, b, b2, s, epi);
    count_launches(1);
    return cudaGetLastError();
  }
  if (plan.parts > 1)
    return plan.bn == 128 ? launch_mma_split<KIND, 128, A_MODE, B_MODE>(plan.parts, a, b, b2, s, epi, st)
                          : launch_mma_split<KIND, 64, A_MODE, B_MODE>(plan.parts, a, b, b2, s, epi, st);
  switch (plan.bn) {
    case 256: return launch_mma_bn<KIND, 256, A_MODE, B_MODE>(a, b, b2, s, epi, st);
    case 192:
      if constexpr (B_MODE == kSym)
        return cudaErrorInvalidValue;
      else
        return launch_mma_bn<KIND, 192, A_MODE, B_MODE>(a, b, b2, s, epi, st);
    case 128: return launch_mma_bn<KIND, 128, A_MODE, B_MODE>(a, b, b2, s, epi, st);
    default: return launch_mma_bn<KIND, 64, A_MODE, B_MODE>(a, b, b2, s, epi, st);
  }
}

}  // namespace dsq
