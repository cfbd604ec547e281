// What stands between two blocks of a network, row by row:
//
//   u = post(y);  h = a x + D(g u);  n = pre(h)        post, pre: RMS or layer norms;  g: a gate;  D: dropout
//
// and all its gradients.  Bound by memory: x and y are read once and h and n written once, with everything between them in
// registers; backward, h is computed again from x and y (which costs no byte more than reading it would) with the norms'
// statistics that the forward pass left, and what parameters get is summed by CTAs that each take a run of rows, a thread
// its eight columns, and added up in the CTAs' order: nothing depends on timing.
//
// What bounds it (16384 x 4096, RMS norms before and after, bf16): forward 91 us, 5.9 TB/s, and backward 164 us, 4.9 TB/s, of a copy's 6.5; parameters and
// sums take the registers of one CTA an SM (128 a thread), and what is left over is the latency of a row's exchanges of sums and the issue of instructions (53 and 60 % of the cycles).
// Layer norms have an exchange more each forward, and backward one exchange of eight sums instead of three: 127 and 221 us.  One CTA a row that read the parameters again took 143 and 514.
#include "dsq_dropout.cuh"
#include "dsq_mma.cuh"
#include "dsq_rows8.cuh"

using namespace dsq;

namespace {

// A matrix: its rows are `pitch` bytes apart (a 32-bit number, so that an address is one multiplication).
struct Rows {
  const uint8_t* p;              // or NULL
  uint32_t pitch;
  __device__ __forceinline__ const uint8_t* at(uint32_t row) const { return p + (uint64_t)row * pitch; }
  template <class T>
  __device__ __forceinline__ T* out(uint32_t row) const { return reinterpret_cast<T*>(const_cast<uint8_t*>(at(row))); }
  __device__ __forceinline__ uint32_t shift(uint32_t row) const { return ((uint32_t)reinterpret_cast<uintptr_t>(p) + row * pitch) & 15; }
};
struct NormParams {
  Rows y, x;
  const float *post_w, *post_b, *gate, *pre_w, *pre_b;      // or NULL
  float residual_scale, eps;
  uint32_t rows, cols, group_rows;      // rows that share a gate
  int layer;                     // layer norms, else RMS
  Drop drop;
  float4* stats;                 // per row: mean and 1/size of y, of h; or NULL
  Rows h, n;                     // forward
  Rows dh, dn, dx, dy;           // backward
  float *gate_part;              // sums of every unit of rows (of every gate, where a gate's rows are one unit); or NULL
  float *part;                   // sums of every CTA: [teams][kinds][cols]
  uint32_t kinds;                // vectors in `part`
  int at_post_w, at_post_b, at_pre_w, at_pre_b;      // their places, or -1
  // both: runs of rows with one gate, and how rows are dealt out
  uint32_t units, unit_rows, units_per_group;
  uint32_t size;                 // CTAs of a cluster
  uint32_t* dev_status;          // or NULL
  int vec;                       // every row starts on a 16-byte boundary, and cols is a multiple of 8
};

// ---- how rows are dealt out -----------------------------------------------------------------------------
// A thread has eight columns.  blockDim.x threads (whole warps, up to 512) have a row, or, above 4096 columns, each CTA of a cluster its share of one; blockDim.y
// slices of a CTA have rows of their own and go at their own pace.  Units (runs of rows that share a gate) go to teams (CTAs or clusters) in turn, the rows of a unit to
// slices in turn.
constexpr uint32_t kNormCols = 4096, kNormThreads = 512;

struct RowWalk {
  uint32_t unit, row, last;      // row >= last: no more in this unit;  unit >= units: no more at all
  __device__ __forceinline__ void enter(const NormParams& p, uint32_t u) {
    unit = u;
    row = last = 0;
    if (u >= p.units) return;
    const uint32_t group = u / p.units_per_group, end = min((group + 1) * p.group_rows, p.rows);
    const uint32_t first = group * p.group_rows + (u - group * p.units_per_group) * p.unit_rows;
    last = min(first + p.unit_rows, end);
    row = first + threadIdx.y;
  }
  // to the first unit from u on that has a row for this slice
  __device__ __forceinline__ void find(const NormParams& p, uint32_t u, uint32_t teams) {
    enter(p, u);
    while (row >= last && unit < p.units) enter(p, unit + teams);
  }
};

// ---- rows on their way ----------------------------------------------------------------------------------
// Each warp copies its 256 columns of the rows to come into shared memory, DEPTH - 1 rows ahead: nothing but the warp itself waits for them, and no
// registers are held.  Whole granules are copied as they lie, so rows may start anywhere.  (A lane's two granules of floats apart, so that
// reading them meets no bank conflicts, made the copies slow: 16384 x 4096 backward 217 to 276 us.)
template <class T>
constexpr uint32_t kWarpBytes = 32 * 16 * (sizeof(T) / 2) + 16;      // 256 entries, and the granule behind them

// `part`: the warp's part of the row, of which `left` entries are there.
template <bool VEC, class T>
__device__ __forceinline__ void fetch_row(uint32_t to, const uint8_t* part, int left, int lane) {
  constexpr int G = sizeof(T) / 2;
  const uint32_t shift = VEC ? 0 : shift_of(part);
  const uint8_t* at = part - shift;
  const int bytes = left * (int)sizeof(T) + (int)shift;      // up to the row's end
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int i = lane + 32 * g;
    if (16 * i < bytes) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 16 * i), "l"(at + 16 * i) : "memory");
  }
  if (!VEC && shift && lane == 0 && bytes > 512 * G)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 512 * G), "l"(at + 512 * G) : "memory");
}
// This lane's eight entries of a row that has arrived; those behind the row's end are 0 (VEC: where nothing arrives, the ring holds zeros).
template <bool VEC, class T>
__device__ __forceinline__ void read_row8(uint32_t from, uint32_t shift, int left, int lane, float (&v)[8]) {
  constexpr int N = kWords<T>;
  constexpr int G = N / 4;
  uint32_t w[N + 4];
#pragma unroll
  for (int g = 0; g < G; ++g)
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4 * g]), "=r"(w[4 * g + 1]), "=r"(w[4 * g + 2]), "=r"(w[4 * g + 3]) : "r"(from + 16 * (G * lane + g)) : "memory");
  if constexpr (!VEC) {
    if (shift) {
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[N]), "=r"(w[N + 1]), "=r"(w[N + 2]), "=r"(w[N + 3]) : "r"(from + 16 * (G * lane + G)) : "memory");
      take_from<N>(w, shift);
    }
  }
  unpack8<T>(w, v);
  if (!VEC && left < 8)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= left) v[j] = 0.f;
}
template <int PENDING>
__device__ __forceinline__ void wait_rows() {
  asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory");
  __syncwarp();      // every lane's copies have landed, and every lane is done with the row before
}
__device__ __forceinline__ void commit_rows() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// VEC: pieces that no row reaches stay zero.
template <bool VEC>
__device__ __forceinline__ void clear_ring(const NormParams& p, uint8_t* ring, uint32_t bytes) {
  if (VEC && p.cols != blockDim.x * 8 * p.size) {
    for (uint32_t i = (threadIdx.y * blockDim.x + threadIdx.x) * 16; i < bytes; i += blockDim.x * blockDim.y * 16)
      *reinterpret_cast<uint4*>(ring + i) = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }
}

// Eight entries of a vector of parameters; `none` where there is no vector, 0 behind its end.
__device__ __forceinline__ void load_param8(const float* p, uint32_t c, uint32_t cols, float none, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = none;
  if (p && c + 8 <= cols && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    const float4 a = ld_plain(reinterpret_cast<const float4*>(p + c)), b = ld_plain(reinterpret_cast<const float4*>(p + c) + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else if (p || c + 8 > cols) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? p ? ld_plain(p + c + j) : none : 0.f;
  }
}

// ---- sums over the threads of a row ---------------------------------------------------------------------
struct alignas(16) SumSpace {
  float warp[2][8][8][16];      // of each slice's values by its warps (0 where there is no warp); the two halves take turns, so that one barrier is enough
  float cta[2][8][8];           // of each CTA of a cluster, written by the CTAs themselves
  uint64_t arrived[2];       // their bytes
  int gave_up;
};
// The CTAs of a cluster send one another their sums by stores that report to the receiver's barrier: nothing else has to be visible.  (A barrier of the cluster waits for
// every store to global memory before it: 8192 x 8192 in bf16 took 151 us forward, 248 backward.)  A CTA is a sum behind the others at most, which two halves are enough for.
struct RowSum {
  SumSpace* space;
  uint32_t sums = 0;      // so many before: which half is next, and its barrier's phase
  __device__ __forceinline__ void begin(uint32_t size) {
    float* zero = &space->warp[0][0][0][0];
    for (uint32_t i = threadIdx.y * blockDim.x + threadIdx.x; i < sizeof(space->warp) / 4; i += blockDim.x * blockDim.y) zero[i] = 0.f;
    if (size > 1 && threadIdx.x == 0 && threadIdx.y == 0) {
      mbar_init(smem_u32(&space->arrived[0]), 1);
      mbar_init(smem_u32(&space->arrived[1]), 1);
      space->gave_up = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (size > 1) cluster_sync();      // the others are there, and their barriers, before anything is sent
  }
  // K values at once.  One or two are added lane by lane.  Of more, lanes halve them between one another as they add (P / 2, P / 4, ... exchanges and then one each, where P
  // sums one by one would be five each): lanes of a group of 32 / P end with one of the sums, join it across the warps and hand it round.  Fewer instructions, a
  // longer way: four values 96 to 91 us (16384 x 4096 forward), two 168 to 174 (65536 x 768 backward, layer norms).
  template <int K>
  __device__ __forceinline__ void operator()(float (&v)[K], uint32_t size) {
    static_assert(K <= 8, "");
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const uint32_t turn = sums & 1;
    const bool joined = warps > 1 || size > 1;
    auto& space_of = space->warp[turn][threadIdx.y];      // [value][warp]
    auto wait = [] { asm volatile("bar.sync %0, %1;" ::"r"(1 + threadIdx.y), "r"(blockDim.x) : "memory"); };      // for this slice alone
    if constexpr (K <= 2) {
#pragma unroll
      for (int o = 16; o; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
      if (joined) {
        if (lane == 0)
#pragma unroll
          for (int k = 0; k < K; ++k) space_of[k][threadIdx.x >> 5] = v[k];
        wait();
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = space_of[k][lane & 15];
#pragma unroll
        for (int o = 8; o; o >>= 1)
#pragma unroll
          for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
      }
    } else {
      constexpr int P = K <= 4 ? 4 : 8, G = 32 / P;
      float w[P];
#pragma unroll
      for (int k = 0; k < P; ++k) w[k] = k < K ? v[k] : 0.f;
#pragma unroll
      for (int half = P / 2, off = 16; half; half /= 2, off /= 2)
#pragma unroll
        for (int i = 0; i < half; ++i) {
          const bool up = lane & off;
          const float mine = up ? w[i + half] : w[i], other = up ? w[i] : w[i + half];
          w[i] = mine + __shfl_xor_sync(0xFFFFFFFFu, other, off);
        }
#pragma unroll
      for (int off = G / 2; off; off /= 2) w[0] += __shfl_xor_sync(0xFFFFFFFFu, w[0], off);
      if (joined) {
        if ((lane & (G - 1)) == 0) space_of[lane / G][threadIdx.x >> 5] = w[0];
        wait();
        if constexpr (P == 8) {
          const float4 q = *reinterpret_cast<const float4*>(&space_of[lane / G][4 * (lane & (G - 1))]);
          w[0] = (q.x + q.y) + (q.z + q.w);
        } else {
          const float2 q = *reinterpret_cast<const float2*>(&space_of[lane / G][2 * (lane & (G - 1))]);
          w[0] = q.x + q.y;
        }
#pragma unroll
        for (int o = G / 2; o; o /= 2) w[0] += __shfl_xor_sync(0xFFFFFFFFu, w[0], o);
      }
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = __shfl_sync(0xFFFFFFFFu, w[0], k * G);
    }
    if (!joined) return;
    if (size > 1) {      // one slice here
      const uint32_t bar = smem_u32(&space->arrived[turn]);
      if (threadIdx.x == 0) mbar_expect_tx(bar, size * K * 4);
      if (threadIdx.x < size) {
        const uint32_t to_bar = in_cta(bar, threadIdx.x), to = in_cta(smem_u32(&space->cta[turn][cluster_rank()][0]), threadIdx.x);
#pragma unroll
        for (int k = 0; k < K; ++k)
          asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(to + 4 * k), "r"(__float_as_uint(v[k])), "r"(to_bar) : "memory");
      }
      __syncwarp();
      (void)mbar_wait(bar, sums >> 1 & 1, &space->gave_up);
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = 0.f;
      for (uint32_t r = 0; r < size; ++r)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += space->cta[turn][r][k];
    }
    ++sums;
  }
  // No CTA's shared memory goes away under a neighbour's store; a wait that ran out is told of.
  __device__ __forceinline__ void end(uint32_t size, uint32_t* dev_status) {
    if (size == 1) return;
    cluster_sync();
    if (threadIdx.x == 0 && space->gave_up && dev_status) atomicOr(dev_status + DS_DEV_WORD_FLAGS, DS_DEV_NORM_TIMEOUT);
  }
};

// What both passes begin with.
struct Place {
  uint32_t rank, team, teams, c, c_warp;
  int lane, warp, left, left_warp;      // entries of a row from this thread's and this warp's first on
  __device__ __forceinline__ Place(const NormParams& p) {
    rank = 0;
    if (p.size > 1) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    team = blockIdx.x / p.size, teams = gridDim.x / p.size;
    c = (rank * blockDim.x + threadIdx.x) * 8;
    lane = threadIdx.x & 31;
    c_warp = c - 8 * lane;
    left = entries_left(c, p.cols), left_warp = entries_left(c_warp, p.cols);
    warp = threadIdx.y * (blockDim.x >> 5) + (threadIdx.x >> 5);
  }
};

// ---- forward --------------------------------------------------------------------------------------------
// FULL: layer norms or biases.  Parameters stay in registers.  A slice has ROWS rows in hand, whose sums share their barriers: a row takes mostly
// the time from its first addition to its sums (16384 x 4096 in bf16, RMS norms before and after: 100 us by two rows, 96 by four; 8192 x 8192: 199 and 151; layer norms
// 144 by two, 139 by three, 174 by four, which no longer fit into the registers; floats fill shared memory with two).
template <class X, class Y, bool FULL>
constexpr int kRowsInHand = sizeof(X) + sizeof(Y) == 8 ? 2 : FULL ? 3 : 4;
template <class X, class Y, int ROWS>
struct ForwardRing {
  static constexpr uint32_t kRow = kWarpBytes<X> + kWarpBytes<Y>, kWarp = ROWS * kRow;      // a warp's part of a row, and of the rows in hand
  static constexpr int kDepth = 16 * kWarp * 3 <= 220 * 1024 ? 3 : 2;
  static constexpr uint32_t kThread = kDepth * kWarp / 32;                                  // bytes a thread
};
template <class X, class Y, bool FULL, bool VEC, int ROWS>
__global__ void __launch_bounds__(kNormThreads, 1) k_norm_forward(const NormParams p) {
  using R = ForwardRing<X, Y, ROWS>;
  constexpr int kRows = ROWS;
  extern __shared__ __align__(16) uint8_t ring[];      // [depth][warps][rows][y | x]
  __shared__ SumSpace space;
  pdl_prologue();
  const Place at(p);
  RowSum row_sum{&space};
  row_sum.begin(p.size);
  auto sum = [&](auto& v) { row_sum(v, p.size); };
  const uint32_t warps = (blockDim.x >> 5) * blockDim.y, slot_bytes = warps * R::kWarp;
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + at.warp * R::kWarp;
  const float inv = 1.f / (float)p.cols;
  clear_ring<VEC>(p, ring, R::kDepth * slot_bytes);
  RowWalk ahead, now;
  uint32_t put = 0, get = 0;
  ahead.find(p, at.team, at.teams);
  auto fetch = [&] {
    if (ahead.unit < p.units) {
      const uint32_t to = mine + put * slot_bytes;
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const uint32_t row = ahead.row + i * blockDim.y;
        if (row < ahead.last) {
          fetch_row<VEC, Y>(to + i * R::kRow, p.y.at(row) + at.c_warp * sizeof(Y), at.left_warp, at.lane);
          if (p.x.p) fetch_row<VEC, X>(to + i * R::kRow + kWarpBytes<Y>, p.x.at(row) + at.c_warp * sizeof(X), at.left_warp, at.lane);
        }
      }
      ahead.row += kRows * blockDim.y;
      if (ahead.row >= ahead.last) ahead.find(p, ahead.unit + at.teams, at.teams);
    }
    commit_rows();
    if (++put == R::kDepth) put = 0;
  };
#pragma unroll
  for (int i = 0; i < R::kDepth - 1; ++i) fetch();

  // parameters: u = hat gw + gb;  n = hat w2 + b2
  float gw[8], gb[8], w2[8], b2[8];
  uint32_t group = 0xFFFFFFFFu;
  load_param8(p.pre_w, at.c, p.cols, 0.f, w2);
  if constexpr (FULL) load_param8(p.pre_b, at.c, p.cols, 0.f, b2);

  // mean and 1 / size of the rows
  auto statistics = [&](const float (&v)[kRows][8], float (&mean)[kRows], float (&r)[kRows]) {
    float q[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) mean[i] = q[i] = 0.f;
    if (FULL && p.layer) {
#pragma unroll
      for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) mean[i] += v[i][j];
      sum(mean);
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        mean[i] *= inv;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = VEC || j < at.left ? v[i][j] - mean[i] : 0.f;
          q[i] = __fmaf_rn(d, d, q[i]);
        }
        if (VEC && at.left <= 0) q[i] = 0.f;      // columns that are not there
      }
    } else {
#pragma unroll
      for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) q[i] = __fmaf_rn(v[i][j], v[i][j], q[i]);
    }
    sum(q);
#pragma unroll
    for (int i = 0; i < kRows; ++i) r[i] = rsqrtf(__fmaf_rn(q[i], inv, p.eps));      // good to 2 units of 2^-23
  };
  for (now.find(p, at.team, at.teams); now.unit < p.units; now.find(p, now.unit + at.teams, at.teams)) {
    const uint32_t g = now.unit / p.units_per_group;
    if (g != group) {
      float t[8];
      load_param8(p.post_w, at.c, p.cols, 1.f, gw);
      if constexpr (FULL) load_param8(p.post_b, at.c, p.cols, 0.f, gb);
      if (p.gate) {
        load_param8(p.gate + (uint64_t)g * p.cols, at.c, p.cols, 1.f, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          gw[j] *= t[j];
          if constexpr (FULL) gb[j] *= t[j];
        }
      }
      group = g;
    }
    for (; now.row < now.last; now.row += kRows * blockDim.y) {
      wait_rows<R::kDepth - 2>();
      fetch();
      const uint32_t from = mine + get * slot_bytes;
      if (++get == R::kDepth) get = 0;
      // rows that are not there are what the ring held: worked on, not stored
      auto there = [&](int i) { return !i || now.row + i * blockDim.y < now.last; };
      auto row = [&](int i) { return now.row + i * blockDim.y; };
      float v[kRows][8], mean[kRows], r[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) read_row8<VEC, Y>(from + i * R::kRow, VEC ? 0 : p.y.shift(row(i)), at.left, at.lane, v[i]);
      float2* st = reinterpret_cast<float2*>(p.stats);
      const bool notes = st && threadIdx.x == 0 && at.rank == 0;
      if (p.post_w) {
        statistics(v, mean, r);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          if (notes && there(i)) st[2 * row(i)] = make_float2(mean[i], r[i]);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = (FULL ? v[i][j] - mean[i] : v[i][j]) * r[i];
        }
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = FULL ? __fmaf_rn(v[i][j], gw[j], gb[j]) : v[i][j] * gw[j];
        if (p.drop.threshold) drop8(p.drop, draw8(p.drop, row(i), at.c), v[i]);
        if (p.x.p) {
          float t[8];
          read_row8<VEC, X>(from + i * R::kRow + kWarpBytes<Y>, VEC ? 0 : p.x.shift(row(i)), at.left, at.lane, t);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = __fmaf_rn(p.residual_scale, t[j], v[i][j]);
        }
        if (p.h.p && there(i)) store_row8<VEC>(p.h.out<X>(row(i)), at.c, p.cols, at.lane, v[i]);
      }
      if (p.pre_w) {
        statistics(v, mean, r);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          if (notes && there(i)) st[2 * row(i) + 1] = make_float2(mean[i], r[i]);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            v[i][j] = (FULL ? v[i][j] - mean[i] : v[i][j]) * r[i];
            v[i][j] = FULL ? __fmaf_rn(v[i][j], w2[j], b2[j]) : v[i][j] * w2[j];
          }
          if (there(i)) store_row8<VEC>(p.n.out<Y>(row(i)), at.c, p.cols, at.lane, v[i]);
        }
      }
    }
  }
  row_sum.end(p.size, p.dev_status);
}

// ---- backward -------------------------------------------------------------------------------------------
//   d = dh + J_pre^T dn;   dx = a d;   q = g D(d);   dy = J_post^T q
//   J^T t = r (w t - mean(w t) - hat mean(w t hat)), the second term for layer norms alone
// A thread sums  A = sum D(d) hat1,  B = sum D(d)  over the rows of a unit, from which the gradients of gate, post weight and bias follow
// (w1 A + b1 B, g A, g B), and  C = sum dn hat2,  E = sum dn  over all of its rows.
template <class X, class Y>
struct BackwardRing {
  static constexpr uint32_t kWarp = 2 * kWarpBytes<X> + 2 * kWarpBytes<Y>;      // y, x, dn, dh
  static constexpr int kDepth = sizeof(X) + sizeof(Y) == 8 ? 2 : sizeof(X) + sizeof(Y) == 6 ? 3 : 4;
};
template <class X, class Y, bool FULL, bool VEC>
__global__ void __launch_bounds__(kNormThreads, 1) k_norm_backward(const NormParams p) {
  using R = BackwardRing<X, Y>;
  extern __shared__ __align__(16) uint8_t ring[];      // [depth][warps][y | x | dn | dh], then sums of the post norm's gradients [2][8][threads], then [threads][8]
  __shared__ SumSpace space;
  pdl_prologue();
  const Place at(p);
  RowSum row_sum{&space};
  row_sum.begin(p.size);
  auto sum = [&](auto& v) { row_sum(v, p.size); };
  const uint32_t threads = blockDim.x * blockDim.y, warps = threads >> 5, slot_bytes = warps * R::kWarp, tid = threadIdx.y * blockDim.x + threadIdx.x;
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + at.warp * R::kWarp;
  float* post = reinterpret_cast<float*>(ring + R::kDepth * slot_bytes) + tid;      // a thread's own, `threads` apart
  float* flush = reinterpret_cast<float*>(ring + R::kDepth * slot_bytes) + 16 * threads;
  const float inv = 1.f / (float)p.cols;
  constexpr uint32_t kAtX = kWarpBytes<Y>, kAtDn = kAtX + kWarpBytes<X>, kAtDh = kAtDn + kWarpBytes<Y>;
  clear_ring<VEC>(p, ring, R::kDepth * slot_bytes);
  RowWalk ahead, now;
  uint32_t put = 0, get = 0;
  ahead.find(p, at.team, at.teams);
  auto fetch = [&] {
    if (ahead.unit < p.units) {
      const uint32_t to = mine + put * slot_bytes, row = ahead.row;
      fetch_row<VEC, Y>(to, p.y.at(row) + at.c_warp * sizeof(Y), at.left_warp, at.lane);
      if (p.x.p) fetch_row<VEC, X>(to + kAtX, p.x.at(row) + at.c_warp * sizeof(X), at.left_warp, at.lane);
      if (p.dn.p) fetch_row<VEC, Y>(to + kAtDn, p.dn.at(row) + at.c_warp * sizeof(Y), at.left_warp, at.lane);
      if (p.dh.p) fetch_row<VEC, X>(to + kAtDh, p.dh.at(row) + at.c_warp * sizeof(X), at.left_warp, at.lane);
      ahead.row += blockDim.y;
      if (ahead.row >= ahead.last) ahead.find(p, ahead.unit + at.teams, at.teams);
    }
    commit_rows();
    if (++put == R::kDepth) put = 0;
  };
#pragma unroll
  for (int i = 0; i < R::kDepth - 1; ++i) fetch();

  float w2[8], gw[8], gb[8], s_a[8], s_b[8], s_c[8], s_e[8];
  load_param8(p.pre_w, at.c, p.cols, 0.f, w2);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    s_a[j] = s_b[j] = s_c[j] = s_e[j] = 0.f;
    post[j * threads] = post[(8 + j) * threads] = 0.f;
  }
  // what the slices summed of one kind, into a vector
  auto flush_to = [&](const float (&s)[8], float* to) {
    const uint32_t width = blockDim.x * 8, c0 = at.rank * width;
    if (blockDim.y == 1) {      // (entry by entry, a warp's stores touch 32 sectors each: a single row of 4096 took 7.9 us)
      if (at.c + 8 <= p.cols && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
        store_piece8(to + at.c, s);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (at.c + j < p.cols) to[at.c + j] = s[j];
      }
    } else {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) flush[threadIdx.y * width + threadIdx.x * 8 + j] = s[j];
      __syncthreads();
      for (uint32_t k = tid; k < width; k += threads) {
        float v = 0.f;
        for (uint32_t i = 0; i < blockDim.y; ++i) v += flush[i * width + k];
        if (c0 + k < p.cols) to[c0 + k] = v;
      }
    }
  };

  uint32_t group = 0xFFFFFFFFu;
  for (uint32_t u = at.team; u < p.units; u += at.teams) {
    const uint32_t g = u / p.units_per_group;
    if (g != group) {
      float t[8];
      load_param8(p.post_w, at.c, p.cols, 1.f, gw);
      if constexpr (FULL) load_param8(p.post_b, at.c, p.cols, 0.f, gb);
      if (p.gate) {
        load_param8(p.gate + (uint64_t)g * p.cols, at.c, p.cols, 1.f, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          gw[j] *= t[j];
          if constexpr (FULL) gb[j] *= t[j];
        }
      }
      group = g;
    }
    now.enter(p, u);
    float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
    if (p.stats && now.row < now.last) st = ld_plain(p.stats + now.row);
    for (; now.row < now.last; now.row += blockDim.y) {
      float4 st_next = st;
      if (p.stats && now.row + blockDim.y < now.last) st_next = ld_plain(p.stats + now.row + blockDim.y);
      wait_rows<R::kDepth - 2>();
      fetch();
      const uint32_t from = mine + get * slot_bytes, row = now.row;
      if (++get == R::kDepth) get = 0;
      float hat1[8], d[8];
      read_row8<VEC, Y>(from, VEC ? 0 : p.y.shift(row), at.left, at.lane, hat1);
      if (p.post_w) {
#pragma unroll
        for (int j = 0; j < 8; ++j) hat1[j] = (FULL ? hat1[j] - st.x : hat1[j]) * st.y;
      }
      uint4 draw = make_uint4(0, 0, 0, 0);
      if (p.drop.threshold) draw = draw8(p.drop, row, at.c);
      if (p.dh.p) {
        read_row8<VEC, X>(from + kAtDh, VEC ? 0 : p.dh.shift(row), at.left, at.lane, d);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = 0.f;
      }
      // One exchange of sums for both norms.  With  e = dh + r2 w2 dn,  q = D(g w1),  S = mean(w2 dn hat2)  and  M = mean(w2 dn)  (layer norms)
      // the gradient of h is  d = e - r2 (M + S hat2),  and what the post norm takes the mean of follows from sums that need neither S nor M:
      //   sum q d = sum q e - r2 M sum q - r2 S sum q hat2,     sum q hat1 d = sum q hat1 e - r2 M sum q hat1 - r2 S sum q hat1 hat2
      float hat2[8], q[8], s[FULL ? 8 : 3];
#pragma unroll
      for (int i = 0; i < (FULL ? 8 : 3); ++i) s[i] = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = FULL ? gw[j] : hat1[j] * gw[j];      // (RMS norms: q hat1)
      if (p.drop.threshold && (!FULL || p.post_w)) drop8(p.drop, draw, q);
      if (p.dn.p) {
        float t[8];
        if constexpr (FULL) {
#pragma unroll
          for (int j = 0; j < 8; ++j) hat2[j] = __fmaf_rn(hat1[j], gw[j], gb[j]);
          if (p.drop.threshold) drop8(p.drop, draw, hat2);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) hat2[j] = q[j];
        }
        if (p.x.p) {
          read_row8<VEC, X>(from + kAtX, VEC ? 0 : p.x.shift(row), at.left, at.lane, t);
#pragma unroll
          for (int j = 0; j < 8; ++j) hat2[j] = __fmaf_rn(p.residual_scale, t[j], hat2[j]);
        }
        read_row8<VEC, Y>(from + kAtDn, VEC ? 0 : p.dn.shift(row), at.left, at.lane, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hat2[j] = (FULL ? hat2[j] - st.z : hat2[j]) * st.w;
          s_c[j] = __fmaf_rn(t[j], hat2[j], s_c[j]);
          if constexpr (FULL) s_e[j] += t[j];
          t[j] *= w2[j];
          s[0] = __fmaf_rn(t[j], hat2[j], s[0]);
          if constexpr (FULL) s[1] += t[j];
          d[j] = __fmaf_rn(st.w, t[j], d[j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) hat2[j] = 0.f;
      }
      float k1 = 0.f, m1 = 0.f;
      if (p.post_w) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if constexpr (FULL) {
            s[2] = __fmaf_rn(q[j], d[j], s[2]);
            s[3] += q[j];
            s[4] = __fmaf_rn(q[j], hat2[j], s[4]);
            const float u = q[j] * hat1[j];
            s[5] = __fmaf_rn(u, d[j], s[5]);
            s[6] += u;
            s[7] = __fmaf_rn(u, hat2[j], s[7]);
          } else {
            s[1] = __fmaf_rn(q[j], d[j], s[1]);
            s[2] = __fmaf_rn(q[j], hat2[j], s[2]);
          }
        }
        sum(s);
      } else if (p.dn.p) {
        if constexpr (FULL)
          sum(*reinterpret_cast<float(*)[2]>(s));
        else
          sum(*reinterpret_cast<float(*)[1]>(s));
      }
      const float r2 = p.dn.p ? st.w * inv : 0.f, k = r2 * s[0];      // without a pre norm its statistics are not there
      if constexpr (FULL) {
        const float m = p.layer ? r2 * s[1] : 0.f;
        m1 = p.layer ? __fmaf_rn(-k, s[4], __fmaf_rn(-m, s[3], s[2])) * inv : 0.f;
        k1 = __fmaf_rn(-k, s[7], __fmaf_rn(-m, s[6], s[5])) * inv;
        if (p.dn.p)
#pragma unroll
          for (int j = 0; j < 8; ++j) d[j] = __fmaf_rn(-hat2[j], k, d[j] - m);
      } else {
        k1 = __fmaf_rn(-k, s[2], s[1]) * inv;
        if (p.dn.p)
#pragma unroll
          for (int j = 0; j < 8; ++j) d[j] = __fmaf_rn(-hat2[j], k, d[j]);
      }
      if (p.dx.p) {
        float t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = p.residual_scale * d[j];
        store_row8<VEC>(p.dx.out<X>(row), at.c, p.cols, at.lane, t);
      }
      if (p.drop.threshold) drop8(p.drop, draw, d);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s_a[j] = __fmaf_rn(d[j], hat1[j], s_a[j]);
        if constexpr (FULL) s_b[j] += d[j];
        d[j] *= gw[j];
        if (p.post_w) d[j] = st.y * __fmaf_rn(-hat1[j], k1, FULL ? d[j] - m1 : d[j]);
      }
      if (p.dy.p) store_row8<VEC>(p.dy.out<Y>(row), at.c, p.cols, at.lane, d);
      st = st_next;
    }
    if (p.gate_part) {
      float t[8], w[8];
      load_param8(p.post_w, at.c, p.cols, 1.f, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) t[j] = w[j] * s_a[j];
      if constexpr (FULL) {
        load_param8(p.post_b, at.c, p.cols, 0.f, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = __fmaf_rn(w[j], s_b[j], t[j]);
      }
      flush_to(t, p.gate_part + (uint64_t)u * p.cols);
    }
    if (p.at_post_w >= 0) {
      float t[8];
      load_param8(p.gate ? p.gate + (uint64_t)g * p.cols : nullptr, at.c, p.cols, 1.f, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        post[j * threads] = __fmaf_rn(t[j], s_a[j], post[j * threads]);
        if constexpr (FULL) post[(8 + j) * threads] = __fmaf_rn(t[j], s_b[j], post[(8 + j) * threads]);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) s_a[j] = s_b[j] = 0.f;
  }
  float* part = p.part + (uint64_t)at.team * p.kinds * p.cols;
  if (p.at_post_w >= 0) {
    float t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = post[j * threads];
    flush_to(t, part + (uint64_t)p.at_post_w * p.cols);
    if (FULL && p.at_post_b >= 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) t[j] = post[(8 + j) * threads];
      flush_to(t, part + (uint64_t)p.at_post_b * p.cols);
    }
  }
  if (p.at_pre_w >= 0) flush_to(s_c, part + (uint64_t)p.at_pre_w * p.cols);
  if (FULL && p.at_pre_b >= 0) flush_to(s_e, part + (uint64_t)p.at_pre_b * p.cols);
  row_sum.end(p.size, p.dev_status);
}

// The CTAs' sums, added in their order: out[v] = sum_i in[v * stride_v + i * stride_i].
struct SumsParams {
  const float* in[5];
  float* out[5];
  uint64_t step[5];       // between what is added
  uint32_t count[5], vectors[5];      // vectors: of this kind (gates: one a group), `count` steps apart
  uint32_t cols;
};
constexpr int kSumThreads = 512;
__global__ void __launch_bounds__(kSumThreads) k_norm_sums(const SumsParams p) {
  constexpr int kWarps = kSumThreads / 32, kBatch = 10;      // loads in flight: those of 160 CTAs' sums at once
  __shared__ float part[kWarps][32];
  pdl_prologue();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t col = blockIdx.x * 32 + lane;
  uint32_t v = blockIdx.y, kind = 0;
  while (v >= p.vectors[kind]) v -= p.vectors[kind++];
  const float* in = p.in[kind] + (uint64_t)v * p.count[kind] * p.step[kind];
  float s = 0.f;
  if (col < p.cols)
    for (uint32_t i = warp; i < p.count[kind]; i += kWarps * kBatch) {
      float t[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) t[b] = i + kWarps * b < p.count[kind] ? ld_plain(in + (i + kWarps * b) * p.step[kind] + col) : 0.f;
#pragma unroll
      for (int b = 0; b < kBatch; ++b) s += t[b];
    }
  part[warp][lane] = s;
  __syncthreads();
  if (warp || col >= p.cols) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) s += part[w][lane];
  p.out[kind][(uint64_t)v * p.cols + col] = s;
}

// ---- host side ------------------------------------------------------------------------------------------

inline uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }
inline bool aligned(const void* p, uint64_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline uint32_t size_of(uint64_t dtype) { return dtype == DS_F32 ? 4 : 2; }
constexpr uint64_t kMaxRows = 1ull << 30;

// How a pass is cut.
struct NormPlan {
  uint32_t size;              // CTAs of a cluster
  uint32_t tx, ty;            // threads of a row (or of its share), slices
  uint32_t units, unit_rows, units_per_group, teams;
  uint64_t gate_bytes, part_bytes;
};
NormPlan norm_plan(const ds_norm_args* p) {
  NormPlan b;
  const uint64_t cols = p->cols, groups = p->groups ? p->groups : 1, group_rows = p->rows / groups;
  b.size = 1;
  while (b.size * (uint64_t)kNormCols < cols) b.size *= 2;
  const uint32_t pieces = (uint32_t)((cols + 8 * b.size - 1) / (8 * b.size));
  b.tx = (uint32_t)round_up(pieces, 32);
  b.ty = b.size > 1 ? 1 : kNormThreads / b.tx;
  // as many teams as run at once (one CTA an SM); with few rows a team has fewer slices, so that all of the device works
  const uint64_t want = b.size > 1 ? (cluster_count(b.size) ? cluster_count(b.size) : 1) : sm_count();
  while (b.ty > 1 && p->rows < want * b.ty) --b.ty;
  // Units of a group: so many that the team with most rows has fewest (units go to teams in turn); tried for one to four units a team.
  const uint64_t most = (group_rows + b.ty - 1) / b.ty;
  uint64_t least = ~0ull;
  for (uint64_t k = 1; k <= 4; ++k) {
    uint64_t per = k * want / groups;
    per = per < 1 ? 1 : per > most ? most : per;
    const uint64_t rows = round_up((group_rows + per - 1) / per, b.ty), units = (group_rows + rows - 1) / rows, cost = (units * groups + want - 1) / want * (rows / b.ty);
    if (cost < least) {
      least = cost;
      b.unit_rows = (uint32_t)rows;
      b.units_per_group = (uint32_t)units;
    }
  }
  b.units = (uint32_t)(b.units_per_group * groups);
  b.teams = b.units < want ? b.units : (uint32_t)want;
  const uint32_t kinds = (p->d_post_w != nullptr || p->d_post_b != nullptr) + (p->d_post_b != nullptr) + (p->d_pre_w != nullptr) + (p->d_pre_b != nullptr);
  b.gate_bytes = p->d_gate && b.units_per_group > 1 ? round_up(4ull * b.units * cols, 256) : 0;
  b.part_bytes = 4ull * b.teams * kinds * cols;
  return b;
}

template <auto KERNEL>
cudaError_t launch(NormParams q, const NormPlan& b, uint32_t smem, uint32_t most, cudaStream_t st) {
  allow_smem_for<KERNEL>(most);
  q.units = b.units, q.unit_rows = b.unit_rows, q.units_per_group = b.units_per_group, q.size = b.size;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(b.teams * b.size);
  cfg.blockDim = dim3(b.tx, b.ty);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = b.size;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = b.size > 1 ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, KERNEL, q);
  count_launches(1);
  return cudaGetLastError();
}
inline bool full(const NormParams& q) { return q.layer || q.post_b || q.pre_b; }
template <class X, class Y, bool FULL, int ROWS>
cudaError_t forward_by(const NormParams& q, const NormPlan& b, cudaStream_t st) {
  constexpr uint32_t kThread = ForwardRing<X, Y, ROWS>::kThread;
  const uint32_t smem = b.tx * b.ty * kThread, most = kNormThreads * kThread;
  return q.vec ? launch<k_norm_forward<X, Y, FULL, true, ROWS>>(q, b, smem, most, st) : launch<k_norm_forward<X, Y, FULL, false, ROWS>>(q, b, smem, most, st);
}
template <class X, class Y>
cudaError_t forward(const NormParams& q, const NormPlan& b, cudaStream_t st) {
  // two rows a slice at most, one after the other: rows that are not there would only cost time (1 x 4096: 4.5 us by four rows, 3.1 by one)
  const bool single = b.unit_rows <= 2 * b.ty && b.units <= b.teams;
  if (full(q)) return single ? forward_by<X, Y, true, 1>(q, b, st) : forward_by<X, Y, true, kRowsInHand<X, Y, true>>(q, b, st);
  return single ? forward_by<X, Y, false, 1>(q, b, st) : forward_by<X, Y, false, kRowsInHand<X, Y, false>>(q, b, st);
}
template <class X, class Y>
cudaError_t backward(const NormParams& q, const NormPlan& b, cudaStream_t st) {
  using R = BackwardRing<X, Y>;
  constexpr uint32_t kThread = R::kDepth * R::kWarp / 32 + 64 + 32;
  const uint32_t smem = b.tx * b.ty * kThread, most = kNormThreads * kThread;
  if (q.vec) return full(q) ? launch<k_norm_backward<X, Y, true, true>>(q, b, smem, most, st) : launch<k_norm_backward<X, Y, false, true>>(q, b, smem, most, st);
  return full(q) ? launch<k_norm_backward<X, Y, true, false>>(q, b, smem, most, st) : launch<k_norm_backward<X, Y, false, false>>(q, b, smem, most, st);
}

template <class F>
cudaError_t by_types(const ds_norm_args* p, F&& f) {
  using H = __half;
  using B = __nv_bfloat16;
  if (p->dtype == DS_F32) return f(float(), float());
  if (p->dtype == DS_BF16) return p->stream_dtype == DS_F32 ? f(float(), B()) : f(B(), B());
  return p->stream_dtype == DS_F32 ? f(float(), H()) : f(H(), H());
}

int check(const ds_norm_args* p, bool back) {
  if (!p || p->dtype > DS_F16 || (p->stream_dtype != p->dtype && p->stream_dtype != DS_F32) || p->norm > DS_NORM_LAYER) return DS_ERR_INVALID_ARG;
  if (p->rows > kMaxRows || p->cols == 0) return DS_ERR_INVALID_ARG;
  if (p->cols > DS_NORM_MAX_COLS) return DS_ERR_UNSUPPORTED;
  if (p->groups && (!p->gate || p->groups > kMaxRows || p->rows % p->groups)) return DS_ERR_INVALID_ARG;
  if (!p->groups && p->gate) return DS_ERR_INVALID_ARG;
  if ((p->post_b && !p->post_w) || (p->pre_b && !p->pre_w)) return DS_ERR_INVALID_ARG;
  if (!(p->eps >= 0) || p->threshold > 65535 || p->layer > 0xFFFFFFFFull || p->step > 0xFFFFFFFFull) return DS_ERR_INVALID_ARG;
  const uint32_t sy = size_of(p->dtype), sx = size_of(p->stream_dtype);
  const void* vectors[] = {p->post_w, p->post_b, p->gate, p->pre_w, p->pre_b, p->d_post_w, p->d_post_b, p->d_gate, p->d_pre_w, p->d_pre_b};
  for (const void* v : vectors)
    if (!aligned(v, 4)) return DS_ERR_ALIGN;
  if (!aligned(p->stats, 16) || !aligned(p->dev_status, 4) || !aligned(p->y, sy) || !aligned(p->n, sy) || !aligned(p->dn, sy) || !aligned(p->dy, sy) || !aligned(p->x, sx) || !aligned(p->h, sx) ||
      !aligned(p->dh, sx) || !aligned(p->dx, sx))
    return DS_ERR_ALIGN;
  if (p->rows == 0) return DS_OK;
  if (!p->y) return DS_ERR_INVALID_ARG;
  const bool many = p->rows > 1;
  auto narrow = [&](const void* q, uint64_t ld) { return many && q && ld < p->cols; };
  // rows 2^30 entries apart at most: addresses are made with 32-bit pitches
  auto far = [&](const void* q, uint64_t ld) { return many && q && ld >= 1ull << 30; };
  if (far(p->y, p->ldy) || far(p->x, p->ldx) || (!back && (far(p->h, p->ldh) || far(p->n, p->ldn))) ||
      (back && (far(p->dh, p->lddh) || far(p->dn, p->lddn) || far(p->dx, p->lddx) || far(p->dy, p->lddy))))
    return DS_ERR_UNSUPPORTED;
  if (narrow(p->y, p->ldy) || narrow(p->x, p->ldx)) return DS_ERR_INVALID_ARG;
  if (!back) {
    if (narrow(p->h, p->ldh) || narrow(p->n, p->ldn)) return DS_ERR_INVALID_ARG;
    if ((p->n != nullptr) != (p->pre_w != nullptr) || (!p->h && !p->n)) return DS_ERR_INVALID_ARG;
  } else {
    if (narrow(p->dh, p->lddh) || narrow(p->dn, p->lddn) || narrow(p->dx, p->lddx) || narrow(p->dy, p->lddy)) return DS_ERR_INVALID_ARG;
    if ((!p->dh && !p->dn) || (p->dn && !p->pre_w) || (p->dx && !p->x)) return DS_ERR_INVALID_ARG;
    if ((p->post_w || p->pre_w) && !p->stats) return DS_ERR_INVALID_ARG;
    if ((p->d_post_w && !p->post_w) || (p->d_post_b && !p->post_b) || (p->d_gate && !p->gate) || (p->d_pre_w && !p->pre_w) || (p->d_pre_b && !p->pre_b))
      return DS_ERR_INVALID_ARG;
  }
  return DS_OK;
}

struct Parameters {
  Span all[5];
};
Parameters parameters(const ds_norm_args* p) {
  auto vector = [&](const float* v, uint64_t n) { return span(v, 1, n, 0, 4); };
  return {{vector(p->post_w, p->cols), vector(p->post_b, p->cols), vector(p->pre_w, p->cols), vector(p->pre_b, p->cols), vector(p->gate, p->groups * p->cols)}};
}

NormParams params(const ds_norm_args* p, bool back) {
  NormParams q{};
  q.post_w = p->post_w, q.post_b = p->post_b, q.gate = p->gate, q.pre_w = p->pre_w, q.pre_b = p->pre_b;
  q.residual_scale = (float)p->residual_scale, q.eps = (float)p->eps;
  q.rows = (uint32_t)p->rows, q.cols = (uint32_t)p->cols, q.group_rows = (uint32_t)(p->rows / (p->groups ? p->groups : 1));
  q.layer = p->norm == DS_NORM_LAYER;
  q.drop = make_drop((uint32_t)p->threshold, p->seed, (uint32_t)p->layer, (uint32_t)p->step);
  q.stats = reinterpret_cast<float4*>(p->stats);
  q.dev_status = p->dev_status;
  const uint32_t sy = size_of(p->dtype), sx = size_of(p->stream_dtype);
  auto rows = [&](const void* m, uint64_t ld, uint32_t size) { return Rows{static_cast<const uint8_t*>(m), p->rows > 1 ? (uint32_t)(ld * size) : 0}; };
  q.y = rows(p->y, p->ldy, sy), q.x = rows(p->x, p->ldx, sx);
  if (back)
    q.dh = rows(p->dh, p->lddh, sx), q.dn = rows(p->dn, p->lddn, sy), q.dx = rows(p->dx, p->lddx, sx), q.dy = rows(p->dy, p->lddy, sy);
  else
    q.h = rows(p->h, p->ldh, sx), q.n = rows(p->n, p->ldn, sy);
  auto on = [&](const void* m, uint64_t ld, uint32_t size) { return rows_on_boundary(m, ld, p->rows, size); };
  q.vec = p->cols % 8 == 0 && on(p->y, p->ldy, sy) && on(p->x, p->ldx, sx) && on(p->h, p->ldh, sx) && on(p->n, p->ldn, sy) && on(p->dh, p->lddh, sx) &&
          on(p->dn, p->lddn, sy) && on(p->dx, p->lddx, sx) && on(p->dy, p->lddy, sy);
  return q;
}

}  // namespace

extern "C" {

int ds_norm_forward(const ds_norm_args* p, void* cuda_stream) {
  const int rc = check(p, false);
  if (rc != DS_OK || p->rows == 0) return rc;
  const uint32_t sy = size_of(p->dtype), sx = size_of(p->stream_dtype);
  const Span y = span(p->y, p->rows, p->cols, p->ldy, sy), x = span(p->x, p->rows, p->cols, p->ldx, sx), h = span(p->h, p->rows, p->cols, p->ldh, sx),
               n = span(p->n, p->rows, p->cols, p->ldn, sy), stats = span(p->stats, 1, 4 * p->rows, 0, 4);
  // a thread reads its entries of x and y before it writes the same ones of h; n comes after them all
  auto over = [&](const void* a, uint64_t lda, uint32_t sa, const void* b, uint64_t ldb, uint32_t sb) { return a == b && sa == sb && (lda == ldb || p->rows == 1); };
  if ((overlap(h, x) && !over(p->h, p->ldh, sx, p->x, p->ldx, sx)) || (overlap(h, y) && !over(p->h, p->ldh, sx, p->y, p->ldy, sy)) ||
      (overlap(n, x) && !over(p->n, p->ldn, sy, p->x, p->ldx, sx)) || (overlap(n, y) && !over(p->n, p->ldn, sy, p->y, p->ldy, sy)) || overlap(h, n) ||
      overlap(stats, h) || overlap(stats, n) || overlap(stats, x) || overlap(stats, y))
    return DS_ERR_INVALID_ARG;
  for (const Span& v : parameters(p).all)      // read by every CTA, whenever it comes to them
    if (overlap(h, v) || overlap(n, v) || overlap(stats, v)) return DS_ERR_INVALID_ARG;
  const NormParams q = params(p, false);
  const NormPlan b = norm_plan(p);
  const cudaError_t e = by_types(p, [&](auto sx_, auto sy_) { return forward<decltype(sx_), decltype(sy_)>(q, b, static_cast<cudaStream_t>(cuda_stream)); });
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "norms around a residual connection");
}

uint64_t ds_norm_backward_workspace(const ds_norm_args* p) {
  if (check(p, true) != DS_OK || p->rows == 0) return 0;
  const NormPlan b = norm_plan(p);
  return b.gate_bytes + b.part_bytes;
}

int ds_norm_backward(const ds_norm_args* p, void* cuda_stream) {
  const int rc = check(p, true);
  if (rc != DS_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  struct { float* to; uint64_t n; } outs[] = {{p->d_post_w, p->cols}, {p->d_post_b, p->cols}, {p->d_gate, p->groups * p->cols}, {p->d_pre_w, p->cols}, {p->d_pre_b, p->cols}};
  if (p->rows == 0) {
    for (auto& o : outs)
      if (o.to && o.n) {
        const cudaError_t e = cudaMemsetAsync(o.to, 0, 4 * o.n, st);
        if (e != cudaSuccess) return cuda_fail(e, "clearing gradients");
      }
    return DS_OK;
  }
  const uint32_t sy = size_of(p->dtype), sx = size_of(p->stream_dtype);
  const NormPlan b = norm_plan(p);
  const uint64_t ws = b.gate_bytes + b.part_bytes;
  if (ws) {
    if (!p->workspace) return DS_ERR_INVALID_ARG;
    if (!aligned(p->workspace, 16)) return DS_ERR_ALIGN;
    if (p->workspace_bytes < ws) return DS_ERR_BUFFER_TOO_SMALL;
  }
  const Span in[] = {span(p->y, p->rows, p->cols, p->ldy, sy), span(p->x, p->rows, p->cols, p->ldx, sx), span(p->dh, p->rows, p->cols, p->lddh, sx),
                       span(p->dn, p->rows, p->cols, p->lddn, sy), span(p->stats, 1, 4 * p->rows, 0, 4)};
  const struct { Span r; const void* p; uint64_t ld; uint32_t size; } to[] = {{span(p->dx, p->rows, p->cols, p->lddx, sx), p->dx, p->lddx, sx},
                                                                                {span(p->dy, p->rows, p->cols, p->lddy, sy), p->dy, p->lddy, sy}};
  const struct { const void* p; uint64_t ld; uint32_t size; } from[] = {{p->y, p->ldy, sy}, {p->x, p->ldx, sx}, {p->dh, p->lddh, sx}, {p->dn, p->lddn, sy}};
  for (auto& t : to) {      // over an input only entry by entry
    for (int i = 0; i < 4; ++i)
      if (overlap(t.r, in[i]) && !(t.p == from[i].p && t.size == from[i].size && (t.ld == from[i].ld || p->rows == 1))) return DS_ERR_INVALID_ARG;
    if (overlap(t.r, in[4])) return DS_ERR_INVALID_ARG;
  }
  if (overlap(to[0].r, to[1].r)) return DS_ERR_INVALID_ARG;
  const Span space = span(p->workspace, 1, ws, 0, 1);
  const Parameters weights = parameters(p);
  for (auto& t : to)
    for (const Span& v : weights.all)
      if (overlap(t.r, v)) return DS_ERR_INVALID_ARG;
  Span small[6];
  int n = 0;
  for (auto& o : outs) small[n++] = span(o.to, 1, o.n, 0, 4);
  small[n++] = space;
  for (int i = 0; i < n; ++i) {
    for (int j = 0; j < i; ++j)
      if (overlap(small[i], small[j])) return DS_ERR_INVALID_ARG;
    for (auto& r : in)
      if (overlap(small[i], r)) return DS_ERR_INVALID_ARG;
    for (auto& t : to)
      if (overlap(small[i], t.r)) return DS_ERR_INVALID_ARG;
    for (const Span& v : weights.all)
      if (overlap(small[i], v)) return DS_ERR_INVALID_ARG;
  }
  NormParams q = params(p, true);
  uint8_t* space_p = static_cast<uint8_t*>(p->workspace);
  q.gate_part = !p->d_gate ? nullptr : b.gate_bytes ? reinterpret_cast<float*>(space_p) : p->d_gate;
  q.at_post_w = q.at_post_b = q.at_pre_w = q.at_pre_b = -1;
  SumsParams s{};
  uint32_t vectors = 0;
  int kinds = 0, sums = 0;
  float* part = reinterpret_cast<float*>(space_p + b.gate_bytes);
  float* outs_p[4] = {p->d_post_w, p->d_post_b, p->d_pre_w, p->d_pre_b};
  int* places[4] = {&q.at_post_w, &q.at_post_b, &q.at_pre_w, &q.at_pre_b};
  for (int i = 0; i < 4; ++i)
    if (outs_p[i] || (i == 0 && p->d_post_b)) *places[i] = kinds++;      // the bias's sums come with the weight's
  q.kinds = (uint32_t)kinds;
  q.part = part;
  for (int i = 0; i < 4; ++i)
    if (outs_p[i]) {
      s.in[sums] = part + (uint64_t)*places[i] * p->cols, s.out[sums] = outs_p[i];
      s.step[sums] = (uint64_t)kinds * p->cols, s.count[sums] = b.teams, s.vectors[sums] = 1;
      ++sums, ++vectors;
    }
  if (b.gate_bytes) {
    s.in[sums] = q.gate_part, s.out[sums] = p->d_gate, s.step[sums] = p->cols, s.count[sums] = b.units_per_group, s.vectors[sums] = (uint32_t)p->groups;
    ++sums, vectors += (uint32_t)p->groups;
  }
  s.cols = (uint32_t)p->cols;
  cudaError_t e = by_types(p, [&](auto sx_, auto sy_) { return backward<decltype(sx_), decltype(sy_)>(q, b, st); });
  if (e == cudaSuccess && vectors) {
    launch_pdl(k_norm_sums, dim3((uint32_t)((p->cols + 31) / 32), vectors), dim3(kSumThreads), st, s);
    count_launches(1);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "gradients of norms around a residual connection");
}

}  // extern "C"
