// What stands between two blocks of a network, row by row:
//
//   u = post(y);  h = a x + D(g u);  n = pre(h)        post, pre: RMS or layer norms;  g: a gate;  D: dropout
//
// and all its gradients.  Bound by memory: x and y are read once and h and n written once, with everything between them in
// registers; backward, h is computed again from x and y (which costs no byte more than reading it would) with the norms'
// statistics that the forward pass left, and what parameters get is summed by CTAs that each take a run of rows, a thread
// its eight columns, and added up in the CTAs' order: nothing depends on timing.
#include "dsq_dropout.cuh"
#include "dsq_rows8.cuh"

using namespace dsq;

namespace {

struct NormParams {
  const void* y;
  const void* x;                 // or NULL
  uint64_t ldy, ldx;
  const float *post_w, *post_b, *gate, *pre_w, *pre_b;      // or NULL
  float residual_scale, eps;
  uint32_t rows, cols, group_rows;      // rows that share a gate
  int layer;                     // layer norms, else RMS
  Drop drop;
  float4* stats;                 // per row: mean and 1/size of y, of h; or NULL
  // forward
  void *h, *n;                   // or NULL
  uint64_t ldh, ldn;
  // backward
  const void *dh, *dn;           // or NULL
  void *dx, *dy;                 // or NULL
  uint64_t lddh, lddn, lddx, lddy;
  float *gate_part;              // sums of every unit of rows (of every gate, where a gate's rows are one unit)
  float *part;                   // sums of every CTA: [grid][kinds][cols]
  uint32_t units, unit_rows, units_per_group;
  uint32_t kinds;                // vectors in `part`
  int at_post_w, at_post_b, at_pre_w, at_pre_b;      // their places, or -1
  int vec;                       // all matrices on 16-byte rows
  int wvec;                      // all vectors on 16-byte boundaries, and cols a multiple of 4
};

// ---- sums over the threads of a row ---------------------------------------------------------------------
// blockDim.x threads (whole warps) have a row, blockDim.y rows are in hand.  K values at once, one barrier: the two halves of `red` take turns.
constexpr int kMostWarps = 32;
template <int K>
struct RowSum {
  float (*red)[kMostWarps][K];      // [2]
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[K]) {
#pragma unroll
    for (int o = 16; o; o >>= 1)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return;
    const int warp = threadIdx.x >> 5, first = threadIdx.y * warps;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) red[turn][first + warp][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = 0.f;
    for (int w = 0; w < warps; ++w)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += red[turn][first + w][k];
    turn ^= 1;
  }
};

// ---- forward --------------------------------------------------------------------------------------------
// A row to blockDim.x threads, NV pieces of eight columns a thread.
template <class X, class Y, int NV>
__global__ void __launch_bounds__(1024) k_norm_forward(const NormParams p) {
  __shared__ float red[2][kMostWarps][1];
  pdl_prologue();
  const uint32_t row = blockIdx.x * blockDim.y + threadIdx.y;
  const bool live = row < p.rows;      // every thread stays for the barriers
  RowSum<1> sum{red};
  const float inv = 1.f / (float)p.cols;
  float v[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const uint32_t c = (threadIdx.x + i * blockDim.x) * 8;
    if (live && c < p.cols)
      load8<Y>(p.y, row * p.ldy, c, p.cols, p.vec, v[i]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
  }
  // mean and 1 / size of the rows in v
  auto statistics = [&](float& mean, float& r) {
    mean = 0.f;
    if (p.layer) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] += v[i][j];
      sum(s);
      mean = s[0] * inv;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t c = (threadIdx.x + i * blockDim.x) * 8;
      if (c + 8 <= p.cols) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = v[i][j] - mean;
          q[0] = __fmaf_rn(d, d, q[0]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = c + j < p.cols ? v[i][j] - mean : 0.f;
          q[0] = __fmaf_rn(d, d, q[0]);
        }
      }
    }
    sum(q);
    r = 1.f / sqrtf(__fmaf_rn(q[0], inv, p.eps));
  };
  float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
  if (p.post_w) statistics(st.x, st.y);
  const float* gate = p.gate ? p.gate + (uint64_t)(row / p.group_rows) * p.cols : nullptr;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const uint32_t c = (threadIdx.x + i * blockDim.x) * 8;
    if (!live || c >= p.cols) continue;
    float t[8];
    if (p.post_w) {
      load8<float>(p.post_w, 0, c, p.cols, p.wvec, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - st.x) * st.y * t[j];
      if (p.post_b) {
        load8<float>(p.post_b, 0, c, p.cols, p.wvec, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += t[j];
      }
    }
    if (gate) {
      load8<float>(gate, 0, c, p.cols, p.wvec, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= t[j];
    }
    if (p.drop.threshold) drop8(p.drop, kept8(p.drop, row, c), v[i]);
    if (p.x) {
      load8<X>(p.x, row * p.ldx, c, p.cols, p.vec, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = __fmaf_rn(p.residual_scale, t[j], v[i][j]);
    }
    if (p.h) store8<X>(p.h, row * p.ldh, c, p.cols, p.vec, v[i]);
  }
  if (p.pre_w) {
    statistics(st.z, st.w);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t c = (threadIdx.x + i * blockDim.x) * 8;
      if (!live || c >= p.cols) continue;
      float t[8];
      load8<float>(p.pre_w, 0, c, p.cols, p.wvec, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - st.z) * st.w * t[j];
      if (p.pre_b) {
        load8<float>(p.pre_b, 0, c, p.cols, p.wvec, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += t[j];
      }
      store8<Y>(p.n, row * p.ldn, c, p.cols, p.vec, v[i]);
    }
  }
  if (live && p.stats && threadIdx.x == 0) p.stats[row] = st;
}

// ---- backward -------------------------------------------------------------------------------------------
//   d = dh + J_pre^T dn;   dx = a d;   q = g D(d);   dy = J_post^T q
//   J^T t = r (w t - mean(w t) - hat mean(w t hat)), the second term for layer norms alone
// A thread has eight columns, blockDim.x threads a part of a row: a whole one, or, above kBackCols columns, its share in a cluster of
// CTAs, which exchange their sums through distributed shared memory.  blockDim.y rows are in hand at once.
constexpr uint32_t kBackCols = 4096, kBackThreads = 512;

template <int K>
struct ClusterSum {
  float (*red)[kMostWarps][K];
  float (*peer)[8][K];              // [2][rank]
  int turn = 0;
  uint32_t rank, size;
  __device__ __forceinline__ void operator()(float (&v)[K]) {
#pragma unroll
    for (int o = 16; o; o >>= 1)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, first = threadIdx.y * warps;
    if (warps > 1 || size > 1) {
      if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) red[turn][first + warp][k] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = 0.f;
      for (int w = 0; w < warps; ++w)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += red[turn][first + w][k];
    }
    if (size > 1) {                 // blockDim.y is 1 here
      if (threadIdx.x < size) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
          uint32_t to;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(&peer[turn][rank][k])), "r"(threadIdx.x));
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(v[k]) : "memory");
        }
      }
      asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = 0.f;
      for (uint32_t r = 0; r < size; ++r)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += peer[turn][r][k];
    }
    turn ^= 1;
  }
};

template <class X, class Y>
__global__ void __launch_bounds__(kBackThreads, 1) k_norm_backward(const NormParams p, const uint32_t size) {
  __shared__ float red[2][kMostWarps][2], peer[2][8][2];
  extern __shared__ float flush[];      // [blockDim.y][blockDim.x * 8]
  pdl_prologue();
  uint32_t rank = 0;
  if (size > 1) {
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // the others are there before their shared memory is written
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  ClusterSum<2> sum{red, peer, 0, rank, size};
  const uint32_t width = blockDim.x * 8, c0 = rank * width, c = c0 + threadIdx.x * 8, team = blockIdx.x / size, teams = gridDim.x / size;
  const float inv = 1.f / (float)p.cols;
  const bool mine = c < p.cols;
  float s_gate[8], s_post_w[8], s_post_b[8], s_pre_w[8], s_pre_b[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) s_gate[j] = s_post_w[j] = s_post_b[j] = s_pre_w[j] = s_pre_b[j] = 0.f;

  // this CTA's sums of one kind, over the rows that were in hand side by side, into a vector
  auto flush_to = [&](float (&s)[8], float* to) {
    if (blockDim.y == 1) {
      if (mine)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < p.cols) to[c + j] = s[j];
    } else {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) flush[threadIdx.y * width + threadIdx.x * 8 + j] = s[j];
      __syncthreads();
      for (uint32_t k = threadIdx.y * blockDim.x + threadIdx.x; k < width; k += blockDim.x * blockDim.y) {
        float v = 0.f;
        for (uint32_t y = 0; y < blockDim.y; ++y) v += flush[y * width + k];
        if (c0 + k < p.cols) to[c0 + k] = v;
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = 0.f;
  };

  for (uint32_t u = team; u < p.units; u += teams) {
    const uint32_t group = u / p.units_per_group, r_end = min((group + 1) * p.group_rows, p.rows);
    const uint32_t first = group * p.group_rows + (u - group * p.units_per_group) * p.unit_rows, last = min(first + p.unit_rows, r_end);
    for (uint32_t r0 = first; r0 < last; r0 += blockDim.y) {
      const uint32_t row = r0 + threadIdx.y;
      const bool live = row < last && mine;
      float hat1[8], d[8], t[8];
      float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
      float x[8];
      if (live) {
        if (p.stats) st = ld_plain(p.stats + row);
        load8<Y>(p.y, row * p.ldy, c, p.cols, p.vec, hat1);
        if (p.x) load8<X>(p.x, row * p.ldx, c, p.cols, p.vec, x);
      }
      if (!live)
#pragma unroll
        for (int j = 0; j < 8; ++j) hat1[j] = 0.f;
      if (!live || !p.x)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
      if (live && p.dh)
        load8<X>(p.dh, row * p.lddh, c, p.cols, p.vec, d);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = 0.f;
      if (live && p.dn)
        load8<Y>(p.dn, row * p.lddn, c, p.cols, p.vec, t);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = 0.f;
      // forward again: v = post(y)
      float v[8], w1[8];
      const uint32_t kept = p.drop.threshold ? kept8(p.drop, row, c) : 0u;
      if (p.post_w) {
        if (live)
          load8<float>(p.post_w, 0, c, p.cols, p.wvec, w1);
        else
#pragma unroll
          for (int j = 0; j < 8; ++j) w1[j] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hat1[j] = (hat1[j] - st.x) * st.y;
          v[j] = hat1[j] * w1[j];
        }
        if (p.post_b && live) {
          float b[8];
          load8<float>(p.post_b, 0, c, p.cols, p.wvec, b);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] += b[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = hat1[j];
      }
      float g[8];
      if (p.gate && live)
        load8<float>(p.gate + (uint64_t)group * p.cols, 0, c, p.cols, p.wvec, g);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 1.f;
      if (p.pre_w) {
        float hat2[8], w2[8], s[2] = {0.f, 0.f};
        if (live)
          load8<float>(p.pre_w, 0, c, p.cols, p.wvec, w2);
        else
#pragma unroll
          for (int j = 0; j < 8; ++j) w2[j] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) hat2[j] = v[j] * g[j];
        if (p.drop.threshold) drop8(p.drop, kept, hat2);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hat2[j] = (__fmaf_rn(p.residual_scale, x[j], hat2[j]) - st.z) * st.w;
          s_pre_w[j] = __fmaf_rn(t[j], hat2[j], s_pre_w[j]);
          s_pre_b[j] += t[j];
          t[j] *= w2[j];
          s[0] += t[j];
          s[1] = __fmaf_rn(t[j], hat2[j], s[1]);
        }
        sum(s);
        const float m = p.layer ? s[0] * inv : 0.f, k = s[1] * inv;
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = __fmaf_rn(st.w, t[j] - m - hat2[j] * k, d[j]);
      }
      if (live && p.dx) {
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = p.residual_scale * d[j];
        store8<X>(p.dx, row * p.lddx, c, p.cols, p.vec, t);
      }
      if (p.drop.threshold) drop8(p.drop, kept, d);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s_gate[j] = __fmaf_rn(d[j], v[j], s_gate[j]);
        d[j] *= g[j];
      }
      if (p.post_w) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          s_post_w[j] = __fmaf_rn(d[j], hat1[j], s_post_w[j]);
          s_post_b[j] += d[j];
          d[j] *= w1[j];
          s[0] += d[j];
          s[1] = __fmaf_rn(d[j], hat1[j], s[1]);
        }
        sum(s);
        const float m = p.layer ? s[0] * inv : 0.f, k = s[1] * inv;
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = st.y * (d[j] - m - hat1[j] * k);
      }
      if (live && p.dy) store8<Y>(p.dy, row * p.lddy, c, p.cols, p.vec, d);
    }
    if (p.gate_part) flush_to(s_gate, p.gate_part + (uint64_t)u * p.cols);
  }
  float* part = p.part + (uint64_t)team * p.kinds * p.cols;
  if (p.at_post_w >= 0) flush_to(s_post_w, part + (uint64_t)p.at_post_w * p.cols);
  if (p.at_post_b >= 0) flush_to(s_post_b, part + (uint64_t)p.at_post_b * p.cols);
  if (p.at_pre_w >= 0) flush_to(s_pre_w, part + (uint64_t)p.at_pre_w * p.cols);
  if (p.at_pre_b >= 0) flush_to(s_pre_b, part + (uint64_t)p.at_pre_b * p.cols);
  if (size > 1) {      // no CTA's shared memory goes away under a neighbour's store
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}

// The CTAs' sums, added in their order: out[v] = sum_i in[v * stride_v + i * stride_i].
struct SumsParams {
  const float* in[5];
  float* out[5];
  uint64_t step[5];       // between what is added
  uint32_t count[5], vectors[5];      // vectors: of this kind (gates: one a group), `count` steps apart
  uint32_t cols;
};
__global__ void __launch_bounds__(256) k_norm_sums(const SumsParams p) {
  __shared__ float part[8][32];
  pdl_prologue();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t col = blockIdx.x * 32 + lane;
  uint32_t v = blockIdx.y, kind = 0;
  while (v >= p.vectors[kind]) v -= p.vectors[kind++];
  const float* in = p.in[kind] + (uint64_t)v * p.count[kind] * p.step[kind];
  float s = 0.f;
  if (col < p.cols)
    for (uint32_t i = warp; i < p.count[kind]; i += 8) s += ld_plain(in + i * p.step[kind] + col);
  part[warp][lane] = s;
  __syncthreads();
  if (warp || col >= p.cols) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) s += part[w][lane];
  p.out[kind][(uint64_t)v * p.cols + col] = s;
}

// ---- host side ------------------------------------------------------------------------------------------

inline uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }
inline bool aligned(const void* p, uint64_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline uint32_t size_of(uint64_t dtype) { return dtype == DS_F32 ? 4 : 2; }
constexpr uint64_t kMaxRows = 1ull << 30;

int sms() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return 148;
  return n;
}

// How the backward pass is cut.
struct BackPlan {
  uint32_t size;              // CTAs of a cluster
  uint32_t tx, ty;            // threads of a row (or of its share), rows in hand
  uint32_t units, unit_rows, units_per_group, teams;
  uint64_t gate_bytes, part_bytes;
};
BackPlan back_plan(const ds_norm_args* p) {
  BackPlan b;
  const uint64_t cols = p->cols, groups = p->groups ? p->groups : 1, group_rows = p->rows / groups;
  b.size = 1;
  while (b.size * (uint64_t)kBackCols < cols) b.size *= 2;
  const uint32_t pieces = (uint32_t)((cols + 8 * b.size - 1) / (8 * b.size));
  b.tx = (uint32_t)round_up(pieces, 32);
  b.ty = b.size > 1 ? 1 : kBackThreads / b.tx;
  if (b.ty > group_rows) b.ty = group_rows ? (uint32_t)group_rows : 1;
  const uint64_t want = (uint64_t)sms() / b.size;      // teams that run at once
  // a group's rows are cut where there are fewer groups than teams, into units of at least one row a slice
  uint64_t per = groups >= want ? 1 : (want + groups - 1) / groups;
  const uint64_t most = (group_rows + b.ty - 1) / b.ty;
  if (per > most) per = most ? most : 1;
  b.unit_rows = (uint32_t)round_up((group_rows + per - 1) / per, b.ty);
  if (!b.unit_rows) b.unit_rows = 1;
  b.units_per_group = group_rows ? (uint32_t)((group_rows + b.unit_rows - 1) / b.unit_rows) : 1;
  b.units = (uint32_t)(b.units_per_group * groups);
  b.teams = b.units < want ? b.units : (uint32_t)want;
  const uint32_t kinds = (p->d_post_w != nullptr) + (p->d_post_b != nullptr) + (p->d_pre_w != nullptr) + (p->d_pre_b != nullptr);
  b.gate_bytes = p->d_gate && b.units_per_group > 1 ? round_up(4ull * b.units * cols, 256) : 0;
  b.part_bytes = 4ull * b.teams * kinds * cols;
  return b;
}

template <class X, class Y>
cudaError_t forward(const NormParams& q, cudaStream_t st) {
  const uint32_t pieces = (q.cols + 7) / 8;
  auto go = [&](auto kernel, uint32_t nv) {
    const uint32_t tx = (uint32_t)round_up((pieces + nv - 1) / nv, 32), ty = tx >= 256 ? 1 : 256 / tx;
    launch_pdl(kernel, dim3((q.rows + ty - 1) / ty), dim3(tx, ty), st, q);
    count_launches(1);
    return cudaGetLastError();
  };
  if (pieces <= 512) return go(k_norm_forward<X, Y, 1>, 1);
  if (pieces <= 1024) return go(k_norm_forward<X, Y, 2>, 2);
  return go(k_norm_forward<X, Y, 4>, 4);
}

template <class X, class Y>
cudaError_t backward(const NormParams& q, const BackPlan& b, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(b.teams * b.size);
  cfg.blockDim = dim3(b.tx, b.ty);
  cfg.dynamicSmemBytes = b.ty > 1 ? b.tx * b.ty * 32 : 0;
  cfg.stream = st;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = b.size;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = b.size > 1 ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, k_norm_backward<X, Y>, q, b.size);
  count_launches(1);
  return cudaGetLastError();
}

template <class F>
cudaError_t by_types(const ds_norm_args* p, F&& f) {
  using H = __half;
  using B = __nv_bfloat16;
  if (p->dtype == DS_F32) return f(float(), float());
  if (p->dtype == DS_BF16) return p->stream_dtype == DS_F32 ? f(float(), B()) : f(B(), B());
  return p->stream_dtype == DS_F32 ? f(float(), H()) : f(H(), H());
}

struct Region {
  uintptr_t p;
  uint64_t bytes;
};
inline Region region(const void* p, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t size) {
  return {reinterpret_cast<uintptr_t>(p), p && rows && cols ? ((rows - 1) * ld + cols) * size : 0};
}
inline bool overlap(const Region& a, const Region& b) { return a.bytes && b.bytes && a.p < b.p + b.bytes && b.p < a.p + a.bytes; }

int check(const ds_norm_args* p, bool back) {
  if (!p || p->dtype > DS_F16 || (p->stream_dtype != p->dtype && p->stream_dtype != DS_F32) || p->norm > DS_NORM_LAYER) return DS_ERR_INVALID_ARG;
  if (p->rows > kMaxRows || p->cols == 0) return DS_ERR_INVALID_ARG;
  if (p->cols > DS_NORM_MAX_COLS) return DS_ERR_UNSUPPORTED;
  if (p->groups && (!p->gate || p->rows % p->groups)) return DS_ERR_INVALID_ARG;
  if (!p->groups && p->gate) return DS_ERR_INVALID_ARG;
  if ((p->post_b && !p->post_w) || (p->pre_b && !p->pre_w)) return DS_ERR_INVALID_ARG;
  if (!(p->eps >= 0) || p->threshold > 65535 || p->layer > 0xFFFFFFFFull || p->step > 0xFFFFFFFFull) return DS_ERR_INVALID_ARG;
  const uint32_t sy = size_of(p->dtype), sx = size_of(p->stream_dtype);
  const void* vectors[] = {p->post_w, p->post_b, p->gate, p->pre_w, p->pre_b, p->d_post_w, p->d_post_b, p->d_gate, p->d_pre_w, p->d_pre_b};
  for (const void* v : vectors)
    if (!aligned(v, 4)) return DS_ERR_ALIGN;
  if (!aligned(p->stats, 16) || !aligned(p->y, sy) || !aligned(p->n, sy) || !aligned(p->dn, sy) || !aligned(p->dy, sy) || !aligned(p->x, sx) || !aligned(p->h, sx) ||
      !aligned(p->dh, sx) || !aligned(p->dx, sx))
    return DS_ERR_ALIGN;
  if (p->rows == 0) return DS_OK;
  if (!p->y) return DS_ERR_INVALID_ARG;
  const bool many = p->rows > 1;
  auto narrow = [&](const void* q, uint64_t ld) { return many && q && ld < p->cols; };
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

NormParams params(const ds_norm_args* p) {
  NormParams q{};
  q.y = p->y, q.x = p->x, q.ldy = p->ldy, q.ldx = p->ldx;
  q.post_w = p->post_w, q.post_b = p->post_b, q.gate = p->gate, q.pre_w = p->pre_w, q.pre_b = p->pre_b;
  q.residual_scale = (float)p->residual_scale, q.eps = (float)p->eps;
  q.rows = (uint32_t)p->rows, q.cols = (uint32_t)p->cols, q.group_rows = (uint32_t)(p->rows / (p->groups ? p->groups : 1));
  q.layer = p->norm == DS_NORM_LAYER;
  q.drop = make_drop((uint32_t)p->threshold, p->seed, (uint32_t)p->layer, (uint32_t)p->step);
  q.stats = reinterpret_cast<float4*>(p->stats);
  bool vec = true;
  auto see = [&](const void* m, uint64_t ld, uint32_t size) { vec = vec && (!m || (aligned(m, 16) && (p->rows == 1 || ld * size % 16 == 0))); };
  const uint32_t sy = size_of(p->dtype), sx = size_of(p->stream_dtype);
  see(p->y, p->ldy, sy), see(p->x, p->ldx, sx), see(p->h, p->ldh, sx), see(p->n, p->ldn, sy);
  see(p->dh, p->lddh, sx), see(p->dn, p->lddn, sy), see(p->dx, p->lddx, sx), see(p->dy, p->lddy, sy);
  q.vec = vec;
  q.wvec = aligned(p->post_w, 16) && aligned(p->post_b, 16) && aligned(p->gate, 16) && aligned(p->pre_w, 16) && aligned(p->pre_b, 16) &&
           (p->groups <= 1 || p->cols % 4 == 0);
  return q;
}

}  // namespace

extern "C" {

int ds_norm_forward(const ds_norm_args* p, void* cuda_stream) {
  const int rc = check(p, false);
  if (rc != DS_OK || p->rows == 0) return rc;
  const uint32_t sy = size_of(p->dtype), sx = size_of(p->stream_dtype);
  const Region y = region(p->y, p->rows, p->cols, p->ldy, sy), x = region(p->x, p->rows, p->cols, p->ldx, sx), h = region(p->h, p->rows, p->cols, p->ldh, sx),
               n = region(p->n, p->rows, p->cols, p->ldn, sy), stats = region(p->stats, 1, 4 * p->rows, 0, 4);
  // a thread reads its entries of x and y before it writes the same ones of h; n comes after them all
  auto over = [&](const void* a, uint64_t lda, uint32_t sa, const void* b, uint64_t ldb, uint32_t sb) { return a == b && sa == sb && (lda == ldb || p->rows == 1); };
  if ((overlap(h, x) && !over(p->h, p->ldh, sx, p->x, p->ldx, sx)) || (overlap(h, y) && !over(p->h, p->ldh, sx, p->y, p->ldy, sy)) ||
      (overlap(n, x) && !over(p->n, p->ldn, sy, p->x, p->ldx, sx)) || (overlap(n, y) && !over(p->n, p->ldn, sy, p->y, p->ldy, sy)) || overlap(h, n) ||
      overlap(stats, h) || overlap(stats, n) || overlap(stats, x) || overlap(stats, y))
    return DS_ERR_INVALID_ARG;
  NormParams q = params(p);
  q.h = p->h, q.ldh = p->ldh, q.n = p->n, q.ldn = p->ldn;
  const cudaError_t e = by_types(p, [&](auto sx_, auto sy_) { return forward<decltype(sx_), decltype(sy_)>(q, static_cast<cudaStream_t>(cuda_stream)); });
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "norms around a residual connection");
}

uint64_t ds_norm_backward_workspace(const ds_norm_args* p) {
  if (check(p, true) != DS_OK || p->rows == 0) return 0;
  const BackPlan b = back_plan(p);
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
  const BackPlan b = back_plan(p);
  const uint64_t ws = b.gate_bytes + b.part_bytes;
  if (ws) {
    if (!p->workspace) return DS_ERR_INVALID_ARG;
    if (!aligned(p->workspace, 16)) return DS_ERR_ALIGN;
    if (p->workspace_bytes < ws) return DS_ERR_BUFFER_TOO_SMALL;
  }
  const Region in[] = {region(p->y, p->rows, p->cols, p->ldy, sy), region(p->x, p->rows, p->cols, p->ldx, sx), region(p->dh, p->rows, p->cols, p->lddh, sx),
                       region(p->dn, p->rows, p->cols, p->lddn, sy), region(p->stats, 1, 4 * p->rows, 0, 4)};
  const struct { Region r; const void* p; uint64_t ld; uint32_t size; } to[] = {{region(p->dx, p->rows, p->cols, p->lddx, sx), p->dx, p->lddx, sx},
                                                                                {region(p->dy, p->rows, p->cols, p->lddy, sy), p->dy, p->lddy, sy}};
  const struct { const void* p; uint64_t ld; uint32_t size; } from[] = {{p->y, p->ldy, sy}, {p->x, p->ldx, sx}, {p->dh, p->lddh, sx}, {p->dn, p->lddn, sy}};
  for (auto& t : to) {      // over an input only entry by entry
    for (int i = 0; i < 4; ++i)
      if (overlap(t.r, in[i]) && !(t.p == from[i].p && t.size == from[i].size && (t.ld == from[i].ld || p->rows == 1))) return DS_ERR_INVALID_ARG;
    if (overlap(t.r, in[4])) return DS_ERR_INVALID_ARG;
  }
  if (overlap(to[0].r, to[1].r)) return DS_ERR_INVALID_ARG;
  const Region space = region(p->workspace, 1, ws, 0, 1);
  const float* weights[] = {p->post_w, p->post_b, p->pre_w, p->pre_b, p->gate};
  Region small[6];
  int n = 0;
  for (auto& o : outs) small[n++] = region(o.to, 1, o.n, 0, 4);
  small[n++] = space;
  for (int i = 0; i < n; ++i) {
    for (int j = 0; j < i; ++j)
      if (overlap(small[i], small[j])) return DS_ERR_INVALID_ARG;
    for (auto& r : in)
      if (overlap(small[i], r)) return DS_ERR_INVALID_ARG;
    for (auto& t : to)
      if (overlap(small[i], t.r)) return DS_ERR_INVALID_ARG;
    for (int j = 0; j < 5; ++j)
      if (overlap(small[i], region(weights[j], 1, j == 4 ? p->groups * p->cols : p->cols, 0, 4))) return DS_ERR_INVALID_ARG;
  }
  NormParams q = params(p);
  q.dh = p->dh, q.dn = p->dn, q.dx = p->dx, q.dy = p->dy;
  q.lddh = p->lddh, q.lddn = p->lddn, q.lddx = p->lddx, q.lddy = p->lddy;
  q.units = b.units, q.unit_rows = b.unit_rows, q.units_per_group = b.units_per_group;
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
    if (outs_p[i]) *places[i] = kinds++;
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
    launch_pdl(k_norm_sums, dim3((uint32_t)((p->cols + 31) / 32), vectors), dim3(256), st, s);
    count_launches(1);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? DS_OK : cuda_fail(e, "gradients of norms around a residual connection");
}

}  // extern "C"
