// The orthogonalised update of small matrices in one launch: X is [m, n], m <= 64, and a cluster of CTAs keeps it in shared
// memory for all steps, each CTA a slice of columns.  Of a step  A = X X^T,  B = b A + c A A,  X = a X + B X  only A needs the
// other slices: the CTAs' sums are added through distributed shared memory, every CTA a share of the rows, and handed to all;
// B is computed by every CTA for itself.  The same goes for the norm.
//
// A launch of the general form costs 3 to 4 us whatever its size, and an update has seventeen of them.  Here a step takes 4 us,
// about a third of it products, a third the exchange of A and a third their latencies: 34 us for four 64 x 576, 62 in the general
// form.  The products are taken in two halves of either operand (hi hi + hi lo + lo hi on 16-bit floats: 22 bits), which small
// matrices need: their roundings do not average out.  The warp instruction m16n8k16 is used, fed from shared memory without
// descriptors, barriers and tensor memory.  The tensor core's own instruction has a tile of 64 rows too; it was not tried here.  (Shorter sides up to 128 were slower than the general form, 77 against 59 us for 128 x 128.)
#include "dsq_mma.cuh"
#include "dsq_orth.cuh"

using namespace dsq;

namespace {

constexpr int kSmallThreads = 512, kSmallWarps = kSmallThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int MP = 64;              // rows of X, those past its end zeros
// (Loops here are unrolled no further than they are written: the whole kernel runs in some ten thousand cycles, and fetching its
// instructions for the first time is a good part of them.  A form with everything unrolled took twice as long.)

__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_cluster2(uint32_t addr, uint32_t a, uint32_t b) {
  asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void st_cluster_f64(uint32_t addr, double v) {
  asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory");
}

// Two floats as hi and lo halves.
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __floats2half2_rn(a, b);
  const float2 r = __half22float2(h);
  const __half2 l = __floats2half2_rn(a - r.x, b - r.y);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  lo = *reinterpret_cast<const uint32_t*>(&l);
}
__device__ __forceinline__ float2 join2(uint32_t hi, uint32_t lo) {
  const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi)), l = __half22float2(*reinterpret_cast<const __half2*>(&lo));
  return make_float2(h.x + l.x, h.y + l.y);
}

// Shared memory of a CTA, in bytes: X hi, X lo [MP][w + 8] halves; A hi, A lo [MP][MP + 8]; and one block that is the CTA's share
// of A in floats [MP][MP + 4], then B hi, B lo.  (Rows 16 bytes longer than a multiple of 32 spread ldmatrix over all banks.)
struct SmallLayout {
  uint32_t w, pitch;      // columns of a slice (a multiple of 16), bytes between rows of X
  static constexpr uint32_t kPitchA = (MP + 8) * 2, kHalfA = MP * kPitchA, kPitchP = (MP + 4) * 4;
  __host__ __device__ explicit SmallLayout(uint32_t w_) : w(w_), pitch((w_ + 8) * 2) {}
  __host__ __device__ uint32_t x_half() const { return MP * pitch; }
  __host__ __device__ uint32_t at_a() const { return 2 * x_half(); }
  __host__ __device__ uint32_t at_p() const { return at_a() + 2 * kHalfA; }
  __host__ __device__ uint32_t bytes() const { return at_p() + 2 * kHalfA; }
};

struct SmallArgs {
  Momentum mo;
  OrthOut to;
  uint32_t rows, cols, m, n, steps, w;
  int tall;
  float a, b, c, eps;
};

template <class T>
__global__ void __launch_bounds__(kSmallThreads, 1) k_orth_small(const SmallArgs p) {
  constexpr int kRowTiles = MP / 16, kHalves = kSmallWarps / kRowTiles, kCols = MP / kHalves, kTiles = kCols / 8;
  constexpr int kChunkTiles = 4, kChunk = kHalves * kChunkTiles * 8;    // 128 columns at a time
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ double sums[kMaxCluster], warp_sum[kSmallWarps];
  pdl_prologue();
  const SmallLayout L(p.w);
  const uint32_t base = smem_u32(dyn), xh = base, xl = base + L.x_half(), ah = base + L.at_a(), al = ah + L.kHalfA, ps = base + L.at_p(),
                 bh = ps, bl = ps + L.kHalfA;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t ctas;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
  const uint32_t rank = cluster_rank(), matrix = blockIdx.x / ctas;
  const uint32_t c0 = rank * p.w, mine = c0 >= p.n ? 0 : min(p.w, p.n - c0);    // columns of X in this slice
  const uint64_t off = (uint64_t)matrix * p.mo.stride;
  const T* g = static_cast<const T*>(p.mo.g) + off;
  float* buf = p.mo.buf ? p.mo.buf + off : nullptr;

  // The slice is `lines` runs of `run` consecutive entries in memory, `apart` entries from one to the next: pieces of the rows of X, or,
  // where X = u^T, whole rows of u, each a column of X.
  const uint32_t lines = p.tall ? mine : p.m, run = p.tall ? p.m : mine, apart = p.tall ? p.m : p.n;
  const uint64_t start = p.tall ? (uint64_t)c0 * p.m : c0;
  const uint32_t x_line = p.tall ? 2 : L.pitch, x_entry = p.tall ? L.pitch : 2;       // bytes between the same in X
  // visits (line, entry) pairs: a warp takes four lines at a time, so that their loads run together
  auto visit = [&](auto&& load, auto&& use) {
#pragma unroll 1
    for (uint32_t l0 = warp * 4; l0 < lines; l0 += kSmallWarps * 4)
#pragma unroll 1
      for (uint32_t i = lane; i < run; i += 32) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (l0 + q < lines) load(q, start + (uint64_t)(l0 + q) * apart + i);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (l0 + q < lines) use(q, start + (uint64_t)(l0 + q) * apart + i, (l0 + q) * x_line + i * x_entry);
      }
  };

  // momentum and norm
  double sum = 0;
  float gv[4], bv[4];
  auto load = [&](int q, uint64_t at) {
    gv[q] = to_f32(g[at]);
    if (buf) bv[q] = buf[at];
  };
  visit(load, [&](int q, uint64_t at, uint32_t) {
    float u = gv[q];
    if (buf) {
      const float v = p.mo.update(u, bv[q]);
      buf[at] = v;
      u = p.mo.direction(u, v);
    }
    sum += (double)u * (double)u;
  });
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) warp_sum[warp] = sum;
  // X starts as zeros: rows and columns past the end stay so
  for (uint32_t i = tid; i < L.at_a() / 16; i += kSmallThreads) reinterpret_cast<uint4*>(dyn)[i] = make_uint4(0, 0, 0, 0);
  cluster_sync();          // every CTA of the cluster runs: its shared memory may be written
  if (tid < (int)ctas) {
    double s = 0;
    for (int i = 0; i < kSmallWarps; ++i) s += warp_sum[i];
    st_cluster_f64(in_cta(smem_u32(&sums[rank]), tid), s);
  }
  cluster_sync();
  double norm2 = 0;
  for (uint32_t i = 0; i < ctas; ++i) norm2 += sums[i];
  const NormFactor scale(norm2, p.eps);
  visit(load, [&](int q, uint64_t, uint32_t at_x) {
    const float v = scale(buf ? p.mo.direction(gv[q], bv[q]) : gv[q]);
    const __half h = __float2half_rn(v);
    *reinterpret_cast<__half*>(dyn + at_x) = h;
    *reinterpret_cast<__half*>(dyn + L.x_half() + at_x) = __float2half_rn(v - __half2float(h));
  });
  __syncthreads();

  const int rt = warp % kRowTiles, half = warp / kRowTiles;
  const uint32_t a_row = rt * 16 + (lane & 15), a_k = (lane >> 4) * 8;                       // ldmatrix places: an operand's rows
  const uint32_t b_row = (lane & 7) + ((lane >> 4) << 3), b_k = ((lane >> 3) & 1) * 8;       // the other's, laid out along K
  const uint32_t t_k = lane & 15, t_n = (lane >> 4) * 8;                                     // the other's, across K
  const int er = lane >> 2, ec = 2 * (lane & 3);                                             // accumulators: rows er, er + 8

#pragma unroll 1
  for (uint32_t step = 0; step < p.steps; ++step) {
    // first this slice's share of A = X X^T, then A A: the same sums over other rows
#pragma unroll 1
    for (int second = 0; second < 2; ++second) {
      const uint32_t oh = second ? ah : xh, ol = second ? al : xl, pitch = second ? L.kPitchA : L.pitch, len = second ? MP : p.w;
      float acc[kTiles][4] = {};
#pragma unroll 1
      for (uint32_t k = 0; k < len; k += 16) {
        uint32_t fh[4], fl[4];
        ldsm(fh, oh + a_row * pitch + 2 * (k + a_k));
        ldsm(fl, ol + a_row * pitch + 2 * (k + a_k));
#pragma unroll
        for (int j = 0; j < kTiles; j += 2) {
          uint32_t gh[4], gl[4];
          const uint32_t at = (half * kCols + j * 8 + b_row) * pitch + 2 * (k + b_k);
          ldsm(gh, oh + at);
          ldsm(gl, ol + at);
#pragma unroll
          for (int q = 0; q < 2; ++q) mma_f16(acc[j + q], fl, gh[2 * q], gh[2 * q + 1]);
#pragma unroll
          for (int q = 0; q < 2; ++q) mma_f16(acc[j + q], fh, gl[2 * q], gl[2 * q + 1]);
#pragma unroll
          for (int q = 0; q < 2; ++q) mma_f16(acc[j + q], fh, gh[2 * q], gh[2 * q + 1]);
        }
      }
      if (second) {   // B = b A + c A A
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const uint32_t at = (rt * 16 + er + 8 * q) * L.kPitchA + 2 * (half * kCols + j * 8 + ec);
            const float2 v = join2(*reinterpret_cast<const uint32_t*>(dyn + L.at_a() + at), *reinterpret_cast<const uint32_t*>(dyn + L.at_a() + L.kHalfA + at));
            uint32_t h, l;
            split2(fmaf(p.c, acc[j][2 * q] * kDown, p.b * v.x), fmaf(p.c, acc[j][2 * q + 1] * kDown, p.b * v.y), h, l);
            *reinterpret_cast<uint32_t*>(dyn + L.at_p() + at) = h;
            *reinterpret_cast<uint32_t*>(dyn + L.at_p() + L.kHalfA + at) = l;
          }
        __syncthreads();
        break;
      }
#pragma unroll
      for (int j = 0; j < kTiles; ++j) {
        float* to = reinterpret_cast<float*>(dyn + L.at_p() + (rt * 16 + er) * L.kPitchP) + half * kCols + j * 8 + ec;
        *reinterpret_cast<float2*>(to) = make_float2(acc[j][0], acc[j][1]);
        *reinterpret_cast<float2*>(reinterpret_cast<uint8_t*>(to) + 8 * L.kPitchP) = make_float2(acc[j][2], acc[j][3]);
      }
      cluster_sync();
      // rows rank, rank + ctas, ... of the sum, in the order of the ranks, to every CTA
      const uint32_t share = (MP - rank + ctas - 1) / ctas;
#pragma unroll 1
      for (uint32_t i = tid; i < share * (MP / 4); i += kSmallThreads) {
        const uint32_t r = rank + (i / (MP / 4)) * ctas, c = i % (MP / 4) * 4, from = ps + r * L.kPitchP + 4 * c;
        float4 v[kMaxCluster], s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (uint32_t q = 0; q < kMaxCluster; ++q)
          if (q < ctas) v[q] = ld_cluster4(in_cta(from, q));
#pragma unroll
        for (uint32_t q = 0; q < kMaxCluster; ++q)
          if (q < ctas) s.x += v[q].x, s.y += v[q].y, s.z += v[q].z, s.w += v[q].w;
        uint32_t h0, h1, l0, l1;
        split2(s.x * kDown, s.y * kDown, h0, l0);
        split2(s.z * kDown, s.w * kDown, h1, l1);
        const uint32_t to = ah + r * L.kPitchA + 2 * c;
#pragma unroll 1
        for (uint32_t q = 0; q < ctas; ++q) {
          st_cluster2(in_cta(to, q), h0, h1);
          st_cluster2(in_cta(to + L.kHalfA, q), l0, l1);
        }
      }
      cluster_sync();
    }
    // X = a X + B X, some columns at a time: they depend on themselves alone
#pragma unroll 1
    for (uint32_t c1 = 0; c1 < p.w; c1 += kChunk) {
      const uint32_t first = c1 + half * (kChunkTiles * 8);
      float acc[kChunkTiles][4] = {};
      if (first < p.w) {
#pragma unroll 1
        for (uint32_t k = 0; k < MP; k += 16) {
          uint32_t fh[4], fl[4];
          ldsm(fh, bh + a_row * L.kPitchA + 2 * (k + a_k));
          ldsm(fl, bl + a_row * L.kPitchA + 2 * (k + a_k));
#pragma unroll
          for (int j = 0; j < kChunkTiles; j += 2) {
            if (first + 8 * j >= p.w) continue;       // w is a multiple of 16: both tiles or none
            uint32_t gh[4], gl[4];
            const uint32_t at = (k + t_k) * L.pitch + 2 * (first + 8 * j + t_n);
            ldsm_t(gh, xh + at);
            ldsm_t(gl, xl + at);
#pragma unroll
            for (int q = 0; q < 2; ++q) mma_f16(acc[j + q], fl, gh[2 * q], gh[2 * q + 1]);
#pragma unroll
            for (int q = 0; q < 2; ++q) mma_f16(acc[j + q], fh, gl[2 * q], gl[2 * q + 1]);
#pragma unroll
            for (int q = 0; q < 2; ++q) mma_f16(acc[j + q], fh, gh[2 * q], gh[2 * q + 1]);
          }
        }
      }
      __syncthreads();     // everybody has read these columns
#pragma unroll
      for (int j = 0; j < kChunkTiles; ++j) {
        if (first + 8 * j >= p.w) continue;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const uint32_t at = (rt * 16 + er + 8 * q) * L.pitch + 2 * (first + 8 * j + ec);
          uint32_t* ph = reinterpret_cast<uint32_t*>(dyn + at);
          uint32_t* pl = reinterpret_cast<uint32_t*>(dyn + L.x_half() + at);
          const float2 v = join2(*ph, *pl);
          split2(fmaf(p.a, v.x, acc[j][2 * q] * kDown), fmaf(p.a, v.y, acc[j][2 * q + 1] * kDown), *ph, *pl);
        }
      }
    }
    __syncthreads();
  }

  float xv[4];
  visit([&](int q, uint64_t at) { xv[q] = p.to.x ? p.to.x[(uint64_t)matrix * p.to.x_stride + at] : 0.f; },
        [&](int q, uint64_t at, uint32_t at_x) {
          const float v = (__half2float(*reinterpret_cast<const __half*>(dyn + at_x)) +
                           __half2float(*reinterpret_cast<const __half*>(dyn + L.x_half() + at_x))) * kDown;
          const uint64_t o = (uint64_t)matrix * p.rows * p.cols + at;
          if (p.to.out) {
            if (p.to.dtype == DS_BF16)
              static_cast<__nv_bfloat16*>(p.to.out)[o] = __float2bfloat16_rn(v);
            else
              static_cast<float*>(p.to.out)[o] = v;
          }
          if (p.to.x) p.to.x[(uint64_t)matrix * p.to.x_stride + at] = __fsub_rn(__fmul_rn(p.to.keep, xv[q]), __fmul_rn(p.to.rate, v));
        });
}

uint32_t slice(uint32_t n, uint32_t ctas) { return ((n + ctas - 1) / ctas + 15) / 16 * 16; }
constexpr uint32_t kSmallSmem = 225 * 1024;
template <class T>
cudaError_t launch(const SmallArgs& a, uint32_t ctas, uint32_t batch, cudaStream_t st) {
  allow_smem_for<k_orth_small<T>>(kSmallSmem);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(ctas * batch);
  cfg.blockDim = dim3(kSmallThreads);
  cfg.dynamicSmemBytes = SmallLayout(a.w).bytes();
  cfg.stream = st;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, k_orth_small<T>, a);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace

namespace dsq {

// Matrices of up to 64 x 2048 take this form, as many CTAs each as the estimate finds best: slices of 32, 64, 80, 128, 256, 512
// columns took 21, 26, 34, 38, 58 and 98 us for one wave of clusters.  Longer ones are faster in the general form (64 x 2048:
// 58 here, 72 there; 64 x 3000: 78 and 79; 64 x 4096: 98 and 76).  The batch does not decide: a few matrices are faster here (16 of 64 x 576: 44 us, 63 there), many
// about the same (400: 344 and 366; 2000 of 64 x 64: 368 and 313; 4000 of 16 x 16: 537 and 443), and these are the sizes that
// need two halves: with the batch deciding, the same matrix came out a thousandfold less exact in a larger batch.
constexpr uint32_t kSmallLength = 2048;
uint32_t orth_small_ctas(uint32_t m, uint32_t n, uint32_t batch) {
  if (m > MP || n > kSmallLength) return 0;
  double least = 1e30;
  uint32_t best = 0;
  for (uint32_t c = 1; c <= kMaxCluster; c *= 2) {
    const uint32_t w = slice(n, c), at_once = c == 1 ? (uint32_t)sm_count() : (uint32_t)cluster_count(c);
    if (SmallLayout(w).bytes() > kSmallSmem || at_once == 0) continue;
    const double t = (double)((batch + at_once - 1) / at_once) * (16 + 0.16 * w + (c > 1 ? 5 : 0));
    if (t < least) least = t, best = c;
  }
  return best;
}

cudaError_t launch_orth_small(const ds_orth_config& c, uint32_t ctas, const Momentum& mo, int g_dtype, const OrthOut& o, cudaStream_t st) {
  SmallArgs a{};
  a.mo = mo;
  a.to = o;
  a.rows = c.rows;
  a.cols = c.cols;
  a.tall = c.rows > c.cols;
  a.m = a.tall ? c.cols : c.rows;
  a.n = a.tall ? c.rows : c.cols;
  a.steps = c.steps;
  a.w = slice(a.n, ctas);
  a.a = c.a;
  a.b = c.b;
  a.c = c.c;
  a.eps = c.eps;
  return g_dtype == DS_F32    ? launch<float>(a, ctas, c.batch, st)
         : g_dtype == DS_BF16 ? launch<__nv_bfloat16>(a, ctas, c.batch, st)
                              : launch<__half>(a, ctas, c.batch, st);
}

}  // namespace dsq
