// Eight neighbouring entries of a row, as floats: rows may start anywhere.  Memory is read and written in whole 16-byte granules; a warp holds 256 neighbouring
// entries, eight a lane, and where a row starts `shift` bytes behind a boundary a lane takes what it lacks from the granule behind its own, or hands over
// the end of its own to the next lane.  (Entry by entry, a warp's 2-byte accesses touch every sector eight times: dropout of 16384 x 8191 in bf16 took 314 us
// so, and 120 with 8192 columns.)  A granule is read only if it holds an entry of the row; what else it holds is dropped.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "dsq_internal.h"

namespace dsq {

// Whether the rows of two matrices share memory: `rows` of `bytes` bytes, `ld` apart.  Rows that lie side by side in wider ones
// (columns of one buffer) do not, nor does a single row (whose ld is not read) between wider ones.
struct Span {
  uintptr_t p;
  uint64_t rows, bytes, ld;
};
inline Span span(const void* p, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t size) {
  return {reinterpret_cast<uintptr_t>(p), rows, cols * size, ld * size};
}
inline bool overlap(const Span& a, const Span& b) {
  if (b.rows == 1 && a.rows != 1) return overlap(b, a);
  if (!a.p || !b.p || !a.rows || !b.rows || !a.bytes || !b.bytes) return false;
  if (a.p >= b.p + (b.rows - 1) * b.ld + b.bytes || b.p >= a.p + (a.rows - 1) * a.ld + a.bytes) return false;
  if (b.rows == 1 || !b.ld || (a.rows != 1 && a.ld != b.ld)) return true;
  const uint64_t off = a.p >= b.p ? (a.p - b.p) % b.ld : (b.ld - (b.p - a.p) % b.ld) % b.ld;      // of a's row within b's rows
  return off < b.bytes || off + a.bytes > b.ld;
}

template <class T>
__device__ __forceinline__ float to_float(T v) {
  if constexpr (std::is_same<T, float>::value) return v;
  else if constexpr (std::is_same<T, __half>::value) return __half2float(v);
  else return __bfloat162float(v);
}
template <class T>
__device__ __forceinline__ T from_float(float v) {
  if constexpr (std::is_same<T, float>::value) return v;
  else if constexpr (std::is_same<T, __half>::value) return __float2half_rn(v);
  else return __float2bfloat16_rn(v);
}
// Words of eight entries.
template <class T>
constexpr int kWords = 2 * sizeof(T);
template <class T>
__device__ __forceinline__ void unpack8(const uint32_t* w, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
      }
    }
  }
}
template <class T>
__device__ __forceinline__ void pack8(const float (&v)[8], uint32_t* w) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      } else {
        const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
  }
}

// w[0..N): the bytes from `shift` on (0..15, a multiple of the entries' size).  LONG: and in w[N..N + 4) what follows, zeros behind the last word.
template <int N, bool LONG = false>
__device__ __forceinline__ void take_from(uint32_t (&w)[N + 4], uint32_t shift) {
  constexpr int L = LONG ? N + 4 : N;
  auto at = [&](int i) { return i < N + 4 ? w[i] : 0u; };
  if (shift & 8)
#pragma unroll
    for (int i = 0; i < (LONG ? L : N + 2); ++i) w[i] = at(i + 2);
  if (shift & 4)
#pragma unroll
    for (int i = 0; i < (LONG ? L : N + 1); ++i) w[i] = at(i + 1);
  if (shift & 2)
#pragma unroll
    for (int i = 0; i < L; ++i) w[i] = __funnelshift_r(w[i], at(i + 1), 16);
}

__device__ __forceinline__ uint32_t shift_of(const void* row) { return (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15); }

// Entries from c on, not counted far: so that bytes fit into 32 bits.
__device__ __forceinline__ int entries_left(uint32_t c, uint32_t cols) {
  const int left = (int)(cols - c);
  return left < 4096 ? left : 4096;
}

// Entries c .. c + 7 of a row of `cols`, lane l of a whole warp those 8 l behind lane 0's.  Entries behind the row's end are 0.
// VEC: kWhole (true): every row starts on a 16-byte boundary and cols is a multiple of 8; kAligned: rows start so; else anywhere.  First as words, for loads that run ahead of
// their use: nothing in them waits (a lane's exchange with the next one does).
constexpr int kAnywhere = 0, kWhole = 1, kAligned = 2;
template <int VEC, class T>
__device__ __forceinline__ void load_words8(const T* row, uint32_t c, uint32_t cols, int lane, uint32_t (&w)[kWords<T> + 4]) {
  constexpr int N = kWords<T>;
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = 0;
  const uint32_t shift = VEC ? 0 : shift_of(row);
  const uint8_t* at = reinterpret_cast<const uint8_t*>(row + c) - shift;
  // the granules that hold something of this row
  const int bytes = VEC == kWhole ? (c < cols ? 4 * N : 0) : entries_left(c, cols) * (int)sizeof(T) + (int)shift;
#pragma unroll
  for (int g = 0; g < N / 4; ++g)
    if (16 * g < bytes) {
      const uint4 q = ld_plain(reinterpret_cast<const uint4*>(at) + g);
      w[4 * g] = q.x, w[4 * g + 1] = q.y, w[4 * g + 2] = q.z, w[4 * g + 3] = q.w;
    }
  if (!VEC && lane == 31 && shift && 4 * N < bytes) {
    const uint4 q = ld_plain(reinterpret_cast<const uint4*>(at) + N / 4);
    w[N] = q.x, w[N + 1] = q.y, w[N + 2] = q.z, w[N + 3] = q.w;
  }
}
// Then as floats: the whole warp together.
template <int VEC, class T>
__device__ __forceinline__ void entries8(const T* row, uint32_t (&w)[kWords<T> + 4], uint32_t c, uint32_t cols, int lane, float (&v)[8]) {
  constexpr int N = kWords<T>;
  if constexpr (VEC == kAnywhere) {
    const uint32_t shift = shift_of(row);
    if (shift) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t next = __shfl_down_sync(0xFFFFFFFFu, w[i], 1);
        if (lane != 31) w[N + i] = next;
      }
      take_from<N>(w, shift);
    }
  }
  unpack8<T>(w, v);
  if (VEC != kWhole && c + 8 > cols)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j >= cols) v[j] = 0.f;
}
template <int VEC, class T>
__device__ __forceinline__ void load_row8(const T* row, uint32_t c, uint32_t cols, int lane, float (&v)[8]) {
  uint32_t w[kWords<T> + 4];
  load_words8<VEC>(row, c, cols, lane, w);
  entries8<VEC>(row, w, c, cols, lane, v);
}

// Eight entries to where they fit whole: a boundary of 16 bytes, for floats of 32 if `at` is on one.
template <class T>
__device__ __forceinline__ void store_piece8(T* at, const float (&v)[8]) {
  constexpr int N = kWords<T>;
  uint32_t w[N];
  pack8<T>(v, w);
  if (sizeof(T) == 4 && (reinterpret_cast<uintptr_t>(at) & 16) == 0) {      // a whole sector at once
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[N - 4]), "r"(w[N - 3]), "r"(w[N - 2]),
                 "r"(w[N - 1])
                 : "memory");
    return;
  }
#pragma unroll
  for (int g = 0; g < N / 4; ++g) reinterpret_cast<uint4*>(at)[g] = make_uint4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]);
}

// The other way round.  The whole warp calls it, lanes behind the row's end, too.
template <int VEC, class T>
__device__ __forceinline__ void store_row8(T* row, uint32_t c, uint32_t cols, int lane, const float (&v)[8]) {
  constexpr int N = kWords<T>, kEach = 16 / sizeof(T);
  uint32_t w[N + 4];
  if constexpr (VEC == kWhole) {
    if (c < cols) store_piece8(row + c, v);
    return;
  }
  const uint32_t shift = VEC ? 0 : shift_of(row);
  const int left = entries_left(c, cols) * (int)sizeof(T);      // bytes of the row from entry c on
  if (VEC || !shift) {
    pack8<T>(v, w);
    uint4* to = reinterpret_cast<uint4*>(row + c);
#pragma unroll
    for (int g = 0; g < N / 4; ++g)
      if (16 * (g + 1) <= left) {
        to[g] = make_uint4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]);
      } else if (16 * g < left) {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
          if (c + g * kEach + j < cols) row[c + g * kEach + j] = from_float<T>(v[g * kEach + j]);
      }
    return;
  }
  // granule g holds `shift` bytes of what comes before it (of the lane before, for the first one), then this lane's
  pack8<T>(v, w + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __shfl_up_sync(0xFFFFFFFFu, w[N + i], 1);
  take_from<N, true>(w, 16 - shift);      // w[N..]: what this lane hands over
  uint8_t* at = reinterpret_cast<uint8_t*>(row + c) - shift;
  const int s = (int)shift;
  auto put = [&](int i, uint32_t word, int byte) {      // the entry at byte i of the granules
    if constexpr (sizeof(T) == 4)
      *reinterpret_cast<uint32_t*>(at + i) = word;
    else
      *reinterpret_cast<uint16_t*>(at + i) = (uint16_t)(byte ? word >> 16 : word);
  };
  const bool ends = left - 8 * (31 - lane) * (int)sizeof(T) < 4 * N;      // the row ends before or within the last lane's entries
#pragma unroll
  for (int g = 0; g < N / 4; ++g) {
    if ((g || lane) && (!ends || 16 * (g + 1) - s <= left)) {
      reinterpret_cast<uint4*>(at)[g] = make_uint4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]);
    } else if (ends && 16 * g - s < left) {      // the row's end, or what begins a warp
#pragma unroll
      for (int i = 16 * g; i < 16 * g + 16; i += sizeof(T))
        if (i - s < left && (lane || i >= s)) put(i, w[i / 4], i & 2);
    }
  }
  if (!ends && (lane == 0 || lane == 31)) {      // the first lane's own part of its first granule, and what the last lane would hand over
    const int from = lane ? 4 * N : 0;
#pragma unroll
    for (int i = 0; i < 16; i += sizeof(T))
      if (lane ? i < s : i >= s) put(from + i, lane ? w[N + i / 4] : w[i / 4], i & 2);
  }
  if (ends && lane == 31)
#pragma unroll
    for (int i = 0; i < 16; i += sizeof(T))
      if (i < s && 4 * N + i - s < left) put(4 * N + i, w[N + i / 4], i & 2);
}

// Whether rows of a matrix start on 16-byte boundaries (or it is not there).
inline bool rows_on_boundary(const void* p, uint64_t ld, uint64_t rows, uint32_t size) {
  return !p || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && (rows <= 1 || ld * size % 16 == 0));
}

}  // namespace dsq
