// Rows of tokens, entries and experts, read and written 16 bytes a lane: what the kernels that gather, add up and scatter whole rows share (kernels_embed.h, kernels_route.h, kernels_order.h).
//
// A row has M elements at element alignment and a lane the n of 16 bytes, from its column on.  Three ways to deal with the row's end (Lines):
//   wide     rows of more than half a wave: a wave has one row, which the compiler knows (addresses of its arrays are scalar, what a token's index leads to is read once a wave).  The last lane's 16
//            bytes begin where they end with the row: it computes what its neighbour does for some of them, from the same values in the same order, and both write the same bits.
//   narrow   the same with several rows a wave.
//   exact    rows shorter than 16 bytes, and those that do not divide by them where results are added to what is there (nothing may be added twice): each lane its own elements.
// Branches at a row's end would cost more than the work does: a load in a branch is waited for there, and code for single elements in every loop fills the instruction cache (rows of 8192 for 16384
// tokens, us: 172 with vector addresses and such branches, 76 without).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernels_basic.h"
#include "mfma_common.h"
#include "tokens.h"

namespace gspmd {

enum Lines { kExact, kNarrow, kWide };

template <typename T> struct Sixteen;          // 16 bytes as float32, back with one rounding, and back the very bits of opened ones
template <> struct Sixteen<bf16_bits> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void open(u32x4_t v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
  }
  static __device__ __forceinline__ u32x4_t close(const float (&f)[8]) {
    typedef __attribute__((ext_vector_type(8))) float float8_t;
    float8_t v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = f[i];
    return __builtin_bit_cast(u32x4_t, __builtin_convertvector(v, bf16x8_t));
  }
  static __device__ __forceinline__ u32x4_t bits(const float (&f)[8]) {
    u32x4_t v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[2 * i]) >> 16 | (__float_as_uint(f[2 * i + 1]) & 0xffff0000u);
    return v;
  }
};
template <> struct Sixteen<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void open(u32x4_t v, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  }
  static __device__ __forceinline__ u32x4_t close(const float (&f)[4]) {
    u32x4_t v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
    return v;
  }
  static __device__ __forceinline__ u32x4_t bits(const float (&f)[4]) { return close(f); }
};
template <typename T> struct AnyAligned;
template <> struct AnyAligned<bf16_bits> {
  typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
  typedef uint32_t two __attribute__((ext_vector_type(2), aligned(2)));
  typedef uint32_t one __attribute__((aligned(2)));
};
template <> struct AnyAligned<float> {
  typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint32_t two __attribute__((ext_vector_type(2), aligned(4)));
  typedef uint32_t one;
};
template <typename T> __device__ __forceinline__ u32x4_t load16(const T* p) { return *(GSPMD_GLOBAL const typename AnyAligned<T>::type*)p; }
template <typename T> __device__ __forceinline__ void store16(T* p, u32x4_t v) { *(GSPMD_GLOBAL typename AnyAligned<T>::type*)p = v; }
// the first `count` elements of 16 bytes, zeros behind them; count: 0 .. n - 1
template <typename T> __device__ __forceinline__ u32x4_t load_some(const T* p, int count) {
  typedef typename AnyAligned<T>::two two;
  typedef typename AnyAligned<T>::one one;
  const int words = sizeof(T) == 2 ? count >> 1 : count;
  u32x4_t v = {0u, 0u, 0u, 0u};
  if (words & 2) {
    const two w = *(GSPMD_GLOBAL const two*)p;
    v[0] = w[0];
    v[1] = w[1];
  }
  if (words & 1) {
    const uint32_t w = *(GSPMD_GLOBAL const one*)(p + (words & 2) * (4 / sizeof(T)));
    if (words & 2) v[2] = w;
    else v[0] = w;
  }
  if constexpr (sizeof(T) == 2) {
    if (count & 1) {
      const uint32_t w = *((GSPMD_GLOBAL const uint16_t*)p + (count - 1));
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] |= words == i ? w : 0u;
    }
  }
  return v;
}
template <typename T> __device__ __forceinline__ void store_some(T* p, u32x4_t v, int count) {
  typedef typename AnyAligned<T>::two two;
  typedef typename AnyAligned<T>::one one;
  const int words = sizeof(T) == 2 ? count >> 1 : count;
  if (words & 2) *(GSPMD_GLOBAL two*)p = two{v[0], v[1]};
  if (words & 1) *(GSPMD_GLOBAL one*)(p + (words & 2) * (4 / sizeof(T))) = words & 2 ? v[2] : v[0];
  if constexpr (sizeof(T) == 2) {
    if (count & 1) {
      uint32_t w = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w = words == i ? v[i] : w;
      *((GSPMD_GLOBAL uint16_t*)p + (count - 1)) = static_cast<uint16_t>(w);
    }
  }
}
template <typename T> __device__ __forceinline__ u32x4_t load_up_to(const T* p, int count) { return count >= Sixteen<T>::n ? load16(p) : load_some(p, count); }
template <typename T> __device__ __forceinline__ void store_up_to(T* p, u32x4_t v, int count) {
  if (count >= Sixteen<T>::n) store16(p, v);
  else store_some(p, v, count);
}

// Where a lane's 16 bytes of a row begin, and the loads and stores there.  (Of a lane behind the row's end: the row's last ones, to be read, not to be written.)
template <int LINES, typename T> __device__ __forceinline__ int line_at(int col, int M) { return LINES == kExact ? col : min(col, M - Sixteen<T>::n); }
template <int LINES, typename T> __device__ __forceinline__ u32x4_t load_line(const T* row, int at, int M) { return LINES == kExact ? load_up_to(row + at, max(M - at, 0)) : load16(row + at); }
template <int LINES, typename T> __device__ __forceinline__ void store_line(T* row, int at, int M, u32x4_t v) {
  if constexpr (LINES == kExact) store_up_to(row + at, v, M - at);
  else store16(row + at, v);
}
// the same of float32 sums, n of them
template <int LINES, int n> __device__ __forceinline__ void load_sums(const float* row, int at, int M, float (&f)[n]) {
  typedef float four __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int i = 0; i < n; i += 4) {
    if constexpr (LINES == kExact) {
#pragma unroll
      for (int e = i; e < i + 4; ++e) f[e] = at + e < M ? ((GSPMD_GLOBAL const float*)row)[at + e] : 0.f;
    } else {
      const four v = *(GSPMD_GLOBAL const four*)(row + at + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[i + e] = v[e];
    }
  }
}
template <int LINES, int n> __device__ __forceinline__ void store_sums(float* row, int at, int M, const float (&f)[n]) {
  typedef float four __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int i = 0; i < n; i += 4) {
    if constexpr (LINES == kExact) {
#pragma unroll
      for (int e = i; e < i + 4; ++e)
        if (at + e < M) ((GSPMD_GLOBAL float*)row)[at + e] = f[e];
    } else {
      *(GSPMD_GLOBAL four*)(row + at + i) = four{f[i], f[i + 1], f[i + 2], f[i + 3]};
    }
  }
}

// How many lanes a row of `elements` takes: a power of two, up to a wave.
__host__ __device__ __forceinline__ int row_lanes_log(int elements, int per_lane) {
  int log = 0;
  while (log < 6 && (per_lane << log) < elements) ++log;
  return log;
}
template <typename T> inline Lines lines_of(int64_t M) { return M < Sixteen<T>::n ? kExact : row_lanes_log(static_cast<int>(M), Sixteen<T>::n) < 6 ? kNarrow : kWide; }
// a launch by them: go(lines), a compile-time constant
template <typename Go>
inline int32_t by_lines(Lines lines, Go go) {
  switch (lines) {
    case kExact: go(std::integral_constant<int, kExact>{}); break;
    case kNarrow: go(std::integral_constant<int, kNarrow>{}); break;
    default: go(std::integral_constant<int, kWide>{});
  }
  return launched();
}
// a value that all lanes have when a wave has one row
template <int LINES> __device__ __forceinline__ int of_row(int v) { return LINES == kWide ? __builtin_amdgcn_readfirstlane(v) : v; }

}  // namespace gspmd
