// The losses over a split vocabulary for a handful of tokens (softmax.hip): the products with the vocabulary matrix as streams through it, in vector instructions.
//
// With T tokens every element of w takes T multiply-adds for its logits, and 2 T for its gradient and what it adds to dx, which fit beside the stream for a few of them: no matrix
// instruction, no padding to a tile of tokens, no copy of x or w for its alignment, D stays float32, and dw and dx come of one pass.  Logits read w once; the gradients read it once more and write
// dw, D coming from where the logits were.  Bound by memory; a thread takes 16 bytes of w at any element alignment, several rows on their way at a time.
// Measured (us; logits, gradients): float32 [V, M] 4096 x 16000, 1 token 71, 88 (262 MB; 524 MB: 6.0 TB/s), 8 tokens 81, 95; [M, V] 4 tokens 78, 95; bfloat16 [V, M] 655 x 10345, 4 tokens 9.4, 16.6.
//
// NT: tokens that the code provides for (the last of them may be missing: what is made for them is not stored, their D is 0).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernels_basic.h"
#include "kernels_softmax.h"
#include "mfma_common.h"

namespace gspmd {

constexpr int kFewWindows = 64, kFewMost = 8;
struct FewTokens {
  const void* w[kFewWindows];    // the vocabulary's shards
  void* dw[kFewWindows];         // null: not wanted
  const void* x[kFewMost];       // a row for each token (beyond `tokens` any of them)
  float* z;                      // [tokens][ldz]: logits, then D
  float* sums;                   // dx's partials, [range][tokens][ld_sum]; null: not wanted
  int64_t ldz, ldw, lddw, ld_sum;
  int32_t tokens, M, vocab;
  int32_t per, per_cols;         // entries of a shard, and columns of a row of logits for it
  int32_t shards;                // with dw: all of them, those without an entry too
  int32_t lanes;                 // [V, M]: lanes of a row, a power of two
  int32_t each;                  // gradients: rows of w of a workgroup
  int32_t blocks;                // workgroups that share a shard's entries
};
static_assert(sizeof(FewTokens) <= 4096, "kernel arguments");

template <typename T> constexpr int few_vec() { return 16 / static_cast<int>(sizeof(T)); }
template <typename T> using few_raw = T __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));

// 16 bytes of elements from `at` on, of which n exist (WHOLE: all): zeros beyond.  Kept as they are in memory until they are multiplied, so that many can be on their way.
template <typename T, bool WHOLE>
__device__ __forceinline__ few_raw<T> few_load(GSPMD_GLOBAL const T* at, int n) {
  constexpr int V = few_vec<T>();
  if (WHOLE || n >= V) return *(GSPMD_GLOBAL const few_raw<T>*)at;
  few_raw<T> v = 0;
#pragma unroll
  for (int e = 0; e < V - 1; ++e)
    if (e < n) v[e] = at[e];
  return v;
}
template <typename T>
__device__ __forceinline__ float few_float(few_raw<T> v, int e) {
  if constexpr (sizeof(T) == 2) return bf16_to_float(v[e]);
  else return v[e];
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void few_store(GSPMD_GLOBAL T* at, const float (&v)[few_vec<T>()], int n) {
  constexpr int V = few_vec<T>();
  few_raw<T> raw;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if constexpr (sizeof(T) == 2) raw[e] = __builtin_bit_cast(bf16_bits, static_cast<__bf16>(v[e]));
    else raw[e] = v[e];
  }
  if (WHOLE || n >= V) {
    *(GSPMD_GLOBAL few_raw<T>*)at = raw;
  } else {
#pragma unroll
    for (int e = 0; e < V - 1; ++e)
      if (e < n) at[e] = raw[e];
  }
}

// Sums over groups of `lanes` (a power of two) neighbouring lanes of N values each (a power of two), lane being this one's place in its group: at every step a lane keeps half of its
// values and gives the other half away, so N values take about N exchanges, not N for every step.  In the end a lane has values number `at` and following, for each of which it calls
// store(number, sum); where there are fewer values than lanes several lanes have the same one.
template <int N, int STEP = 0, int ALL, typename Store>
__device__ __forceinline__ void few_reduce(float (&v)[ALL], int lanes, int lane, Store store, int at = 0) {
  constexpr int d = 1 << STEP;
  if constexpr (STEP < 6) {
    if (d < lanes) {
      const bool upper = (lane & d) != 0;
      if constexpr (N >= 2) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          const float give = upper ? v[i] : v[i + N / 2], keep = upper ? v[i + N / 2] : v[i];
          v[i] = keep + __shfl_xor(give, d);
        }
        few_reduce<N / 2, STEP + 1>(v, lanes, lane, store, at + (upper ? N / 2 : 0));
      } else {
        v[0] += __shfl_xor(v[0], d);
        few_reduce<1, STEP + 1>(v, lanes, lane, store, at);
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) store(at + i, v[i]);
}

// ---- w [V, M]: `lanes` lanes go along a row, ROWS rows of one shard at a time; their sums over M meet in the end.
template <typename T, int NT, int ROWS>
__global__ __launch_bounds__(256) void few_logits_kernel(const FewTokens args) {
  constexpr int V = few_vec<T>();
  const GSPMD_KERNARG FewTokens& a = *first_kernel_argument<FewTokens>();
  const int lane = threadIdx.x & 63, lanes = a.lanes, sub = lane & (lanes - 1), groups = 64 / lanes;
  const int j = blockIdx.x / a.blocks, valid = min(a.per, a.vocab - j * a.per);
  const int first = (((blockIdx.x - j * a.blocks) * 4 + (threadIdx.x >> 6)) * groups + lane / lanes) * ROWS;
  GSPMD_GLOBAL const T* row[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) row[r] = (GSPMD_GLOBAL const T*)a.w[j] + static_cast<int64_t>(min(first + r, valid - 1)) * a.ldw;
  float sum[ROWS * NT];
#pragma unroll
  for (int i = 0; i < ROWS * NT; ++i) sum[i] = 0.f;
  // Whole vectors only, where a row has one: the last lane's is moved back to end with the row, and x and w there are 0 for what its neighbour has (both: either may be infinite, which 0 times it is not).
  struct Held { few_raw<T> w[ROWS]; };
  const bool narrow = a.M < V;
  auto load = [&](int m) {
    Held held;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) held.w[r] = narrow ? few_load<T, false>(row[r], a.M) : few_load<T, true>(row[r] + min(m, a.M - V), V);
    return held;
  };
  auto take = [&](Held held, int m) {
    few_raw<T> xv[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      GSPMD_GLOBAL const T* const x = (GSPMD_GLOBAL const T*)a.x[t];
      xv[t] = narrow ? few_load<T, false>(x, a.M) : few_load<T, true>(x + min(m, a.M - V), V);
    }
    if (!narrow && m + V > a.M)
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (a.M - V + e < m) {
#pragma unroll
          for (int t = 0; t < NT; ++t) xv[t][e] = 0;
#pragma unroll
          for (int r = 0; r < ROWS; ++r) held.w[r][e] = 0;
        }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int e = 0; e < V; ++e) sum[r * NT + t] = fmaf(few_float<T>(held.w[r], e), few_float<T>(xv[t], e), sum[r * NT + t]);
  };
  int m = sub * V;
  const int step = lanes * V;
  if (m < a.M) {                                  // the next vectors are on their way while these are taken
    Held held = load(m);
    for (;;) {
      const bool more = m + step < a.M;
      Held after = held;
      if (more) after = load(m + step);
      take(held, m);
      if (!more) break;
      held = after;
      m += step;
    }
  }
  few_reduce<ROWS * NT>(sum, lanes, sub, [&](int n, float s) {
    const int r = n / NT, t = n % NT;
    if (first + r < valid && t < a.tokens) a.z[t * a.ldz + j * a.per_cols + first + r] = s;
  });
}

// dw and dx's partials: a workgroup takes `each` entries of a shard and lanes * V columns; a thread has x and its part of dx in registers, the entries' D come through LDS.
template <typename T, int NT>
__global__ __launch_bounds__(256) void few_gradients_kernel(const FewTokens args) {
  constexpr int V = few_vec<T>(), kChunk = 128, kAhead = 4, kPass = NT < 2 ? NT : 2;
  const GSPMD_KERNARG FewTokens& a = *first_kernel_argument<FewTokens>();
  extern __shared__ __attribute__((aligned(16))) float lds[];     // [kChunk][NT] of D; in the end [4][kPass][lanes * V]
  const int t0 = threadIdx.x, lane = t0 & 63, wave = t0 >> 6, lanes = a.lanes, sub = lane & (lanes - 1), groups = 64 / lanes;
  // the last vector of a row is moved back to end with it (its neighbour's columns are then made, alike, by both)
  const int own = (blockIdx.x * lanes + sub) * V, m = a.M >= V ? min(own, a.M - V) : own, side = wave * groups + lane / lanes, sides = 4 * groups, room = own < a.M ? a.M - m : 0;
  const int j = blockIdx.y / a.blocks, begin = (blockIdx.y - j * a.blocks) * a.each, end = min(begin + a.each, a.per), valid = min(a.per, a.vocab - j * a.per);
  GSPMD_GLOBAL const T* const w = (GSPMD_GLOBAL const T*)a.w[j] + m;
  GSPMD_GLOBAL T* const dw = (GSPMD_GLOBAL T*)a.dw[j] + m;
  const bool has_dw = a.dw[j] != nullptr, has_dx = a.sums != nullptr, whole = a.M >= V;
  few_raw<T> xv[NT];
  float sum[NT][V];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    xv[t] = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) sum[t][e] = 0.f;
    if (t < a.tokens && room > 0) xv[t] = few_load<T, false>((GSPMD_GLOBAL const T*)a.x[t] + m, room);
  }
  auto take = [&](auto whole_tag, auto full_tag, int chunk, int stop, int r0) {   // the chunk's rows r0, r0 + sides, .. before `stop` (full: all of them are, and are entries)
    constexpr bool kWhole = decltype(whole_tag)::value, kFull = decltype(full_tag)::value;
    few_raw<T> wv[kAhead];
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const int v = chunk + r0 + n * sides;
      wv[n] = 0;
      if (has_dx && (kFull || (v < stop && v < valid))) wv[n] = few_load<T, kWhole>(w + static_cast<int64_t>(v) * a.ldw, room);
    }
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const int v = chunk + r0 + n * sides;
      if (!kFull && v >= stop) break;
      float out[V];
#pragma unroll
      for (int e = 0; e < V; ++e) out[e] = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float d = lds[(r0 + n * sides) * NT + t];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sum[t][e] = fmaf(d, few_float<T>(wv[n], e), sum[t][e]);
          out[e] = fmaf(d, few_float<T>(xv[t], e), out[e]);
        }
      }
      if constexpr (!kFull)
        if (v >= valid)                           // padding: zeros, whatever x is
#pragma unroll
          for (int e = 0; e < V; ++e) out[e] = 0.f;
      if (has_dw) few_store<T, kWhole>(dw + static_cast<int64_t>(v) * a.lddw, out, room);
    }
  };
  for (int chunk = begin; chunk < end; chunk += kChunk) {
    __syncthreads();
    const int stop = min(chunk + kChunk, end), full = min(stop, valid) - chunk;
    for (int i = t0; i < (stop - chunk) * NT; i += 256) {
      const int t = i % NT, v = chunk + i / NT;
      lds[i] = t < a.tokens && v < valid ? a.z[t * a.ldz + j * a.per_cols + v] : 0.f;
    }
    __syncthreads();
    if (room <= 0) continue;
    int r0 = side;
    if (whole)
      for (; r0 + (kAhead - 1) * sides < full; r0 += sides * kAhead) take(std::true_type{}, std::true_type{}, chunk, stop, r0);
    for (; chunk + r0 < stop; r0 += sides * kAhead) take(std::false_type{}, std::false_type{}, chunk, stop, r0);
  }
  if (!has_dx) return;
  // ---- over the groups of a wave, then over the waves
  for (int d = lanes; d < 64; d <<= 1)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < V; ++e) sum[t][e] += __shfl_xor(sum[t][e], d);
  const int cols = lanes * V;
  float* const out = a.sums + static_cast<int64_t>(blockIdx.y) * a.tokens * a.ld_sum;
#pragma unroll
  for (int p = 0; p < NT; p += kPass) {
    __syncthreads();
    if (lane < lanes && room > 0)
#pragma unroll
      for (int t = 0; t < kPass; ++t)
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (m + e >= own || !whole) lds[(wave * kPass + t) * cols + m - blockIdx.x * cols + e] = sum[p + t][e];
    __syncthreads();
    for (int i = t0; i < kPass * cols; i += 256) {
      const int t = i / cols, c = i - t * cols, at = blockIdx.x * cols + c;
      if (p + t < a.tokens && at < a.M) out[(p + t) * a.ld_sum + at] = ((lds[t * cols + c] + lds[(kPass + t) * cols + c]) + lds[(2 * kPass + t) * cols + c]) + lds[(3 * kPass + t) * cols + c];
    }
  }
}
// LDS bytes
template <typename T, int NT> constexpr int few_pass() { return NT < 2 ? NT : 2; }
template <typename T, int NT> int few_gradients_lds(int lanes) {
  const int chunk = 128 * NT * 4, end = 4 * few_pass<T, NT>() * lanes * few_vec<T>() * 4;
  return chunk > end ? chunk : end;
}

// ---- w [M, V]: a thread has V entries of every row, SIDE lanes beside each other, the others on other rows.  Sums over the rows meet in the end.
constexpr int kFewAcross = 512;
template <typename T, int NT, int SIDE>
__global__ __launch_bounds__(kFewAcross) void few_logits_across_kernel(const FewTokens args) {
  constexpr int THREADS = kFewAcross, V = few_vec<T>(), kRows = THREADS / SIDE, kAhead = 8, kChunk = 512;
  const GSPMD_KERNARG FewTokens& a = *first_kernel_argument<FewTokens>();
  extern __shared__ __attribute__((aligned(16))) float lds[];     // [kChunk][NT] of x; in the end [waves][NT][SIDE * V]
  const int t0 = threadIdx.x, lane = t0 & 63, wave = t0 >> 6, sub = t0 & (SIDE - 1), side = t0 / SIDE;
  const int j = blockIdx.x / a.blocks, from = (blockIdx.x - j * a.blocks) * SIDE * V, valid = min(a.per, a.vocab - j * a.per), room = valid - from - sub * V;
  GSPMD_GLOBAL const T* const w = (GSPMD_GLOBAL const T*)a.w[j] + from + sub * V;
  const bool whole = from + SIDE * V <= valid;
  float sum[NT][V];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < V; ++e) sum[t][e] = 0.f;
  auto take = [&](auto whole_tag, auto full_tag, int chunk, int r0, int rows) {
    constexpr bool kWhole = decltype(whole_tag)::value, kFull = decltype(full_tag)::value;
    few_raw<T> wv[kAhead];
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      wv[n] = 0;
      if (kFull || r0 + n * kRows < rows) wv[n] = few_load<T, kWhole>(w + static_cast<int64_t>(chunk + r0 + n * kRows) * a.ldw, room);
    }
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      if (!kFull && r0 + n * kRows >= rows) break;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float xt = lds[(r0 + n * kRows) * NT + t];
#pragma unroll
        for (int e = 0; e < V; ++e) sum[t][e] = fmaf(xt, few_float<T>(wv[n], e), sum[t][e]);
      }
    }
  };
  for (int chunk = 0; chunk < a.M; chunk += kChunk) {
    __syncthreads();
    const int rows = min(kChunk, a.M - chunk);
    for (int i = t0; i < rows * NT; i += THREADS) lds[i] = load_as_float(static_cast<const T*>(a.x[i % NT]) + chunk + i / NT);
    __syncthreads();
    if (room <= 0) continue;
    int r0 = side;
    if (whole)
      for (; r0 + (kAhead - 1) * kRows < rows; r0 += kRows * kAhead) take(std::true_type{}, std::true_type{}, chunk, r0, rows);
    for (; r0 < rows; r0 += kRows * kAhead) take(std::false_type{}, std::false_type{}, chunk, r0, rows);
  }
#pragma unroll
  for (int d = SIDE; d < 64; d <<= 1)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < V; ++e) sum[t][e] += __shfl_xor(sum[t][e], d);
  __syncthreads();
  constexpr int kCols = SIDE * V, kWaves = THREADS / 64;
  if (lane < SIDE)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < V; ++e) lds[(wave * NT + t) * kCols + sub * V + e] = sum[t][e];
  __syncthreads();
  for (int i = t0; i < a.tokens * kCols; i += THREADS) {
    const int t = i / kCols, c = i % kCols;
    float s = 0.f;
#pragma unroll
    for (int n = 0; n < kWaves; ++n) s += lds[(n * NT + t) * kCols + c];
    if (from + c < valid) a.z[t * a.ldz + j * a.per_cols + from + c] = s;
  }
}

// dw and dx's partials: a workgroup takes 64 V entries of a shard and `each` rows; a thread has D of its entries in registers, a row's sums over the entries meet over the wave, ROWS rows
// at a time.
template <typename T, int NT>
__global__ __launch_bounds__(256) void few_gradients_across_kernel(const FewTokens args) {
  constexpr int V = few_vec<T>(), ROWS = 8, kChunk = 256;
  const GSPMD_KERNARG FewTokens& a = *first_kernel_argument<FewTokens>();
  extern __shared__ __attribute__((aligned(16))) float lds[];     // [kChunk][NT] of x
  const int t0 = threadIdx.x, lane = t0 & 63, wave = t0 >> 6;
  const int j = blockIdx.x / a.blocks, from = (blockIdx.x - j * a.blocks) * 64 * V, at = from + lane * V, valid = min(a.per, a.vocab - j * a.per);
  const int room = valid - at, store_room = a.per - at;       // entries that exist, and that the shard has a place for
  const int begin = blockIdx.y * a.each, end = min(begin + a.each, a.M);
  const bool has_dw = a.dw[j] != nullptr, has_dx = a.sums != nullptr, whole = from + 64 * V <= valid;
  float d[NT][V];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int e = 0; e < V; ++e) d[t][e] = 0.f;
    if (t >= a.tokens) continue;
    GSPMD_GLOBAL const float* const from_d = (GSPMD_GLOBAL const float*)a.z + t * a.ldz + j * a.per_cols + at;
    if (whole) {
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const float4_t four = *(GSPMD_GLOBAL const float4_t*)(from_d + e);
#pragma unroll
        for (int n = 0; n < 4; ++n) d[t][e + n] = four[n];
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e < room) d[t][e] = from_d[e];
    }
  }
  GSPMD_GLOBAL const T* const w = (GSPMD_GLOBAL const T*)a.w[j] + at;
  GSPMD_GLOBAL T* const dw = (GSPMD_GLOBAL T*)a.dw[j] + at;
  struct Held { few_raw<T> w[ROWS]; };
  auto load = [&](auto whole_tag, auto full_tag, int chunk, int r0, int rows) {
    constexpr bool kWhole = decltype(whole_tag)::value, kFull = decltype(full_tag)::value;
    Held held;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      held.w[r] = 0;
      if (has_dx && (kFull || r0 + r < rows) && (kWhole || room > 0)) held.w[r] = few_load<T, kWhole>(w + static_cast<int64_t>(chunk + r0 + r) * a.ldw, room);
    }
    return held;
  };
  auto take = [&](auto whole_tag, auto full_tag, const Held& held, int chunk, int r0, int rows) {
    constexpr bool kWhole = decltype(whole_tag)::value, kFull = decltype(full_tag)::value;
    float sum[ROWS * NT];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float out[V];
#pragma unroll
      for (int e = 0; e < V; ++e) out[e] = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float xt = lds[(r0 + r) * NT + t];
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          out[e] = fmaf(xt, d[t][e], out[e]);
          s = fmaf(d[t][e], few_float<T>(held.w[r], e), s);
        }
        sum[r * NT + t] = s;
      }
      if constexpr (!kWhole)
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (e >= room) out[e] = 0.f;            // padding: zeros, whatever x is
      if (has_dw && (kFull || r0 + r < rows) && (kWhole || store_room > 0)) few_store<T, kWhole>(dw + static_cast<int64_t>(chunk + r0 + r) * a.lddw, out, store_room);
    }
    if (!has_dx) return;
    few_reduce<ROWS * NT>(sum, 64, lane, [&](int n, float total) {
      const int r = n / NT, t = n % NT;
      if ((kFull || r0 + r < rows) && t < a.tokens) a.sums[(static_cast<int64_t>(blockIdx.x) * a.tokens + t) * a.ld_sum + chunk + r0 + r] = total;
    });
  };
  for (int chunk = begin; chunk < end; chunk += kChunk) {
    __syncthreads();
    const int rows = min(kChunk, end - chunk);
    for (int i = t0; i < rows * NT; i += 256) lds[i] = load_as_float(static_cast<const T*>(a.x[i % NT]) + chunk + i / NT);
    __syncthreads();
    int r0 = wave * ROWS;
    if (whole && r0 + ROWS <= rows) {             // the next rows are on their way while these are taken
      const std::true_type yes{};
      Held held = load(yes, yes, chunk, r0, rows);
      for (;;) {
        const int next = r0 + 4 * ROWS;
        const bool more = next + ROWS <= rows;
        Held after = held;
        if (more) after = load(yes, yes, chunk, next, rows);
        take(yes, yes, held, chunk, r0, rows);
        r0 = next;
        if (!more) break;
        held = after;
      }
    }
    const std::false_type no{};
    for (; r0 < rows; r0 += 4 * ROWS) take(no, no, load(no, no, chunk, r0, rows), chunk, r0, rows);
  }
}

// Token shards of dx = the sum of `count` partials of few rows: 16 threads side by side (4 columns each), 16 sharing the partials of each, whose sums meet in LDS in ascending order.
template <typename T>
__global__ __launch_bounds__(256) void add_up_few_kernel(const AddUp args) {
  const GSPMD_KERNARG AddUp& a = *first_kernel_argument<AddUp>();
  __shared__ f32x4 parts[16][16];
  const int x = threadIdx.x & 15, part = threadIdx.x >> 4, col = (blockIdx.x * 16 + x) * 4, row = blockIdx.y;
  const int g = a.first + row, i = g / a.per_row, at = g - i * a.per_row, each = (a.count + 15) / 16, begin = part * each;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (col < a.cols && g < a.tokens) sum = sum_partials((GSPMD_GLOBAL const float*)a.partials + static_cast<int64_t>(row) * a.ld_in + col, a.stride, begin, min(begin + each, a.count));
  parts[part][x] = sum;
  __syncthreads();
  if (part != 0 || col >= a.cols) return;
  for (int p = 1; p < 16; ++p) sum += parts[p][x];
  store_sum<T>((GSPMD_GLOBAL T*)a.to[i - a.first_shard] + static_cast<int64_t>(at) * a.ld_out + col, sum, a.cols - col);
}

}  // namespace gspmd
