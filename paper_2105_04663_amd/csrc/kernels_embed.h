// Rows of a vocabulary matrix by tokens' entries, and their gradient (gspmd_embed, gspmd_embed_grad).
//
// Both are bound by memory: the rows that are read and the rows that are written, once each.  A vocabulary matrix [V, M] has an entry's row in one piece, read and written 16 bytes a lane at
// element alignment, neighbouring lanes side by side; in one [M, V] an entry is a column, and tiles turn in LDS.
// The gradient has one writer for each of its elements: tokens are ordered by entry (kernels_order.h), a row of dw is the sum over its run of them, in float32, in ascending order of the tokens -- but
// for whole chunks of that order that lie inside one run, which are added up by themselves first, so that an entry that half of a text consists of is no chain of
// thousands of loads.  So equal inputs give equal bits, and a row without tokens is zeros.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels_basic.h"
#include "mfma_common.h"

namespace gspmd {

constexpr int kTokenShards = 64, kVocabShards = 64;

struct TokenShard {
  const int32_t* ids;
  void* rows;                  // y or dy; null: none to be written
};
// The first thing in a kernel's arguments (its shards are read there with run-time indexes).
struct EmbedArgs {
  TokenShard tokens[kTokenShards];
  void* vocab[kVocabShards];   // null: none to be written
  int32_t T, ts, token_shards; // tokens, of a shard, shards
  int32_t V, vs, vocab_shards;
  int32_t M, ld_rows;
  int64_t ld_vocab;
  float scale;
  int32_t accumulate;
  // the gradient's: tokens in the order of their entries, where an entry's begin [V + 1], and sums of whole chunks of the order, [chunk][M]
  const int32_t *order, *begins;
  float* chunks;
};
constexpr int kChunk = 32;     // tokens

typedef __attribute__((address_space(4))) const EmbedArgs embed_args;
__device__ __forceinline__ embed_args* embed_arguments() { return first_kernel_argument<EmbedArgs>(); }
// (one shard: no division)
__device__ __forceinline__ int embed_shard(int i, int per, int shards) { return shards == 1 ? 0 : static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(per)); }

template <typename T> struct Sixteen;          // 16 bytes as float32, and back with one rounding
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
};
template <typename T> struct AnyAligned;
template <> struct AnyAligned<bf16_bits> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct AnyAligned<float> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4))); };
template <typename T> __device__ __forceinline__ u32x4_t load16(const T* p) { return *(GSPMD_GLOBAL const typename AnyAligned<T>::type*)p; }
template <typename T> __device__ __forceinline__ void store16(T* p, u32x4_t v) { *(GSPMD_GLOBAL typename AnyAligned<T>::type*)p = v; }
// the first `count` elements of 16 bytes
template <typename T> __device__ __forceinline__ u32x4_t load_some(const T* p, int count) {
  u32x4_t v = {0u, 0u, 0u, 0u};
  constexpr int n = Sixteen<T>::n;
#pragma unroll
  for (int i = 0; i < n; ++i)
    if (i < count) {
      const uint32_t bits = sizeof(T) == 2 ? static_cast<uint32_t>(((GSPMD_GLOBAL const uint16_t*)p)[i]) : ((GSPMD_GLOBAL const uint32_t*)p)[i];
      if constexpr (sizeof(T) == 2) v[i >> 1] |= bits << ((i & 1) * 16);
      else v[i] = bits;
    }
  return v;
}
template <typename T> __device__ __forceinline__ void store_some(T* p, u32x4_t v, int count) {
  constexpr int n = Sixteen<T>::n;
#pragma unroll
  for (int i = 0; i < n; ++i)
    if (i < count) {
      if constexpr (sizeof(T) == 2) ((GSPMD_GLOBAL uint16_t*)p)[i] = static_cast<uint16_t>(v[i >> 1] >> ((i & 1) * 16));
      else ((GSPMD_GLOBAL uint32_t*)p)[i] = v[i];
    }
}
template <typename T> __device__ __forceinline__ u32x4_t load_up_to(const T* p, int count) { return count >= Sixteen<T>::n ? load16(p) : load_some(p, count); }
template <typename T> __device__ __forceinline__ void store_up_to(T* p, u32x4_t v, int count) {
  if (count >= Sixteen<T>::n) store16(p, v);
  else store_some(p, v, count);
}

// How many lanes a row of `elements` takes: a power of two, up to a wave.
__host__ __device__ __forceinline__ int row_lanes_log(int elements, int per_lane) {
  int log = 0;
  while (log < 6 && (per_lane << log) < elements) ++log;
  return log;
}

// y [V, M]: a wave has a piece of a row (or a few short rows), kEmbedUnroll x 16 bytes a lane.
constexpr int kEmbedUnroll = 8;
template <typename T, bool SCALED>
__global__ __launch_bounds__(256) void embed_rows_kernel(const EmbedArgs a, int log_lanes, int pieces) {
  constexpr int n = Sixteen<T>::n;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lanes = 1 << log_lanes;
  const int group = blockIdx.x / pieces, piece = blockIdx.x - group * pieces;              // (neighbouring pieces of rows together)
  const int row = ((group * 4 + wave) << (6 - log_lanes)) + (lane >> log_lanes);            // static rows of all shards, one after the other
  if (row >= a.ts * a.token_shards) return;
  const int shard = embed_shard(row, a.ts, a.token_shards), within = row - shard * a.ts;
  const TokenShard to = {embed_arguments()->tokens[shard].ids, embed_arguments()->tokens[shard].rows};
  if (to.rows == nullptr) return;
  const int id = row < a.T ? ((GSPMD_GLOBAL const int32_t*)to.ids)[within] : -1;
  const bool there = static_cast<uint32_t>(id) < static_cast<uint32_t>(a.V);
  T* const y = static_cast<T*>(to.rows) + static_cast<int64_t>(within) * a.ld_rows;
  const int of = there ? embed_shard(id, a.vs, a.vocab_shards) : 0;
  const T* const w = static_cast<const T*>(embed_arguments()->vocab[of]) + (there ? static_cast<int64_t>(id - of * a.vs) * a.ld_vocab : 0);
  const int col0 = ((piece * kEmbedUnroll) << log_lanes) * n + (lane & (lanes - 1)) * n, step = n << log_lanes;
  u32x4_t v[kEmbedUnroll];
#pragma unroll
  for (int u = 0; u < kEmbedUnroll; ++u) {
    v[u] = u32x4_t{0u, 0u, 0u, 0u};
    const int col = col0 + u * step;
    if (there && col < a.M) v[u] = load_up_to(w + col, a.M - col);
  }
#pragma unroll
  for (int u = 0; u < kEmbedUnroll; ++u) {
    const int col = col0 + u * step;
    if (SCALED && there) {
      float f[n];
      Sixteen<T>::open(v[u], f);
#pragma unroll
      for (int i = 0; i < n; ++i) f[i] *= a.scale;
      v[u] = Sixteen<T>::close(f);
    }
    if (col < a.M) store_up_to(y + col, v[u], a.M - col);
  }
}

// y from [M, V]: 64 tokens x 32 columns of y a workgroup.  A lane has a token and reads its column of eight rows of w, element by element: neighbouring tokens' entries lie anywhere in a row, so what
// has to be near is the row.  Workgroups of one XCD take the same 32 rows of w for all tokens, one after the other, out of its L2.
constexpr int kColumnTokens = 64, kColumnCols = 32;
template <typename T>
__global__ __launch_bounds__(256) void embed_columns_kernel(const EmbedArgs a, int token_blocks, int col_blocks) {
  __shared__ float tile[kColumnTokens][kColumnCols + 1];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3, block = xcd + 8 * (turn / token_blocks);
  if (block >= col_blocks) return;
  const int row0 = (turn % token_blocks) * kColumnTokens, col0 = block * kColumnCols, rows = a.ts * a.token_shards;
  {
    const int row = row0 + lane;
    int id = -1;
    if (row < a.T) {
      const int shard = embed_shard(row, a.ts, a.token_shards);
      id = ((GSPMD_GLOBAL const int32_t*)embed_arguments()->tokens[shard].ids)[row - shard * a.ts];
    }
    const bool there = static_cast<uint32_t>(id) < static_cast<uint32_t>(a.V);
    const int of = there ? embed_shard(id, a.vs, a.vocab_shards) : 0;
    GSPMD_GLOBAL const T* const w = (GSPMD_GLOBAL const T*)embed_arguments()->vocab[of] + (there ? id - of * a.vs : 0);
    float v[kColumnCols / 4];
#pragma unroll
    for (int i = 0; i < kColumnCols / 4; ++i) {
      const int col = col0 + wave * (kColumnCols / 4) + i;
      v[i] = 0.f;
      if (there && col < a.M) {
        const T e = w[col * a.ld_vocab];
        v[i] = sizeof(T) == 2 ? __uint_as_float(static_cast<uint32_t>(e) << 16) : static_cast<float>(e);
      }
    }
#pragma unroll
    for (int i = 0; i < kColumnCols / 4; ++i) tile[lane][wave * (kColumnCols / 4) + i] = v[i];
  }
  __syncthreads();
  constexpr int n = Sixteen<T>::n, per_row = kColumnCols / n;
  for (int i = t; i < kColumnTokens * per_row; i += 256) {
    const int r = i / per_row, c = (i - r * per_row) * n, row = row0 + r, col = col0 + c;
    if (row >= rows || col >= a.M) continue;
    const int shard = embed_shard(row, a.ts, a.token_shards);
    T* const y = static_cast<T*>(embed_arguments()->tokens[shard].rows);
    if (y == nullptr) continue;
    float f[n];
#pragma unroll
    for (int e = 0; e < n; ++e) f[e] = a.scale == 1.f ? tile[r][c + e] : tile[r][c + e] * a.scale;
    store_up_to(y + static_cast<int64_t>(row - shard * a.ts) * a.ld_rows + col, Sixteen<T>::close(f), a.M - col);
  }
}

// ---- the gradient
// dy's row of a token
template <typename T>
__device__ __forceinline__ const T* token_row(const EmbedArgs& a, int token) {
  const int shard = embed_shard(token, a.ts, a.token_shards);
  return static_cast<const T*>(embed_arguments()->tokens[shard].rows) + static_cast<int64_t>(token - shard * a.ts) * a.ld_rows;
}

// sum += the `count` tokens' 16 bytes at `col` from place `at` of the order on, ascending
template <typename T>
__device__ __forceinline__ void add_tokens(const EmbedArgs& a, int at, int count, int col, float (&sum)[Sixteen<T>::n]) {
  constexpr int n = Sixteen<T>::n, kAhead = 8;
  GSPMD_GLOBAL const int32_t* const order = (GSPMD_GLOBAL const int32_t*)a.order + at;
  int i = 0;
  for (; i + kAhead <= count; i += kAhead) {
    u32x4_t v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = load_up_to(token_row<T>(a, order[i + u]) + col, a.M - col);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float f[n];
      Sixteen<T>::open(v[u], f);
#pragma unroll
      for (int e = 0; e < n; ++e) sum[e] += f[e];
    }
  }
  for (; i < count; ++i) {
    float f[n];
    Sixteen<T>::open(load_up_to(token_row<T>(a, order[i]) + col, a.M - col), f);
#pragma unroll
    for (int e = 0; e < n; ++e) sum[e] += f[e];
  }
}

// Sums of the chunks that lie inside one entry's run: blockIdx.x the chunk, blockIdx.y 64 x 16 bytes of the row; a wave a quarter of the tokens.
template <typename T>
__global__ __launch_bounds__(256) void embed_chunks_kernel(const EmbedArgs a) {
  constexpr int n = Sixteen<T>::n;
  const int at = blockIdx.x * kChunk, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  GSPMD_GLOBAL const int32_t* const begins = (GSPMD_GLOBAL const int32_t*)a.begins;
  if (at + kChunk > begins[a.V]) return;        // some of it no token's place
  const int first = ((GSPMD_GLOBAL const int32_t*)a.order)[at], shard = embed_shard(first, a.ts, a.token_shards);
  const int key = ((GSPMD_GLOBAL const int32_t*)embed_arguments()->tokens[shard].ids)[first - shard * a.ts];
  if (static_cast<uint32_t>(key) >= static_cast<uint32_t>(a.V) || begins[key + 1] < at + kChunk) return;
  __shared__ float sums[4][64 * n];
  const int col = (blockIdx.y * 64 + lane) * n;
  float sum[n];
#pragma unroll
  for (int e = 0; e < n; ++e) sum[e] = 0.f;
  if (col < a.M) add_tokens<T>(a, at + wave * (kChunk / 4), kChunk / 4, col, sum);
#pragma unroll
  for (int e = 0; e < n; ++e) sums[wave][lane * n + e] = sum[e];
  __syncthreads();
  float* const out = a.chunks + static_cast<int64_t>(blockIdx.x) * a.M + blockIdx.y * 64 * n;
  for (int i = threadIdx.x; i < 64 * n && blockIdx.y * 64 * n + i < a.M; i += 256) out[i] = ((sums[0][i] + sums[1][i]) + sums[2][i]) + sums[3][i];
}

// The sum over places [begin, end) of the order, one entry's run, for the columns from `col` on.
template <typename T>
__device__ __forceinline__ void add_run(const EmbedArgs& a, int begin, int end, int col, float (&sum)[Sixteen<T>::n]) {
  constexpr int n = Sixteen<T>::n;
  const int first = (begin + kChunk - 1) / kChunk, last = end / kChunk;        // whole chunks
  if (first >= last) {
    add_tokens<T>(a, begin, end - begin, col, sum);
    return;
  }
  add_tokens<T>(a, begin, first * kChunk - begin, col, sum);
  GSPMD_GLOBAL const float* at = (GSPMD_GLOBAL const float*)a.chunks + static_cast<int64_t>(first) * a.M + col;
  constexpr int kAhead = 4;
  int c = first;
  for (; c < last; c += kAhead) {
    float v[kAhead][n];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int e = 0; e < n; ++e) v[u][e] = c + u < last && col + e < a.M ? at[u * static_cast<int64_t>(a.M) + e] : 0.f;
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int e = 0; e < n; ++e) sum[e] += v[u][e];
    at += kAhead * static_cast<int64_t>(a.M);
  }
  add_tokens<T>(a, last * kChunk, end - last * kChunk, col, sum);
}

// dw [V, M]: a workgroup has kRowsSide entries and 4 waves' columns of them (blockIdx.y), or fewer columns and the rows shared out.  Most entries have no token, and most that have any have one: where the
// runs begin is read at once, and the first tokens of four rows are on their way together.
constexpr int kRowsSide = 16, kRowsAhead = 4;
template <typename T>
__global__ __launch_bounds__(256) void embed_grad_rows_kernel(const EmbedArgs a, int log_lanes, int log_across) {
  constexpr int n = Sixteen<T>::n;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = blockIdx.x * kRowsSide, rows = a.vs * a.vocab_shards;
  const int begins = a.T > 0 ? ((GSPMD_GLOBAL const int32_t*)a.begins)[min(row0 + min(lane, kRowsSide), a.V)] : 0;      // (of a row behind the last entry: the end of all, as its successor's)
  const int across = 1 << log_across, side = 64 >> log_lanes;        // waves along a row; rows of a wave at a time
  const int col = ((blockIdx.y * across + (wave & (across - 1))) << log_lanes) * n + (lane & ((1 << log_lanes) - 1)) * n;
  const int turn = (4 >> log_across) * side;                          // from a lane's row to its next
  const bool in = col < a.M;
  for (int r0 = (wave >> log_across) * side + (lane >> log_lanes); r0 - (lane >> log_lanes) < kRowsSide; r0 += kRowsAhead * turn) {
    int begin[kRowsAhead], end[kRowsAhead], token[kRowsAhead];
    u32x4_t v[kRowsAhead];
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const int r = r0 + u * turn;
      begin[u] = __shfl(begins, min(r, kRowsSide));
      end[u] = __shfl(begins, min(r + 1, kRowsSide));
      token[u] = 0;
      v[u] = u32x4_t{0u, 0u, 0u, 0u};
    }
    bool any = false;
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) any = any || begin[u] < end[u];
    if (any && in) {
#pragma unroll
      for (int u = 0; u < kRowsAhead; ++u) token[u] = ((GSPMD_GLOBAL const int32_t*)a.order)[begin[u] < end[u] ? begin[u] : 0];
      const bool whole = col + n <= a.M;
#pragma unroll
      for (int u = 0; u < kRowsAhead; ++u)
        if (whole) v[u] = load16(token_row<T>(a, begin[u] < end[u] ? token[u] : 0) + col);
        else if (begin[u] < end[u]) v[u] = load_some(token_row<T>(a, token[u]) + col, a.M - col);
    }
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const int r = r0 + u * turn, row = row0 + r;
      if (r >= kRowsSide || row >= rows || !in) continue;
      const int shard = embed_shard(row, a.vs, a.vocab_shards);
      T* dw = static_cast<T*>(embed_arguments()->vocab[shard]);
      if (dw == nullptr) continue;
      dw += static_cast<int64_t>(row - shard * a.vs) * a.ld_vocab + col;
      if (begin[u] == end[u]) {
        if (!a.accumulate || row >= a.V) store_up_to(dw, u32x4_t{0u, 0u, 0u, 0u}, a.M - col);
        continue;
      }
      float sum[n];
      Sixteen<T>::open(v[u], sum);
      if (begin[u] + 1 < end[u]) add_run<T>(a, begin[u] + 1, end[u], col, sum);
#pragma unroll
      for (int e = 0; e < n; ++e) sum[e] *= a.scale;
      if (a.accumulate) {
        float f[n];
        Sixteen<T>::open(load_up_to(dw, a.M - col), f);
#pragma unroll
        for (int e = 0; e < n; ++e) sum[e] += f[e];
      }
      store_up_to(dw, Sixteen<T>::close(sum), a.M - col);
    }
  }
}

// dw [M, V]: 64 entries x 16 lanes' 16 bytes of dw's rows a workgroup.  Sixteen lanes have an entry, four of them one after the other, whose first tokens are on their way together; what they add up turns in
// LDS, rounded but for what is still to be added to (TTile float).  Bound by what is on its way: 8 workgroups on a compute unit, each 5 KB of rows and 16 of dw.
constexpr int kTurnEntries = 64, kTurnLanes = 16;
template <typename T, typename TTile>
__global__ __launch_bounds__(256) void embed_grad_columns_kernel(const EmbedArgs a) {
  constexpr int n = Sixteen<T>::n, kRows = kTurnLanes * n, side = 64 / kTurnLanes, kEach = kTurnEntries / (4 * side), kPitch = kTurnEntries + (sizeof(TTile) == 2 ? 2 : 1);
  __shared__ __attribute__((aligned(4))) TTile tile[kRows][kPitch];
  __shared__ int begins[kTurnEntries + 1];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  // entries of one shard: blockIdx.x counts blocks of every shard
  const int per_shard = (a.vs + kTurnEntries - 1) / kTurnEntries, shard = blockIdx.x / per_shard, c0 = (blockIdx.x - shard * per_shard) * kTurnEntries;
  const int row0 = shard * a.vs + c0, m0 = blockIdx.y * kRows, entries = min(kTurnEntries, a.vs - c0);
  T* const dw = static_cast<T*>(embed_arguments()->vocab[shard]);
  if (dw == nullptr) return;
  if (t <= kTurnEntries) begins[t] = a.T > 0 ? ((GSPMD_GLOBAL const int32_t*)a.begins)[min(row0 + t, a.V)] : 0;
  __syncthreads();
  const int col = m0 + (lane & (kTurnLanes - 1)) * n, r0 = wave * side + lane / kTurnLanes;
  int begin[kEach], end[kEach], token[kEach];
  u32x4_t v[kEach];
  bool any = false;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int r = r0 + u * 4 * side;
    begin[u] = begins[r];
    end[u] = r < entries ? begins[r + 1] : begin[u];
    any = any || begin[u] < end[u];
    v[u] = u32x4_t{0u, 0u, 0u, 0u};
    token[u] = 0;
  }
  if (any && col < a.M) {
#pragma unroll
    for (int u = 0; u < kEach; ++u) token[u] = ((GSPMD_GLOBAL const int32_t*)a.order)[begin[u] < end[u] ? begin[u] : 0];
    const bool whole = col + n <= a.M;
#pragma unroll
    for (int u = 0; u < kEach; ++u)
      if (whole) v[u] = load16(token_row<T>(a, begin[u] < end[u] ? token[u] : 0) + col);
      else if (begin[u] < end[u]) v[u] = load_some(token_row<T>(a, token[u]) + col, a.M - col);
  }
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    float sum[n];
    Sixteen<T>::open(v[u], sum);
    if (begin[u] + 1 < end[u] && col < a.M) add_run<T>(a, begin[u] + 1, end[u], col, sum);
    const int r = r0 + u * 4 * side;
#pragma unroll
    for (int e = 0; e < n; ++e) store_from_float<TTile>(&tile[(lane & (kTurnLanes - 1)) * n + e][r], begin[u] < end[u] ? sum[e] * a.scale : 0.f);
  }
  __syncthreads();
  for (int i = t; i < kRows * (kTurnEntries / n); i += 256) {
    const int m = i / (kTurnEntries / n), c = (i - m * (kTurnEntries / n)) * n, count = entries - c;
    if (m0 + m >= a.M || count <= 0) continue;
    T* const at = dw + (m0 + m) * a.ld_vocab + c0 + c;
    if constexpr (sizeof(TTile) == 2) {
      u32x4_t o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = *reinterpret_cast<const uint32_t*>(&tile[m][c + 2 * e]);
      store_up_to(at, o, count);
    } else {
      float f[n];
#pragma unroll
      for (int e = 0; e < n; ++e) f[e] = tile[m][c + e];
      if (a.accumulate) {                       // entries without tokens keep what they have
        float before[n];
        Sixteen<T>::open(load_up_to(at, count), before);
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (e < count && row0 + c + e < a.V) f[e] = begins[c + e] == begins[c + e + 1] ? before[e] : before[e] + f[e];
      }
      store_up_to(at, Sixteen<T>::close(f), count);
    }
  }
}

}  // namespace gspmd
