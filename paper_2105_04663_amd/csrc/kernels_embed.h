// Rows of a vocabulary matrix by tokens' entries, and their gradient (gspmd_embed, gspmd_embed_grad).
//
// Both are bound by memory: the rows that are read and the rows that are written, once each.  A vocabulary matrix [V, M] has an entry's row in one piece, read and written 16 bytes a lane at
// element alignment, neighbouring lanes side by side; in one [M, V] an entry is a column, and tiles turn in LDS.
// The gradient has one writer for each of its elements.  Tokens are ordered by entry (kernels_order.h); an entry's are a run of that order, and its row of dw is the sum over the run, in float32.  The
// order is cut into chunks of a few tokens, which are added up side by side whatever the runs are, so that an entry that half of a text consists of is no chain of thousands of loads: a run inside a chunk
// is finished there, what a chunk has of runs that begin before it or end behind it are partial sums, added up by the chunk that a run begins in, in a second launch.  All sums have one
// fixed order, so equal inputs give equal bits.  Rows of dw [V, M] without tokens are zeroed in the launch that orders; a dw [M, V] is written whole from the sums.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels_basic.h"
#include "kernels_rows.h"
#include "mfma_common.h"
#include "tile_index.h"

namespace gspmd {

constexpr int kTokenShards = 64, kVocabShards = 64, kFewShards = 8;

struct TokenShard {
  const int32_t* ids;
  void* rows;                  // y or dy; null: none to be written
};
struct EmbedSizes {
  int32_t T, ts, token_shards; // tokens, of a shard, shards
  int32_t V, vs, vocab_shards;
  int32_t M, ld_rows;
  int64_t ld_vocab;
  float scale;
  int32_t accumulate;
  // the gradient's: the token and its entry at every place of the order, where an entry's begin [V + 1], chunks' sums [chunk][M] of a run that began before and of one that begins there and ends
  // behind it, and (dw [M, V]) runs' sums, at half the place where they begin, [T / 2][M]
  const int32_t *order, *entries, *begins;
  float *heads, *tails, *sums;
};
// The first of a kernel's arguments (its shards are read there with run-time indexes).  A table of few shards where that is enough: what a launch costs the host goes by the arguments that it copies (us a
// call, one token, 64 / 8: 6.7 / 6.3).
template <int SHARDS>
struct EmbedArgsOf : EmbedSizes {
  TokenShard tokens[SHARDS];
  void* vocab[SHARDS];         // null: none to be written
};
typedef EmbedArgsOf<kTokenShards> EmbedArgs;
static_assert(kTokenShards == kVocabShards, "one size of table");
// Tokens of a chunk: few where there are few chunks, as a chunk's tokens wait for each other; more where there are many, as their sums are read again (us, 8 / 16: 2048 tokens of 2048 29.3 / 30.9,
// 8192 of 1024 25.1 / 25.5, 32768 of 4096 172 / 159).
constexpr int kSmallChunk = 8, kLargeChunk = 16, kFewTokens = 8192;
// Up to so many tokens nothing is joined: a launch less, but a run of all of them is a chain of their loads (us, joined / alone, texts: 100 tokens of 832, 1152 entries 13.2 / 10.4, 512 13.1 / 16.1; beside
// the 131 MB of 32000 entries of 2048, where the host is ahead, 100 tokens 26.6 / 28.1).
constexpr int kAloneTokens = 128;

// (one shard: no division)
__device__ __forceinline__ int embed_shard(int i, int per, int shards) { return shards == 1 ? 0 : static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(per)); }

// y from [V, M]: a wave has a piece of a row (or a few short rows), kEmbedUnroll x 16 bytes a lane (16384 tokens of 8192 from 32000 entries: 74 us, 268 MB written at 3.6 TB/s).
constexpr int kEmbedUnroll = 4;
template <typename T, int LINES, bool SCALED, typename A>
__global__ __launch_bounds__(256) void embed_rows_kernel(const A a, int log_lanes, int pieces) {
  constexpr int n = Sixteen<T>::n;
  const int log = LINES == kWide ? 6 : log_lanes, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = blockIdx.x / pieces, piece = blockIdx.x - group * pieces;              // (neighbouring pieces of rows together)
  const int row = of_row<LINES>(((group * 4 + wave) << (6 - log)) + (lane >> log));        // static rows of all shards, one after the other
  if (row >= a.ts * a.token_shards) return;
  const int shard = of_row<LINES>(embed_shard(row, a.ts, a.token_shards)), within = row - shard * a.ts;
  const TokenShard to = {first_kernel_argument<A>()->tokens[shard].ids, first_kernel_argument<A>()->tokens[shard].rows};
  if (to.rows == nullptr) return;
  const int id = row < a.T ? of_row<LINES>(((GSPMD_GLOBAL const int32_t*)to.ids)[within]) : -1;
  const bool there = static_cast<uint32_t>(id) < static_cast<uint32_t>(a.V);
  T* const y = static_cast<T*>(to.rows) + static_cast<int64_t>(within) * a.ld_rows;
  const int of = there ? of_row<LINES>(embed_shard(id, a.vs, a.vocab_shards)) : 0;
  const T* const w = static_cast<const T*>(first_kernel_argument<A>()->vocab[of]) + (there ? static_cast<int64_t>(id - of * a.vs) * a.ld_vocab : 0);
  const int col0 = (((piece * kEmbedUnroll) << log) + (lane & ((1 << log) - 1))) * n, step = n << log;
  u32x4_t v[kEmbedUnroll];
  if (there) {
#pragma unroll
    for (int u = 0; u < kEmbedUnroll; ++u) v[u] = load_line<LINES, T>(w, line_at<LINES, T>(col0 + u * step, a.M), a.M);
  } else {
#pragma unroll
    for (int u = 0; u < kEmbedUnroll; ++u) v[u] = u32x4_t{0u, 0u, 0u, 0u};
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
    if (col < a.M) store_line<LINES, T>(y, line_at<LINES, T>(col, a.M), a.M, v[u]);
  }
}

// y from [M, V]: 64 tokens x 32 columns of y a workgroup.  A lane has a token and reads its column of eight rows of w, element by element: neighbouring tokens' entries lie anywhere in a row, so what
// has to be near is the row.  Workgroups of one XCD take the same 32 rows of w for all tokens, one after the other, out of its L2.  Bound by
// one line a cycle from the caches for every lane (19870 tokens of 1792 from 5248 entries: 87 us).
constexpr int kColumnTokens = 64, kColumnCols = 32;
template <typename T, typename A>
__global__ __launch_bounds__(256) void embed_columns_kernel(const A a, int col_blocks) {
  __shared__ float tile[kColumnTokens][kColumnCols + 1];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int xcd = blockIdx.x & 7, block = xcd + 8 * blockIdx.y;         // (eight divides gridDim.x)
  if (block >= col_blocks) return;
  const int row0 = (blockIdx.x >> 3) * kColumnTokens, col0 = block * kColumnCols, rows = a.ts * a.token_shards;
  {
    const int row = row0 + lane;
    int id = -1;
    if (row < a.T) {
      const int shard = embed_shard(row, a.ts, a.token_shards);
      id = ((GSPMD_GLOBAL const int32_t*)first_kernel_argument<A>()->tokens[shard].ids)[row - shard * a.ts];
    }
    const bool there = static_cast<uint32_t>(id) < static_cast<uint32_t>(a.V);
    const int of = there ? embed_shard(id, a.vs, a.vocab_shards) : 0;
    GSPMD_GLOBAL const T* const w = (GSPMD_GLOBAL const T*)first_kernel_argument<A>()->vocab[of] + (there ? id - of * a.vs : 0);
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
    T* const y = static_cast<T*>(first_kernel_argument<A>()->tokens[shard].rows);
    if (y == nullptr) continue;
    float f[n];
#pragma unroll
    for (int e = 0; e < n; ++e) f[e] = a.scale == 1.f ? tile[r][c + e] : tile[r][c + e] * a.scale;
    store_up_to(y + static_cast<int64_t>(row - shard * a.ts) * a.ld_rows + col, a.scale == 1.f ? Sixteen<T>::bits(f) : Sixteen<T>::close(f), a.M - col);
  }
}

// ---- the gradient
// dy's row of a token
template <typename T, typename A>
__device__ __forceinline__ const T* token_row(const A& a, int token) {
  const int shard = embed_shard(token, a.ts, a.token_shards);
  return static_cast<const T*>(first_kernel_argument<A>()->tokens[shard].rows) + static_cast<int64_t>(token - shard * a.ts) * a.ld_rows;
}

enum RunsTo { kRows, kAddedRows, kSums };        // what becomes of a run's sum: dw's row [V, M], the same added to what is there, or it is put by for dw [M, V]

// dw's row of an entry [V, M] from its sum.
template <typename T, int LINES, int TO, typename A>
__device__ __forceinline__ void finish_row(const A& a, int entry, int at, float (&sum)[Sixteen<T>::n]) {
  constexpr int n = Sixteen<T>::n;
  const int shard = of_row<LINES>(embed_shard(entry, a.vs, a.vocab_shards));
  T* dw = static_cast<T*>(first_kernel_argument<A>()->vocab[shard]);
  if (dw == nullptr) return;
  dw += static_cast<int64_t>(entry - shard * a.vs) * a.ld_vocab;
#pragma unroll
  for (int e = 0; e < n; ++e) sum[e] *= a.scale;
  if constexpr (TO == kAddedRows) {
    float f[n];
    Sixteen<T>::open(load_line<LINES, T>(dw, at, a.M), f);
#pragma unroll
    for (int e = 0; e < n; ++e) sum[e] += f[e];
  }
  store_line<LINES, T>(dw, at, a.M, Sixteen<T>::close(sum));
}

// Chunks of the order: a wave (or a few lanes of one, with short rows) has a chunk and 16 bytes a lane of its tokens' rows, all on their way together (2048 tokens of 2048: 6.8 us, 9999 of 1001 9.3).
// kSums: runs of several tokens are put by for embed_grad_columns_kernel, those of one it reads itself.  ALONE: of few tokens a run is added up by the chunk that it begins in, to its end, and there
// is nothing to join.
template <typename T, int LINES, int TO, int CHUNK, bool ALONE, typename A>
__global__ __launch_bounds__(256) void embed_runs_kernel(const A a, int log_lanes, int log_across) {
  constexpr int n = Sixteen<T>::n;
  const int log = LINES == kWide ? 6 : log_lanes, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int across = 1 << log_across, units = (4 >> log_across) << (6 - log);              // waves along a row; chunks of a workgroup
  const int chunk = of_row<LINES>(blockIdx.x * units + ((wave >> log_across) << (6 - log)) + (lane >> log));
  const int col = (((blockIdx.y * across + (wave & (across - 1))) << log) + (lane & ((1 << log) - 1))) * n;
  const int total = ((GSPMD_GLOBAL const int32_t*)a.begins)[a.V], begin = chunk * CHUNK, end = min(begin + CHUNK, total);
  if (begin >= total || col >= a.M) return;
  GSPMD_GLOBAL const int32_t* const order = (GSPMD_GLOBAL const int32_t*)a.order;
  GSPMD_GLOBAL const int32_t* const entries = (GSPMD_GLOBAL const int32_t*)a.entries;
  const int at = line_at<LINES, T>(col, a.M);
  int first = begin;                                                                       // the run's first place here
  bool open = false;                                                                       // it began before the chunk
  float sum[n];
#pragma unroll
  for (int e = 0; e < n; ++e) sum[e] = 0.f;
#pragma unroll 1
  for (int base = begin; base < total; base += CHUNK) {
    int entry[CHUNK + 1];
    u32x4_t v[CHUNK];
#pragma unroll
    for (int u = 0; u < CHUNK; ++u) {           // (places up to the chunk's end exist; those behind the last token hold anything)
      const int token = of_row<LINES>(order[base + u]);
      entry[u] = of_row<LINES>(entries[base + u]);
      v[u] = load_line<LINES, T>(token_row<T>(a, base + u < total ? token : 0), at, a.M);
    }
    entry[CHUNK] = base + CHUNK < total ? of_row<LINES>(entries[base + CHUNK]) : a.V;
    if (base == begin) open = begin > 0 && of_row<LINES>(entries[max(begin - 1, 0)]) == entry[0];
    bool done = !ALONE;
#pragma unroll
    for (int u = 0; u < CHUNK; ++u) {
      const int place = base + u;
      if (place < total && (!ALONE || !done)) {
        float f[n];
        Sixteen<T>::open(v[u], f);
#pragma unroll
        for (int e = 0; e < n; ++e) sum[e] += f[e];
        const bool ends = place + 1 == total || entry[u + 1] != entry[u];
        if (ends || (!ALONE && place + 1 == end)) {
          const bool part = open || !ends;
          if (ALONE && open) {                  // another chunk's
          } else if (part || TO == kSums) {
            float* const to = open ? a.heads + static_cast<int64_t>(chunk) * a.M : part ? a.tails + static_cast<int64_t>(chunk) * a.M : a.sums + static_cast<int64_t>(first >> 1) * a.M;
            if (part || first != place) store_sums<LINES, n>(to, at, a.M, sum);
          } else {
            finish_row<T, LINES, TO>(a, entry[u], at, sum);
          }
          open = false;
          first = place + 1;
          done = !ALONE || first >= end;        // the next run begins in another chunk
#pragma unroll
          for (int e = 0; e < n; ++e) sum[e] = 0.f;
        }
      }
    }
    if (done || open) break;                    // (open: all of the chunk belongs to a run of an earlier one)
  }
}

// Runs of several chunks: a workgroup for the chunk that one begins in (blockIdx.x) and 64 x 16 bytes of the row (blockIdx.y), a wave every fourth of the chunks behind it.  (4 us where there are
// hardly any, and the launch is all.)
template <typename T, int LINES, int TO, int CHUNK, typename A>
__global__ __launch_bounds__(256) void embed_joins_kernel(const A a) {
  constexpr int n = Sixteen<T>::n, kAhead = 4;
  const int chunk = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  GSPMD_GLOBAL const int32_t* const entries = (GSPMD_GLOBAL const int32_t*)a.entries;
  GSPMD_GLOBAL const int32_t* const begins = (GSPMD_GLOBAL const int32_t*)a.begins;
  const int begin = chunk * CHUNK, end = begin + CHUNK;
  if (end >= begins[a.V]) return;               // nothing behind it
  const int entry = entries[end - 1];
  if (entries[end] != entry || begins[entry] < begin) return;
  const int last = (begins[entry + 1] - 1) / CHUNK, col = (blockIdx.y * 64 + lane) * n, at = line_at<LINES, T>(col, a.M);
  float sum[n];
#pragma unroll
  for (int e = 0; e < n; ++e) sum[e] = 0.f;
#pragma unroll 1
  for (int c = chunk + 1 + wave; c <= last; c += 4 * kAhead) {
    float v[kAhead][n];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load_sums<LINES, n>(a.heads + static_cast<int64_t>(min(c + 4 * u, last)) * a.M, at, a.M, v[u]);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int e = 0; e < n; ++e) sum[e] += c + 4 * u <= last ? v[u][e] : 0.f;
  }
  __shared__ float sums[4][n][64];
#pragma unroll
  for (int e = 0; e < n; ++e) sums[wave][e][lane] = sum[e];
  __syncthreads();
  if (wave > 0 || col >= a.M) return;
  load_sums<LINES, n>(a.tails + static_cast<int64_t>(chunk) * a.M, at, a.M, sum);
#pragma unroll
  for (int w = 0; w < 4; ++w)
#pragma unroll
    for (int e = 0; e < n; ++e) sum[e] += sums[w][e][lane];
  if constexpr (TO == kSums) store_sums<LINES, n>(a.sums + static_cast<int64_t>(begins[entry] >> 1) * a.M, at, a.M, sum);
  else finish_row<T, LINES, TO>(a, entry, at, sum);
}

// sum += the rows of `count` tokens from place `begin` of the order on, eight on their way at a time.
template <typename T, int LINES, typename A>
__device__ __forceinline__ void add_run(const A& a, int begin, int count, int at, float (&sum)[Sixteen<T>::n]) {
  constexpr int n = Sixteen<T>::n, kAhead = 8;
  GSPMD_GLOBAL const int32_t* const order = (GSPMD_GLOBAL const int32_t*)a.order + begin;
#pragma unroll 1
  for (int i = 0; i < count; i += kAhead) {
    u32x4_t v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = load_line<LINES, T>(token_row<T>(a, order[min(i + u, count - 1)]), at, a.M);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float f[n];
      Sixteen<T>::open(v[u], f);
#pragma unroll
      for (int e = 0; e < n; ++e) sum[e] += i + u < count ? f[e] : 0.f;
    }
  }
}

// dw [M, V]: 64 entries x 16 lanes' 16 bytes of dw's rows a workgroup.  Sixteen lanes have an entry, four of them one after the other, on their way together: the row of its token, or the sum of its
// tokens' (ALONE: added up here, of few tokens; 100 of 896, 2560 entries, in two launches 14.7 -> 11.5 us).  They turn in LDS, rounded but for what is still to be added to (TTile float).  Bound by waits, for where runs begin, their tokens and the rows (9999 tokens, 1001 x 32003: 22 us, 64 MB of
// dw at 2.9 TB/s; 48 in all with neighbouring tiles on different XCDs, 44 with one).
// Added to what is there every tile reads its part of dw, too: 53 in all; 100 tokens, 2048 x 32000 51, written whole 36.
constexpr int kTurnEntries = 64, kTurnLanes = 16;
template <typename T, int LINES, typename TTile, bool ALONE, typename A>
__global__ __launch_bounds__(256) void embed_grad_columns_kernel(const A a, int blocks_x) {
  constexpr int n = Sixteen<T>::n, kRows = kTurnLanes * n, side = 64 / kTurnLanes, kEach = kTurnEntries / (4 * side), kPitch = kTurnEntries + (sizeof(TTile) == 2 ? 2 : 1);
  __shared__ __attribute__((aligned(4))) TTile tile[n + kRows][kPitch];        // (n rows before the tile's: what the lane at the row's end has of its neighbours' may begin there)
  __shared__ int begins[kTurnEntries + 1];
  // Of a row of the tile as words of dw, what is added to what is there, and what keeps its bits: entries without tokens, which float32 and back would change (a signalling NaN).  Padding is neither, and 0.
  constexpr int kWords = sizeof(TTile) == 4 ? kTurnEntries * sizeof(T) / 4 : 0;
  __shared__ __attribute__((aligned(16))) uint32_t added[kWords > 0 ? kWords : 1], kept[kWords > 0 ? kWords : 1];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  // neighbouring entries' tiles, whose lines of dw are shared where rows are not aligned, on one XCD
  const int logical = logical_tile(blockIdx.x, gridDim.x), block_m = logical / blocks_x, block_x = logical - block_m * blocks_x;
  // entries of one shard: block_x counts blocks of every shard
  const int per_shard = (a.vs + kTurnEntries - 1) / kTurnEntries, shard = block_x / per_shard, c0 = (block_x - shard * per_shard) * kTurnEntries;
  const int row0 = shard * a.vs + c0, m0 = block_m * kRows, entries = min(kTurnEntries, a.vs - c0);
  T* const dw = static_cast<T*>(first_kernel_argument<A>()->vocab[shard]);
  if (dw == nullptr) return;
  if (t <= kTurnEntries) begins[t] = a.T > 0 ? ((GSPMD_GLOBAL const int32_t*)a.begins)[min(row0 + t, a.V)] : 0;
  __syncthreads();
  if (a.accumulate && t < kWords) {
    constexpr int each = 4 / sizeof(T);
    uint32_t sums = 0u, same = 0u;
#pragma unroll
    for (int i = 0; i < each; ++i) {
      const int r = t * each + i;
      const uint32_t bits = each == 1 ? ~0u : 0xffffu << 16 * i;
      if (begins[r] != begins[r + 1]) sums |= bits;
      else if (row0 + r < a.V) same |= bits;
    }
    added[t] = sums;
    kept[t] = same;
  }
  const int col = m0 + (lane & (kTurnLanes - 1)) * n, at = line_at<LINES, T>(col, a.M), r0 = wave * side + lane / kTurnLanes;
  int begin[kEach], count[kEach], token[kEach];
  u32x4_t v[kEach];
  bool any = false;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int r = r0 + u * 4 * side;
    begin[u] = begins[r];
    count[u] = r < entries ? begins[r + 1] - begin[u] : 0;
    any = any || count[u] > 0;
    v[u] = u32x4_t{0u, 0u, 0u, 0u};
    token[u] = 0;
  }
  if (any && col < a.M) {
#pragma unroll
    for (int u = 0; u < kEach; ++u) token[u] = ((GSPMD_GLOBAL const int32_t*)a.order)[count[u] > 0 ? begin[u] : 0];
#pragma unroll
    for (int u = 0; u < kEach; ++u) v[u] = load_line<LINES, T>(token_row<T>(a, count[u] > 0 ? token[u] : 0), at, a.M);
  }
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    float sum[n];
    Sixteen<T>::open(v[u], sum);
    if (count[u] > 1 && col < a.M) {
      if constexpr (ALONE) add_run<T, LINES>(a, begin[u] + 1, count[u] - 1, at, sum);
      else load_sums<LINES, n>(a.sums + static_cast<int64_t>(begin[u] >> 1) * a.M, at, a.M, sum);
    }
#pragma unroll
    for (int e = 0; e < n; ++e)
      if (col < a.M) store_from_float<TTile>(&tile[n + at - m0 + e][r0 + u * 4 * side], count[u] > 0 ? sum[e] * a.scale : 0.f);
  }
  __syncthreads();
  for (int i = t; i < kRows * (kTurnEntries / n); i += 256) {
    const int m = i / (kTurnEntries / n), c = (i - m * (kTurnEntries / n)) * n, keep = entries - c;
    if (m0 + m >= a.M || keep <= 0) continue;
    T* const to = dw + (m0 + m) * a.ld_vocab + c0 + c;
    if constexpr (sizeof(TTile) == 2) {
      u32x4_t o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = *reinterpret_cast<const uint32_t*>(&tile[n + m][c + 2 * e]);
      store_up_to(to, o, keep);
    } else {
      float f[n];
#pragma unroll
      for (int e = 0; e < n; ++e) f[e] = tile[n + m][c + e];
      if (a.accumulate) {
        const u32x4_t held = load_up_to(to, keep);
        float before[n];
        Sixteen<T>::open(held, before);
#pragma unroll
        for (int e = 0; e < n; ++e) f[e] += before[e];
        const int at = c / n * 4;
        store_up_to(to, (held & *reinterpret_cast<const u32x4_t*>(kept + at)) | (Sixteen<T>::close(f) & *reinterpret_cast<const u32x4_t*>(added + at)), keep);
      } else {
        store_up_to(to, Sixteen<T>::close(f), keep);
      }
    }
  }
}

}  // namespace gspmd
