// The losses over a split vocabulary (softmax.hip): what happens beside the products.
//
// A row of logits z holds the vocabulary's shards one after the other, each `per_cols` columns wide, of which the first `per` (of the last shard: what is left of the vocabulary) stand for entries.
// per_cols is a multiple of 8, so that no vector of four logits and no 16 bytes of an operand lie in two shards, and of 64 where the products may end in statistics.  With u = z / tau, the entries' maximum m and total = sum exp(u - m), and the token's
// targets p (one label: p = 1; a teacher's entries: the softmax of their logits / tau):
//   lse = m + log(total)     loss = sum_k p_k (log p_k - (u_k - lse))     D = weight / tau (exp(u - lse) - p)
// D replaces the logits in place, in the operands' type: a bfloat16 row then takes the first half of its float32 row's bytes.  Everything up to D is float32, and D is
// rounded to the operands' type once: it is an operand of the products that make the gradients, whose matrix instructions take that type.  With few tokens what that rounding loses is kept as a second
// row (LOST) and takes part in the products too, which are bound by the vocabulary matrix then; with many it would be twice the flops of two products of three.  exp is v_exp_f32 of the exponent times log2(e), of differences to the maximum.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernels_basic.h"
#include "mfma_common.h"

namespace gspmd {

// One shard of tokens: its arrays (device), all of them in the shard's static size.
struct TokenShard {
  const int32_t* ids;            // [tokens, targets]
  const void* logits;            // [tokens, targets], float32 or bfloat16; null: one label
  const float* weights;          // [tokens]; null: 1
  float* loss;                   // [tokens]
  float* lse;                    // [tokens]; null: not wanted
};
constexpr int kInlineTokenShards = 64;

struct SoftmaxRows {
  TokenShard shard[kInlineTokenShards];
  float* z;                      // the row of token `first`
  int64_t ldz;                   // float32 elements
  int64_t lost;                  // rows from D to what its rounding lost
  int32_t first, tokens, per_shard;        // first token of the launch, tokens in all, and of a shard
  int32_t first_shard;           // the table's first
  int32_t cols, vocab, per, per_cols, targets;
  FastDiv by_cols;               // by per_cols
  float inv_tau;
  int32_t logits_bf16;
  const bf16_bits* x;            // with D in two parts: the tokens' activations (of one shard), put together beside them, or null
  bf16_bits* x_copies;           // two of them, `lost` rows apart
  int64_t ldx, ld_copy;
  int32_t x_cols;
};
static_assert(sizeof(SoftmaxRows) <= 4096, "kernel arguments");

template <typename Op>
__device__ __forceinline__ float over_wave(float v, Op op) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = op(v, __shfl_xor(v, d));
  return v;
}
template <int THREADS, typename Op>
__device__ __forceinline__ float over_block(float v, float* shared, Op op) {
  v = over_wave(v, op);
  if constexpr (THREADS > 64) {
    constexpr int kWaves = THREADS / 64;
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = shared[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = op(v, shared[w]);
    __syncthreads();             // the words are free again
  }
  return v;
}

constexpr float kLog2e = 1.4426950408889634f;

// The teacher's logit of a target; of a label 0.
__device__ __forceinline__ float teachers_logit(const GSPMD_KERNARG TokenShard& s, int is_bf16, int64_t at) {
  if (s.logits == nullptr) return 0.f;
  return is_bf16 ? bf16_to_float(static_cast<const bf16_bits*>(s.logits)[at]) : static_cast<const float*>(s.logits)[at];
}

// A token's targets, by one wave: shares p_k = softmax of q_k / tau (-infinity: no target), given to `keep`, and sum_k p_k (log p_k - u_k).  Differences to the largest q are divided by tau, not the q: at
// a tau below 1 the lowest and largest values of their type would become infinite.
// A NaN among the teacher's logits stays: the shares, the loss and the gradient of its token are NaN.
struct TargetSums {
  bool any;
  float sum;
};
template <typename Q, typename U, typename Keep>
__device__ __forceinline__ TargetSums over_targets(int K, float inv_tau, Q q_of, U u_of, Keep keep) {
  const int lane = threadIdx.x & 63;
  auto most = [](float x, float y) { return x != x ? x : y != y ? y : fmaxf(x, y); };
  auto plus = [](float x, float y) { return x + y; };
  // A label, most often: p = 1 (of a logit that is no number: none), without the exchanges (1 us of a row, for which its other waves wait: 1 token, 2048 x 32000 36.5 -> 35.5, 16 tokens, 1024 x 8000 with
  // gradients 33.6 -> 32.7).
  if (K == 1) {
    auto first_lane = [](float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); };
    const float q = first_lane(q_of(0)), zero = q - q;
    if (q == -INFINITY) return TargetSums{false, 0.f};
    if (lane == 0) keep(0, 1.f + zero);
    return TargetSums{true, (1.f + zero) * (zero - first_lane(u_of(0)))};
  }
  float q_most = -INFINITY;
  for (int k = lane; k < K; k += 64) q_most = most(q_most, q_of(k));
  q_most = over_wave(q_most, most);
  if (q_most == -INFINITY) return TargetSums{false, 0.f};
  float total = 0.f, sum = 0.f;
  for (int k = lane; k < K; k += 64) total += __builtin_amdgcn_exp2f((q_of(k) - q_most) * inv_tau * kLog2e);
  total = over_wave(total, plus);
  const float log_total = logf(total);
  for (int k = lane; k < K; k += 64) {
    const float q = (q_of(k) - q_most) * inv_tau, p = __builtin_amdgcn_exp2f(q * kLog2e) / total;
    if (p != 0.f) sum += p * ((q - log_total) - u_of(k));
    keep(k, p);
  }
  return TargetSums{true, over_wave(sum, plus)};
}

// Bound by memory: reads 4 bytes a logit, writes 2 (4 in float32).  A workgroup takes a row and keeps it in registers between the maximum and D, so that it is read once (LONG,
// beyond 64 K columns: twice, the second time mostly from the caches).  The row's loads go first: what a token's targets need, two accesses one after the other, comes while they are under way.
// Measured: 2048 x 32000 bfloat16 73 us (393 MB, 5.4 TB/s), 16384 x 32000 580 (3.1 GB, 5.4 TB/s); one workgroup of 1024 a compute unit beyond 32 K columns, 1365 x 41728 87 (3.9 TB/s); 16 x 32000, a row a
// compute unit, 15, of which its instructions are about half.
// T: the operands' type.  A thread holds VECS vectors of 4 logits; LONG: rows of more than THREADS * VECS * 4, taken in several rounds.
template <typename T, int THREADS, int VECS, bool LONG, bool GRAD, bool LOST>
__global__ __launch_bounds__(THREADS, LONG ? 6 : VECS <= 8 ? 8 : 4) void softmax_rows_kernel(const SoftmaxRows args) {
  extern __shared__ __attribute__((aligned(16))) float targets_lds[];       // u, p (first: the teacher's logit) and id of every target, in fours
  __shared__ float shared[16];
  __shared__ bool any_target;
  const GSPMD_KERNARG SoftmaxRows& a = *first_kernel_argument<SoftmaxRows>();
  const int t = threadIdx.x;
  const int at_token = a.first + static_cast<int>(blockIdx.x), i = at_token / a.per_shard, token = at_token - i * a.per_shard;
  const GSPMD_KERNARG TokenShard& s = a.shard[i - a.first_shard];
  if (at_token >= a.tokens) {                   // padding of the last shards
    if (t == 0) {
      s.loss[token] = 0.f;
      if (s.lse) s.lse[token] = 0.f;
    }
    return;
  }
  float* const z = a.z + static_cast<int64_t>(blockIdx.x) * a.ldz;
  const int K = a.targets, K4 = (K + 3) & ~3;
  const float inv_tau = a.inv_tau, c = inv_tau * kLog2e;
  float *const u_of = targets_lds, *const p_of = targets_lds + K4;
  int32_t* const id_of = reinterpret_cast<int32_t*>(targets_lds + 2 * K4);
  const FastDiv by_cols{a.by_cols.mul, a.by_cols.shift};
  auto column = [&](int id) {
    const int j = id / a.per;
    return j * a.per_cols + (id - j * a.per);
  };
  const uint32_t lane_bytes = static_cast<uint32_t>(t) * 16;     // (a uniform part and 32 bits of the lane's own: fewer registers than an address for each vector)
  auto load = [&](int at) { return *(GSPMD_GLOBAL const float4_t*)((GSPMD_GLOBAL const char*)(GSPMD_GLOBAL const float*)(z + at) + lane_bytes); };
  auto cut = [&](int at, float4_t& x) {         // columns that are no entries
    const int j = static_cast<int>(div_by(static_cast<uint32_t>(at), by_cols));
    const int n = min(a.per, a.vocab - j * a.per) - (at - j * a.per_cols);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e >= n) x[e] = -INFINITY;
  };
  const float4_t none = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  constexpr int kRound = THREADS * 4 * VECS;
  float4_t x[VECS];
  auto load_round = [&](int first) {
#pragma unroll
    for (int n = 0; n < VECS; ++n) {
      const int at = first + (n * THREADS + t) * 4;
      x[n] = none;
      if (at < a.cols) x[n] = load(first + n * THREADS * 4);
    }
  };
  load_round(0);
  if constexpr (LOST)
    if (a.x)
      for (int m = t; m < a.x_cols; m += THREADS) {
        const bf16_bits v = a.x[static_cast<int64_t>(token) * a.ldx + m];
        bf16_bits* const to = a.x_copies + static_cast<int64_t>(blockIdx.x) * a.ld_copy + m;
        to[0] = v;
        to[a.lost * a.ld_copy] = v;
      }
  auto plus = [](float x, float y) { return x + y; };

  // ---- the targets, by the first wave: their logits (before D takes the logits' place), shares, and what the loss takes from them
  float of_targets = 0.f;                       // sum_k p_k (log p_k - u_k)
  if (t < 64) {
    for (int k = t; k < K; k += 64) {
      const int64_t at = static_cast<int64_t>(token) * K + k;
      int id = s.ids[at];
      if (id < 0 || id >= a.vocab) id = -1;
      u_of[k] = id >= 0 ? z[column(id)] * inv_tau : 0.f;
      p_of[k] = id >= 0 ? teachers_logit(s, a.logits_bf16, at) : -INFINITY;
      id_of[k] = id;
    }
    if (t < K4 - K) id_of[K + t] = -1;
    const TargetSums of = over_targets(K, inv_tau, [&](int k) { return p_of[k]; }, [&](int k) { return u_of[k]; }, [&](int k, float p) { p_of[k] = p; });
    of_targets = of.sum;
    if (t == 0) any_target = of.any;
  }

  // ---- maximum and total
  float m = -INFINITY, total = 0.f;
  for (int first = 0; first < (LONG ? a.cols : 1); first += kRound) {
    if (LONG && first > 0) load_round(first);
    float here = -INFINITY;
#pragma unroll
    for (int n = 0; n < VECS; ++n) {
      cut(first + (n * THREADS + t) * 4, x[n]);
#pragma unroll
      for (int e = 0; e < 4; ++e) here = fmaxf(here, x[n][e]);
    }
    if constexpr (LONG) {        // a running maximum and sum of this thread's own
      const float next = fmaxf(m, here), from = next == -INFINITY ? 0.f : next;
      total *= __builtin_amdgcn_exp2f((m - from) * c);
#pragma unroll
      for (int n = 0; n < VECS; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) total += __builtin_amdgcn_exp2f((x[n][e] - from) * c);
      m = next;
    } else {
      m = here;
    }
  }
  const float own = m;
  m = over_block<THREADS>(m, shared, [](float p, float q) { return fmaxf(p, q); });
  const float finite_m = m == -INFINITY ? 0.f : m;               // a row of -infinity: total 0, lse -infinity
  if constexpr (LONG) {
    total = own == -INFINITY ? total : total * __builtin_amdgcn_exp2f((own - m) * c);
  } else {
#pragma unroll
    for (int n = 0; n < VECS; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[n][e] = __builtin_amdgcn_exp2f((x[n][e] - finite_m) * c);
        total += x[n][e];
      }
  }
  total = over_block<THREADS>(total, shared, plus);
  const float u_most = m * inv_tau, log_total = logf(total);

  if constexpr (THREADS == 64) __syncthreads();
  const bool any = any_target;                  // (written before the barrier above, or those of the sums)
  if (t == 0) {
    s.loss[token] = any ? of_targets + u_most + log_total : 0.f;
    if (s.lse) s.lse[token] = u_most + log_total;
  }

  // ---- D in the logits' place.  A round's logits have all been read (the barrier) before any of it is written; what bfloat16 writes lies no further on than what
  // has been read.
  if constexpr (GRAD) {
    const float weight = s.weights ? s.weights[token] : 1.f;
    const float scale = any ? weight * inv_tau : 0.f, factor = scale / total;
    GSPMD_GLOBAL T* const d = (GSPMD_GLOBAL T*)reinterpret_cast<T*>(z);
    GSPMD_GLOBAL T* const d_lost = (GSPMD_GLOBAL T*)reinterpret_cast<T*>(z + a.lost * a.ldz);
    typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4_t;
    auto store = [&](int at, float4_t v) {      // (at: the first thread's)
      constexpr int kBytes = 4 * static_cast<int>(sizeof(T));
      auto place = [&](GSPMD_GLOBAL T* row) { return (GSPMD_GLOBAL char*)(row + at) + lane_bytes / 16 * kBytes; };
      if (scale == 0.f) v = float4_t{0.f, 0.f, 0.f, 0.f};         // (a token without targets takes no part, whatever its logits are)
      if constexpr (sizeof(T) == 2) {
        const bf16x4_t r = {static_cast<__bf16>(v[0]), static_cast<__bf16>(v[1]), static_cast<__bf16>(v[2]), static_cast<__bf16>(v[3])};
        *(GSPMD_GLOBAL bf16x4_t*)place(d) = r;
        if constexpr (LOST)
          *(GSPMD_GLOBAL bf16x4_t*)place(d_lost) = bf16x4_t{static_cast<__bf16>(v[0] - static_cast<float>(r[0])), static_cast<__bf16>(v[1] - static_cast<float>(r[1])),
                                                               static_cast<__bf16>(v[2] - static_cast<float>(r[2])), static_cast<__bf16>(v[3] - static_cast<float>(r[3]))};
      } else {
        *(GSPMD_GLOBAL float4_t*)place(d) = v;
      }
    };
    for (int first = 0; first < (LONG ? a.cols : 1); first += kRound) {
      if constexpr (LONG) {
        load_round(first);
#pragma unroll
        for (int n = 0; n < VECS; ++n) {
          cut(first + (n * THREADS + t) * 4, x[n]);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[n][e] = __builtin_amdgcn_exp2f((x[n][e] - finite_m) * c);
        }
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < VECS; ++n) {
        const int at = first + (n * THREADS + t) * 4;
        if (at < a.cols) store(first + n * THREADS * 4, x[n] * factor);
      }
    }
    __syncthreads();                            // the targets' columns are written again, each by one thread (a target given twice: the same value by each)
    if (scale != 0.f)
      for (int k = t; k < K; k += THREADS) {
        const int id = id_of[k];
        if (id < 0) continue;
        float p = 0.f;
        for (int n = 0; n < K4; n += 4) {
          const int4 ids = *reinterpret_cast<const int4*>(id_of + n);
          if (ids.x == id) p += p_of[n];
          if (ids.y == id) p += p_of[n + 1];
          if (ids.z == id) p += p_of[n + 2];
          if (ids.w == id) p += p_of[n + 3];
        }
        const float v = scale * (__builtin_amdgcn_exp2f(((u_of[k] - u_most) - log_total) * kLog2e) - p);
        if constexpr (sizeof(T) == 2) {
          const __bf16 r = static_cast<__bf16>(v);
          d[column(id)] = __builtin_bit_cast(bf16_bits, r);
          if constexpr (LOST) d_lost[column(id)] = __builtin_bit_cast(bf16_bits, static_cast<__bf16>(v - static_cast<float>(r)));
        } else {
          d[column(id)] = v;
        }
      }
  }
}

// ---- logits that are not kept (kernels_stats.h): the targets' columns before the products, and what their tiles leave put together after them.
struct SoftmaxMerge {
  SoftmaxRows rows;              // z: the table of pairs [group][ldz rows], `cols` its groups
  int32_t* columns;              // [rows][targets]; of one shard of tokens and one of the vocabulary the targets' own ids
  float* logits;                 // [rows][targets]
  int32_t count;                 // rows of the launch (for the columns: tokens)
  int32_t end;                   // columns of a row of logits: others are none
};
static_assert(sizeof(SoftmaxMerge) <= 4096, "kernel arguments");

__device__ __forceinline__ int target_column(int id, int vocab, int per, int per_cols) {
  if (id < 0 || id >= vocab) return -1;
  const int j = id / per;
  return j * per_cols + (id - j * per);
}

__global__ __launch_bounds__(256) static void target_columns_kernel(const SoftmaxMerge args) {
  const GSPMD_KERNARG SoftmaxRows& a = first_kernel_argument<SoftmaxMerge>()->rows;
  const int K = a.targets;
  int32_t* const columns = first_kernel_argument<SoftmaxMerge>()->columns;
  const int64_t total = static_cast<int64_t>(first_kernel_argument<SoftmaxMerge>()->count) * K;
  for (int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; n < total; n += static_cast<int64_t>(gridDim.x) * 256) {
    const int row = static_cast<int>(n / K), g = a.first + row, i = g / a.per_shard;
    columns[n] = target_column(a.shard[i - a.first_shard].ids[static_cast<int64_t>(g - i * a.per_shard) * K + (n - static_cast<int64_t>(row) * K)], a.vocab, a.per, a.per_cols);
  }
}

// Bound by memory, and by a row's chain of loads where there are few: 16384 x 32000 21 us (66 MB of pairs, 3.1 TB/s), 1024 x 128000 with 100 targets 15 (17 MB).
// TOKENS tokens a workgroup (16, whose pairs are whole lines, or with few tokens 4): the threads go through the groups of 64 columns, then a wave takes a token's targets.
constexpr int kMergeThreads = 1024;
constexpr int32_t kStatsTargets = 128;           // of a token, at most
template <int TOKENS>
__global__ __launch_bounds__(kMergeThreads) void softmax_merge_kernel(const SoftmaxMerge args) {
  constexpr int kMergeTokens = TOKENS, kSides = kMergeThreads / TOKENS;
  const GSPMD_KERNARG SoftmaxRows& a = first_kernel_argument<SoftmaxMerge>()->rows;
  typedef __attribute__((ext_vector_type(2))) float float2_t;
  __shared__ float2_t part[kSides][kMergeTokens];
  const int count = first_kernel_argument<SoftmaxMerge>()->count;
  const int t = threadIdx.x, r = t & (kMergeTokens - 1), row0 = blockIdx.x * kMergeTokens;
  const float inv_tau = a.inv_tau, c = inv_tau * kLog2e;
  GSPMD_GLOBAL const float2_t* const pairs = (GSPMD_GLOBAL const float2_t*)a.z;
  auto join = [&](float2_t p, float2_t q) {
    const float m = fmaxf(p.x, q.x), from = m == -INFINITY ? 0.f : m;
    return float2_t{m, p.y * __builtin_amdgcn_exp2f((p.x - from) * c) + q.y * __builtin_amdgcn_exp2f((q.x - from) * c)};
  };
  // this wave's token and its targets, two a lane: on their way first
  const int wave = t >> 6, lane = t & 63, g = a.first + row0 + wave, i = g / a.per_shard, token = g - i * a.per_shard, K = a.targets;
  const bool has_row = wave < kMergeTokens && row0 + wave < count, has_token = has_row && g < a.tokens;
  const GSPMD_KERNARG TokenShard& s = a.shard[has_row ? i - a.first_shard : 0];
  const int64_t at = static_cast<int64_t>(row0 + wave) * K;
  float q[2], u[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int k = n * 64 + lane;
    q[n] = -INFINITY;
    u[n] = 0.f;
    const int column = has_token && k < K ? ((GSPMD_GLOBAL const int32_t*)first_kernel_argument<SoftmaxMerge>()->columns)[at + k] : -1;
    if (column >= 0 && column < first_kernel_argument<SoftmaxMerge>()->end) {
      q[n] = teachers_logit(s, a.logits_bf16, static_cast<int64_t>(token) * K + k);
      u[n] = ((GSPMD_GLOBAL const float*)first_kernel_argument<SoftmaxMerge>()->logits)[at + k] * inv_tau;
    }
  }
  float2_t mine = {-INFINITY, 0.f};
  if (row0 + r < count && a.first + row0 + r < a.tokens)
    for (int group = t / kMergeTokens; group < a.cols; group += 4 * kSides) {
      float2_t next[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int at = group + n * kSides;
        next[n] = float2_t{-INFINITY, 0.f};
        if (at < a.cols) next[n] = pairs[static_cast<int64_t>(at) * a.ldz + row0 + r];
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) mine = join(mine, next[n]);
    }
  part[t / kMergeTokens][r] = mine;
  __syncthreads();
  if (!has_row) return;
  if (!has_token) {                             // padding of the last shards
    if (lane == 0) {
      s.loss[token] = 0.f;
      if (s.lse) s.lse[token] = 0.f;
    }
    return;
  }
  mine = part[lane][wave];
#pragma unroll
  for (int n = 64; n < kSides; n += 64) mine = join(mine, part[n + lane][wave]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) mine = join(mine, float2_t{__shfl_xor(mine.x, d), __shfl_xor(mine.y, d)});
  const float u_most = mine.x * inv_tau, log_total = logf(mine.y);
  const TargetSums of = over_targets(K, inv_tau, [&](int k) { return q[k >> 6]; }, [&](int k) { return u[k >> 6]; }, [](int, float) {});
  if (lane == 0) {
    s.loss[token] = of.any ? of.sum + u_most + log_total : 0.f;
    if (s.lse) s.lse[token] = u_most + log_total;
  }
}

// Shards put together in one padded matrix, 16 bytes a thread: rows of `per_row` from each row shard, of `per_col` columns (`cols` of it at most valid) from each column shard; zeros
// beyond what is valid.  Loads at the elements' alignment.  Bound by memory: 1001 x 32003 from 4 shards and 1999 x 1001 from 2 (136 MB read and written) 34 us, 4.0 TB/s; rows of whole
// lines, 32000 x 2048 from 4 shards and 4096 x 2048 (296 MB) 45 us, 6.5 TB/s.
struct PackRows {
  const void* from[kInlineTokenShards];
  void* to;                      // first row of the launch
  int64_t ld, ld_from;           // elements
  int32_t rows, chunks;          // of the result; 16-byte chunks of a row
  int32_t first, total, per_row;           // row shards: the result's first row is row `first` of all, rows that exist in all, rows apart in the result
  int32_t first_shard;           // the table's first
  int32_t by_columns;            // column shards (one row shard) instead
  int32_t per_cols, per, cols;   // column shards: columns apart in the result; shards of either kind: rows or columns of one; columns that exist in all
  int32_t copies, apart;         // the rows again, `apart` rows further on (of all of a piece's rows: a launch may have a table's only)
};
// One or two of them in a launch, whose workgroups are the first's across x down, then the second's.
struct PackTwo {
  PackRows two[2];
  int32_t across[2], down[2];
};
static_assert(sizeof(PackTwo) <= 4096, "kernel arguments");

template <typename T>
__global__ __launch_bounds__(256) void pack_rows_kernel(const PackTwo args) {
  const GSPMD_KERNARG PackTwo& both = *first_kernel_argument<PackTwo>();
  const int firsts = both.across[0] * both.down[0], which = static_cast<int>(blockIdx.x) >= firsts, block = blockIdx.x - which * firsts, across = both.across[which], down = both.down[which];
  const GSPMD_KERNARG PackRows& a = both.two[which];
  constexpr int V = 16 / static_cast<int>(sizeof(T));
  typedef T vec __attribute__((ext_vector_type(V)));
  typedef T vec_any __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  const int chunk = block % across * 256 + threadIdx.x;
  if (chunk >= a.chunks) return;
  for (int row = block / across; row < a.rows; row += down) {
    const int col = chunk * V;
    GSPMD_GLOBAL const T* from;
    int n;                                      // columns that exist from `col` on
    if (a.by_columns) {
      const int j = col / a.per_cols, at = col - j * a.per_cols;
      from = (GSPMD_GLOBAL const T*)a.from[j - a.first_shard] + static_cast<int64_t>(row) * a.ld_from + at;
      n = min(a.per, a.cols - j * a.per) - at;
    } else {
      const int g = a.first + row, i = g / a.per_row, at = g - i * a.per_row;
      from = (GSPMD_GLOBAL const T*)a.from[i - a.first_shard] + static_cast<int64_t>(at) * a.ld_from + col;
      n = at < a.per && i * a.per + at < a.total ? a.cols - col : 0;
    }
    vec v;
    if (n >= V) {
      v = *(GSPMD_GLOBAL const vec_any*)from;
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = 0;
#pragma unroll
      for (int e = 0; e < V - 1; ++e)
        if (e < n) v[e] = from[e];
    }
    GSPMD_GLOBAL T* const to = (GSPMD_GLOBAL T*)a.to + static_cast<int64_t>(row) * a.ld + col;
    for (int k = 0; k < a.copies; ++k) *(GSPMD_GLOBAL vec*)(to + static_cast<int64_t>(k) * a.apart * a.ld) = v;
  }
}

// Shards = the sum of `count` partials (fp32, one after the other) in ascending order; a launch's rows are rows first .. of all shards (dx: tokens; dw: entries), padding is written as zeros.
// Or the shards are beside each other, `apart` columns each, in every row.  Bound by memory: 4 partials of 2048 x 2048 to bfloat16 13.6 us (75 MB, 5.5 TB/s).
struct AddUp {
  void* to[kInlineTokenShards];
  const float* partials;         // [count][rows][cols]
  int64_t stride;                // elements from one partial to the next
  int64_t ld_in, ld_out;
  int32_t count, rows, cols;
  int32_t first, tokens, per_row, first_shard;     // tokens: rows (columns) that exist in all; per_row: of a shard
  int32_t apart;                 // rows (columns) from one shard to the next in the partials
  int32_t by_columns;
};
static_assert(sizeof(AddUp) <= 4096, "kernel arguments");

// Four columns a thread: partials' rows are padded to 16 bytes; the result is stored at its elements' alignment (column by column 8 partials of 1999 x 1001 took 26 us).
template <typename T>
__device__ __forceinline__ void store_sum(GSPMD_GLOBAL T* to, f32x4 sum, int n) {
  typedef T out_vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  out_vec o;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2) o[e] = __builtin_bit_cast(bf16_bits, static_cast<__bf16>(sum[e]));
    else o[e] = sum[e];
  }
  if (n >= 4) {
    *(GSPMD_GLOBAL out_vec*)to = o;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) to[e] = o[e];
  }
}

// begin .. end of the partials of four columns, four on their way at a time (one after the other, 32 of them took 9 us)
__device__ __forceinline__ f32x4 sum_partials(GSPMD_GLOBAL const float* from, int64_t stride, int begin, int end) {
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  int p = begin;
  auto at = [&](int n) { return *(GSPMD_GLOBAL const f32x4*)(from + static_cast<int64_t>(n) * stride); };
  for (; p + 4 <= end; p += 4) {
    const f32x4 a = at(p), b = at(p + 1), c = at(p + 2), d = at(p + 3);
    sum = (((sum + a) + b) + c) + d;
  }
  for (; p < end; ++p) sum += at(p);
  return sum;
}

template <typename T>
__global__ __launch_bounds__(256) void add_up_kernel(const AddUp args) {
  const GSPMD_KERNARG AddUp& a = *first_kernel_argument<AddUp>();
  const int col = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (col >= a.cols) return;
  for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (a.by_columns) {
      const int i = col / a.apart, at = col - i * a.apart, g = a.first + i * a.per_row + at;      // (beyond what exists: zeros, as D's columns are; of a shard without entries there are none)
      if (at >= a.per_row) continue;
      if (g < a.tokens) sum = sum_partials((GSPMD_GLOBAL const float*)a.partials + static_cast<int64_t>(row) * a.ld_in + col, a.stride, 0, a.count);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (g + e >= a.tokens) sum[e] = 0.f;
      store_sum<T>((GSPMD_GLOBAL T*)a.to[i] + static_cast<int64_t>(row) * a.ld_out + at, sum, a.per_row - at);
      continue;
    }
    const int g = a.first + row, i = g / a.per_row, at = g - i * a.per_row;
    const int64_t from = row + static_cast<int64_t>(i - a.first_shard) * (a.apart - a.per_row);
    if (g < a.tokens) sum = sum_partials((GSPMD_GLOBAL const float*)a.partials + from * a.ld_in + col, a.stride, 0, a.count);
    store_sum<T>((GSPMD_GLOBAL T*)a.to[i - a.first_shard] + static_cast<int64_t>(at) * a.ld_out + col, sum, a.cols - col);
  }
}

// rows x cols elements from one buffer to another: results for partitions that hold the same data in buffers of their own
template <typename T>
__global__ __launch_bounds__(256) void copy_rows_kernel(const T* __restrict__ from, T* __restrict__ to, int64_t rows, int64_t cols, int64_t ld_from, int64_t ld_to) {
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
    for (int64_t c = blockIdx.x * 256 + threadIdx.x; c < cols; c += static_cast<int64_t>(gridDim.x) * 256) to[r * ld_to + c] = from[r * ld_from + c];
}

}  // namespace gspmd
