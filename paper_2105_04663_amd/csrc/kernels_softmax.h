// The losses over a split vocabulary (softmax.hip): what happens beside the products.
//
// A row of logits z holds the vocabulary's shards one after the other, each `per_cols` columns wide (a multiple of 64), of which the first `per` (of the
// last shard: what is left of the vocabulary) stand for entries.  With u = z / tau, the entries' maximum m and total = sum exp(u - m), and the token's
// targets p (one label: p = 1; a teacher's entries: the softmax of their logits / tau):
//   lse = m + log(total)     loss = sum_k p_k (log p_k - (u_k - lse))     D = weight / tau (exp(u - lse) - p)
// D replaces the logits in place, in the operands' type: a bfloat16 row then takes the first half of its float32 row's bytes.  Everything up to D is float32, and D is
// rounded to the operands' type once: it is an operand of the products that make the gradients.  With few tokens what that rounding loses is kept as a second
// row (LOST) and takes part in the products too, which are bound by the vocabulary matrix then.
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

// Bound by memory: reads 4 bytes a logit, writes 2 (4 in float32).  A workgroup takes a row and keeps it in registers between the maximum and D, so that it is read once (LONG,
// beyond 48 K columns: twice, the second time mostly from the caches).  The row's loads go first: what a token's targets need, two accesses one after the other, comes while they are under way.
// T: the operands' type.  A thread holds VECS vectors of 4 logits; LONG: rows of more than THREADS * VECS * 4, taken in several rounds.
template <typename T, int THREADS, int VECS, bool LONG, bool GRAD, bool LOST>
__global__ __launch_bounds__(THREADS, LONG ? 6 : VECS <= 8 ? 8 : 5) void softmax_rows_kernel(const SoftmaxRows args) {
  extern __shared__ float targets_lds[];       // u, p (first: the teacher's logit / tau) and id of every target
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
  const int K = a.targets;
  const float inv_tau = a.inv_tau, c = inv_tau * kLog2e;
  float *const u_of = targets_lds, *const p_of = targets_lds + K;
  int32_t* const id_of = reinterpret_cast<int32_t*>(targets_lds + 2 * K);
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
  auto plus = [](float x, float y) { return x + y; };

  // ---- the targets, by the first wave: their logits (before D takes the logits' place), shares, and what the loss takes from them
  const bool teacher = s.logits != nullptr;
  float of_targets = 0.f;                       // sum_k p_k (log p_k - u_k)
  if (t < 64) {
    // (a NaN among the teacher's logits stays: the shares, the loss and the gradient of its token are NaN)
    auto most = [](float x, float y) { return x != x ? x : y != y ? y : fmaxf(x, y); };
    float q_most = -INFINITY;
    for (int k = t; k < K; k += 64) {
      const int64_t at = static_cast<int64_t>(token) * K + k;
      int id = s.ids[at];
      if (id < 0 || id >= a.vocab) id = -1;
      float u = 0.f, q = -INFINITY;
      if (id >= 0) {
        u = z[column(id)] * inv_tau;
        q = !teacher ? 0.f : (a.logits_bf16 ? bf16_to_float(static_cast<const bf16_bits*>(s.logits)[at]) : static_cast<const float*>(s.logits)[at]) * inv_tau;
        q_most = most(q_most, q);
      }
      u_of[k] = u;
      p_of[k] = q;
      id_of[k] = id;
    }
    q_most = over_wave(q_most, most);
    const bool some = q_most != -INFINITY;
    if (some) {
      float q_total = 0.f;
      for (int k = t; k < K; k += 64) {
        p_of[k] -= q_most;
        q_total += __builtin_amdgcn_exp2f(p_of[k] * kLog2e);
      }
      q_total = over_wave(q_total, plus);
      const float log_q = logf(q_total);
      for (int k = t; k < K; k += 64) {
        const float p = __builtin_amdgcn_exp2f(p_of[k] * kLog2e) / q_total;
        if (p != 0.f) of_targets += p * ((p_of[k] - log_q) - u_of[k]);
        p_of[k] = p;
      }
      of_targets = over_wave(of_targets, plus);
    }
    if (t == 0) any_target = some;
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
  if constexpr (LONG) {
    total = own == -INFINITY ? total : total * __builtin_amdgcn_exp2f((own - m) * c);
  } else {
#pragma unroll
    for (int n = 0; n < VECS; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[n][e] = __builtin_amdgcn_exp2f((x[n][e] - m) * c);
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
          for (int e = 0; e < 4; ++e) x[n][e] = __builtin_amdgcn_exp2f((x[n][e] - m) * c);
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
        for (int n = 0; n < K; ++n) p += id_of[n] == id ? p_of[n] : 0.f;
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

// Shards put together in one padded matrix, 16 bytes a thread: rows of `per_row` from each row shard, of `per_col` columns (`cols` of it at most valid) from each column shard; zeros
// beyond what is valid.  Loads at the elements' alignment.
struct PackRows {
  const void* from[kInlineTokenShards];
  void* to;                      // first row of the launch
  int64_t ld, ld_from;           // elements
  int32_t rows, chunks;          // of the result; 16-byte chunks of a row
  int32_t first, tokens, per_row;          // the result's first row is row `first` of all shards; rows that exist, and of a shard
  int32_t first_shard;           // the table's first
  int32_t by_columns;            // column shards (one row shard) instead
  int32_t per_cols, per, cols;   // column shards: columns apart in the result and wide, and columns that exist in all; else the row's `cols`
  int32_t copies;                // the rows again, `rows` further on
};
static_assert(sizeof(PackRows) <= 4096, "kernel arguments");

template <typename T>
__global__ __launch_bounds__(256) void pack_rows_kernel(const PackRows args) {
  const GSPMD_KERNARG PackRows& a = *first_kernel_argument<PackRows>();
  constexpr int V = 16 / static_cast<int>(sizeof(T));
  typedef T vec __attribute__((ext_vector_type(V)));
  typedef T vec_any __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const int chunk = blockIdx.x * 256 + threadIdx.x;
    if (chunk >= a.chunks) continue;
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
      n = g < a.tokens ? a.cols - col : 0;
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
    for (int k = 0; k < a.copies; ++k) *(GSPMD_GLOBAL vec*)(to + static_cast<int64_t>(k) * a.rows * a.ld) = v;
  }
}

// Token shards of dx = the sum of `count` partials (fp32, one after the other) in ascending order; a launch's rows are tokens first .. of all shards, padding is written as zeros.
struct AddUp {
  void* to[kInlineTokenShards];
  const float* partials;         // [count][rows][cols]
  int64_t stride;                // elements from one partial to the next
  int64_t ld_in, ld_out;
  int32_t count, rows, cols;
  int32_t first, tokens, per_row, first_shard;
};
static_assert(sizeof(AddUp) <= 4096, "kernel arguments");

template <typename T, int V>
__global__ __launch_bounds__(256) void add_up_kernel(const AddUp args) {
  const GSPMD_KERNARG AddUp& a = *first_kernel_argument<AddUp>();
  typedef float in_vec __attribute__((ext_vector_type(V)));
  for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const int col = (blockIdx.x * 256 + threadIdx.x) * V;
    if (col >= a.cols) continue;
    const int g = a.first + row, i = g / a.per_row, at = g - i * a.per_row;
    in_vec sum{};
    if (g < a.tokens) {
      GSPMD_GLOBAL const float* from = (GSPMD_GLOBAL const float*)a.partials + static_cast<int64_t>(row) * a.ld_in + col;
      sum = *(GSPMD_GLOBAL const in_vec*)from;
      for (int p = 1; p < a.count; ++p) sum += *(GSPMD_GLOBAL const in_vec*)(from + static_cast<int64_t>(p) * a.stride);
    }
    GSPMD_GLOBAL T* const to = (GSPMD_GLOBAL T*)a.to[i - a.first_shard] + static_cast<int64_t>(at) * a.ld_out + col;
    typedef T out_vec __attribute__((ext_vector_type(V)));
    out_vec o;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if constexpr (sizeof(T) == 2) o[e] = __builtin_bit_cast(bf16_bits, static_cast<__bf16>(sum[e]));
      else o[e] = sum[e];
    }
    *(GSPMD_GLOBAL out_vec*)to = o;
  }
}

// rows x cols elements from one buffer to another: results for partitions that hold the same data in buffers of their own
template <typename T>
__global__ __launch_bounds__(256) void copy_rows_kernel(const T* __restrict__ from, T* __restrict__ to, int64_t rows, int64_t cols, int64_t ld_from, int64_t ld_to) {
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
    for (int64_t c = blockIdx.x * 256 + threadIdx.x; c < cols; c += static_cast<int64_t>(gridDim.x) * 256) to[r * ld_to + c] = from[r * ld_from + c];
}

}  // namespace gspmd
