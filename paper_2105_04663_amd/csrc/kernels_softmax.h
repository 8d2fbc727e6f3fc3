// The losses over a split vocabulary (softmax.hip): what happens to a piece of logits between the products.
//
// A row of logits z holds the vocabulary's shards one after the other, each `per_cols` columns wide (a multiple of 64), of which the first `per` (of the
// last shard: what is left of the vocabulary) stand for entries.  With u = z / tau, the entries' maximum m and total = sum exp(u - m), and the token's
// targets p (one label: p = 1; a teacher's entries: the softmax of their logits / tau):
//   lse = m + log(total)     loss = sum_k p_k (log p_k - (u_k - lse))     D = weight / tau (exp(u - lse) - p)
// D replaces the logits in place, in the operands' type: a bfloat16 row then takes the first half of its float32 row's bytes.  Everything up to D is float32, and D is
// rounded to the operands' type once: it is an operand of the products that make the gradients.
//
// Bound by memory: reads 4 bytes a logit, writes 2 (4 in float32).  A workgroup takes a row and keeps it in registers between the maximum and D, so that it is read once
// (rows beyond kLongest: twice, the second time mostly from the caches).
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
  int32_t valid, pad;            // tokens
};
constexpr int kInlineTokenShards = 64;

struct SoftmaxRows {
  TokenShard shard[kInlineTokenShards];
  void* z;                       // rows_per rows for each token shard
  int64_t ldz;                   // float32 elements
  int32_t rows_per, first;       // rows of a shard in this piece, and which of the shard's tokens is the first of them
  int32_t tokens;                // static tokens of a shard
  int32_t cols, vocab, per, per_cols, targets;
  FastDiv by_cols;               // by per_cols
  float inv_tau;
  int32_t logits_bf16;
};
static_assert(sizeof(SoftmaxRows) <= 4096, "kernel arguments");

template <int THREADS, typename Op>
__device__ __forceinline__ float over_block(float v, float* shared, Op op) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = op(v, __shfl_xor(v, d));
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

// T: the operands' type.  A thread holds VECS vectors of 4 logits; LONG: rows of more than THREADS * VECS * 4, taken in several rounds.
template <typename T, int THREADS, int VECS, bool LONG, bool GRAD>
__global__ __launch_bounds__(THREADS) void softmax_rows_kernel(const SoftmaxRows args) {
  extern __shared__ float targets_lds[];       // u, p (first: the teacher's logit / tau) and id of every target
  __shared__ float shared[16];
  const GSPMD_KERNARG SoftmaxRows& a = *first_kernel_argument<SoftmaxRows>();
  const int t = threadIdx.x;
  const int row = blockIdx.x, i = row / a.rows_per, token = a.first + row - i * a.rows_per;
  const GSPMD_KERNARG TokenShard& s = a.shard[i];
  if (token >= a.tokens) return;
  if (token >= s.valid) {
    if (t == 0) {
      s.loss[token] = 0.f;
      if (s.lse) s.lse[token] = 0.f;
    }
    return;
  }
  float* const z = static_cast<float*>(a.z) + static_cast<int64_t>(row) * a.ldz;
  const int K = a.targets;
  const float inv_tau = a.inv_tau, c = inv_tau * kLog2e;
  float *const u_of = targets_lds, *const p_of = targets_lds + K;
  int32_t* const id_of = reinterpret_cast<int32_t*>(targets_lds + 2 * K);
  auto column = [&](int id) {
    const int j = id / a.per;
    return j * a.per_cols + (id - j * a.per);
  };

  // ---- the targets: their logits (before D takes the logits' place) and shares
  const bool teacher = s.logits != nullptr;
  // (a NaN among the teacher's logits stays: the shares, the loss and the gradient of its token are NaN)
  auto most = [](float x, float y) { return x != x ? x : y != y ? y : fmaxf(x, y); };
  auto plus = [](float x, float y) { return x + y; };
  float q_most = -INFINITY;
  for (int k = t; k < K; k += THREADS) {
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
  q_most = over_block<THREADS>(q_most, shared, most);
  const bool any = q_most != -INFINITY;
  float q_total = 0.f;
  if (any) {
    for (int k = t; k < K; k += THREADS) q_total += __builtin_amdgcn_exp2f((p_of[k] - q_most) * kLog2e);
    q_total = over_block<THREADS>(q_total, shared, plus);
  }

  // ---- maximum and total
  const FastDiv by_cols{a.by_cols.mul, a.by_cols.shift};
  auto valid_columns = [&](int at) {            // of the four from `at` on
    const int j = static_cast<int>(div_by(static_cast<uint32_t>(at), by_cols)), v = at - j * a.per_cols;
    return max(0, min(min(a.per, a.vocab - j * a.per) - v, 4));
  };
  auto load = [&](int at) {
    float4_t x = *reinterpret_cast<const float4_t*>(z + at);
    const int n = valid_columns(at);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e >= n) x[e] = -INFINITY;
    return x;
  };
  const float4_t none = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  constexpr int kRound = THREADS * 4 * VECS;
  float4_t x[VECS];
  float m = -INFINITY, total = 0.f;
  for (int first = 0; first < (LONG ? a.cols : 1); first += kRound) {
#pragma unroll
    for (int n = 0; n < VECS; ++n) {
      const int at = first + (n * THREADS + t) * 4;
      x[n] = at < a.cols ? load(at) : none;
    }
    float here = -INFINITY;
#pragma unroll
    for (int n = 0; n < VECS; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) here = fmaxf(here, x[n][e]);
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
  const float u_most = m * inv_tau, log_total = logf(total), lse = u_most + log_total;

  // ---- the loss
  float loss = 0.f;
  if (any) {
    const float log_q = logf(q_total);
    for (int k = t; k < K; k += THREADS) {
      const float p = __builtin_amdgcn_exp2f((p_of[k] - q_most) * kLog2e) / q_total;
      if (p != 0.f) loss += p * ((p_of[k] - q_most - log_q) + ((u_most - u_of[k]) + log_total));
      p_of[k] = p;
    }
  }
  loss = over_block<THREADS>(loss, shared, plus);
  if (t == 0) {
    s.loss[token] = loss;
    if (s.lse) s.lse[token] = lse;
  }

  // ---- D in the logits' place.  A round's logits have all been read (the barrier) before any of it is written; what bfloat16 writes lies no further on than what
  // has been read.
  if constexpr (GRAD) {
    const float weight = s.weights ? s.weights[token] : 1.f;
    const float scale = any ? weight * inv_tau : 0.f, inv_total = 1.f / total;
    T* const d = reinterpret_cast<T*>(z);
    auto store = [&](int at, float4_t v) {
      if (scale == 0.f) v = float4_t{0.f, 0.f, 0.f, 0.f};         // (a token without targets takes no part, whatever its logits are)
      if constexpr (sizeof(T) == 2) {
        typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4_t;
        *reinterpret_cast<bf16x4_t*>(d + at) = bf16x4_t{static_cast<__bf16>(v[0]), static_cast<__bf16>(v[1]), static_cast<__bf16>(v[2]), static_cast<__bf16>(v[3])};
      } else {
        *reinterpret_cast<float4_t*>(d + at) = v;
      }
    };
    for (int first = 0; first < (LONG ? a.cols : 1); first += kRound) {
      if constexpr (LONG) {
#pragma unroll
        for (int n = 0; n < VECS; ++n) {
          const int at = first + (n * THREADS + t) * 4;
          x[n] = at < a.cols ? load(at) : none;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[n][e] = __builtin_amdgcn_exp2f((x[n][e] - m) * c);
        }
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < VECS; ++n) {
        const int at = first + (n * THREADS + t) * 4;
        if (at < a.cols) store(at, x[n] * (inv_total * scale));
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
        if constexpr (sizeof(T) == 2) d[column(id)] = __builtin_bit_cast(bf16_bits, static_cast<__bf16>(v));
        else d[column(id)] = v;
      }
  }
}

// rows x cols elements of SIZE bytes from one buffer to others: results for partitions that hold the same data in buffers of their own
template <typename T>
__global__ __launch_bounds__(256) void copy_rows_kernel(const T* __restrict__ from, T* __restrict__ to, int64_t rows, int64_t cols, int64_t ld_from, int64_t ld_to) {
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
    for (int64_t c = blockIdx.x * 256 + threadIdx.x; c < cols; c += static_cast<int64_t>(gridDim.x) * 256) to[r * ld_to + c] = from[r * ld_from + c];
}

}  // namespace gspmd
