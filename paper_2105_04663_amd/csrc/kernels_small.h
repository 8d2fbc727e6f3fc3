// The losses over a split vocabulary where the whole vocabulary matrix is small (softmax.hip): a workgroup takes 16 tokens through everything -- their logits, which stay in LDS, the softmax,
// D in the logits' place, their rows of dx, and, where 16 tokens are all there are, its share of dw.
//
// These calls are bound by launches and by what their kernels wait for, not by memory or arithmetic: the others take four to six launches of 5 to 8 us (8 tokens, 64 x 90 float32 in 4 shards:
// 14 us, with the kernels for a handful of tokens 24).  Every workgroup reads w once for its logits and once more for dx, from L2, which is why w has to be small.  A launch of few tokens has
// several workgroups for the same ones: each makes all their logits, and a part of dx's columns and of dw.
// Code is kept short for the same reason: each instruction is fetched once and used a few times (with loops of their own for whole fragments, and two tokens a wave, the kernel was 36 KB;
// 106 tokens, 90 x 217 in 4 shards, losses alone, 16 us, so 9).
// Fragments go from global memory straight to matrix instructions, at any element alignment.  An operand whose sum runs along its rows is loaded along them; of one whose sum runs across them a
// lane loads four neighbouring columns of each of its rows, which are its fragments of four tiles (whose columns are then 4 n + tile).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernels_basic.h"
#include "kernels_few.h"
#include "kernels_softmax.h"
#include "mfma_common.h"
#include "tile_index.h"

namespace gspmd {

constexpr int kSmallShards = 16, kSmallTargets = 128, kSmallTokens = 16, kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64;
constexpr int kSmallColumns = 1280;               // of a row of logits: what there is room for
struct SmallLoss {
  SoftmaxRows rows;              // z: where D goes for the product that makes dw (null: not wanted); x_copies: with D in two parts both copies of x, else one (null: not wanted)
  const void* w[kSmallShards];   // the vocabulary's shards
  void* dw[kSmallShards];        // null: not wanted here
  const void* x[kSmallShards];   // the tokens' shards
  void* dx[kSmallShards];        // null: not wanted
  int64_t ldw, lddw, lddx;
  int32_t M, shards;             // shards of the vocabulary, those without an entry too
  int32_t token_shards;
  int32_t lost;                  // D in two parts
};
static_assert(sizeof(SmallLoss) <= 4096, "kernel arguments");

template <typename T> constexpr int small_vec() { return 16 / static_cast<int>(sizeof(T)); }       // of a sum's terms in a lane's fragment
template <typename T> using small_four = T __attribute__((ext_vector_type(4), aligned(sizeof(T))));

// c += the product of two fragments: a bfloat16 instruction, or four float32 ones.
template <typename T>
__device__ __forceinline__ void small_multiply(float4_t& c, few_raw<T> a, few_raw<T> b) {
  if constexpr (sizeof(T) == 2) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  }
}
// Terms k and following of a sum along a row of `len` elements (at least as many as a fragment has): zeros beyond it.  What a row has left is loaded with what is before it and moved down.
template <typename T>
__device__ __forceinline__ few_raw<T> small_along(GSPMD_GLOBAL const T* row, int k, int len) {
  constexpr int V = small_vec<T>();
  const int at = min(k, len - V);
  few_raw<T> v = *(GSPMD_GLOBAL const few_raw<T>*)(row + at);
  if (k > at) {
    typedef uint64_t u64x2_t __attribute__((ext_vector_type(2)));
    u64x2_t b = __builtin_bit_cast(u64x2_t, v);
    const int shift = (k - at) * 8 * static_cast<int>(sizeof(T));
    if (shift >= 64) b = u64x2_t{shift >= 128 ? 0 : b[1] >> (shift & 63), 0};
    else b = u64x2_t{b[0] >> shift | b[1] << (64 - shift), b[1] >> shift};
    v = __builtin_bit_cast(few_raw<T>, b);
  }
  return v;
}
// The first n of a fragment's terms (any n), zeros for the others.
template <typename T>
__device__ __forceinline__ few_raw<T> small_keep(few_raw<T> v, int n) {
#pragma unroll
  for (int e = 0; e < small_vec<T>(); ++e)
    if (e >= n) v[e] = 0;
  return v;
}
// float32 values as an operand: rounded, and (bfloat16) what that loses.
template <typename T>
__device__ __forceinline__ void small_operand(const float (&f)[small_vec<T>()], few_raw<T>& rounded, few_raw<T>& lost) {
#pragma unroll
  for (int i = 0; i < small_vec<T>(); ++i) {
    if constexpr (sizeof(T) == 2) {
      const __bf16 r = static_cast<__bf16>(f[i]);
      rounded[i] = __builtin_bit_cast(bf16_bits, r);
      lost[i] = __builtin_bit_cast(bf16_bits, static_cast<__bf16>(f[i] - static_cast<float>(r)));
    } else {
      rounded[i] = f[i];
      lost[i] = 0.f;
    }
  }
}
template <typename T>
__device__ __forceinline__ T small_round(float v) {
  if constexpr (sizeof(T) == 2) return __builtin_bit_cast(bf16_bits, static_cast<__bf16>(v));
  else return v;
}

// ORDER: vocab_dim (0: w [V, M], 1: [M, V]).  DW: dw is made here, of 16 tokens in all, by the workgroups of the first 16 rows.
template <typename T, int ORDER, bool DW>
__global__ __launch_bounds__(kSmallThreads) void small_loss_kernel(const SmallLoss args) {
  constexpr int V = small_vec<T>(), kStep = 4 * V, kWaves = kSmallWaves;        // terms of a sum that an instruction (four, in float32) takes
  constexpr int kPartCols = 64 * kWaves;                                        // logits in parts: columns of all of them
  constexpr int kPartLd = 68, COLS = kSmallColumns;
  constexpr int kLogits = COLS > kPartCols ? kSmallTokens * (COLS + 4) : kSmallTokens * (kPartCols + 4 * kWaves);
  __shared__ __attribute__((aligned(16))) float logits[kLogits];                // [part][token][ld]
  __shared__ __attribute__((aligned(16))) float part[kWaves * kSmallTokens * kPartLd];
  const GSPMD_KERNARG SmallLoss& a = *first_kernel_argument<SmallLoss>();
  const GSPMD_KERNARG SoftmaxRows& r = a.rows;
  const int t0 = threadIdx.x, lane = t0 & 63, wave = __builtin_amdgcn_readfirstlane(t0 >> 6), n16 = lane & 15, quad = lane >> 4;
  const int first = blockIdx.x * kSmallTokens, slice = blockIdx.y, slices = gridDim.y, M = a.M, cols = r.cols, K = r.targets;
  const int groups = (cols + 63) >> 6, ld = groups * 64 + 4;
  auto x_row = [&](int token) {                 // (of no token: another's)
    token = min(token, r.tokens - 1);
    const int i = token / r.per_shard;
    return (GSPMD_GLOBAL const T*)a.x[i] + static_cast<int64_t>(token - i * r.per_shard) * r.ldx;
  };
  const FastDiv by_cols{r.by_cols.mul, r.by_cols.shift};
  // a column's shard, place in it, and entries from there on (none: at most 0)
  struct Place { int j, at, valid, stored; };
  auto place = [&](int col) {
    const int j = static_cast<int>(div_by(static_cast<uint32_t>(col), by_cols)), at = col - j * r.per_cols;
    return Place{j, at, min(r.per, r.vocab - j * r.per) - at, r.per - at};
  };

  // Waves and workgroups begin a sum at places of their own: at one place in rows a power of two apart they would all read from a few of L2's channels at a time.
  auto turned = [&](int it, int its, int begin, int step) {
    const int from = it + (wave + blockIdx.x * 3) % its;
    return begin + (from >= its ? from - its : from) * step;
  };
  // Four neighbouring columns of one shard from `col` on, moved back to end with the shard's static part (what lies there beyond its entries may be anything).
  struct Four { int j, at, col, others; bool there; };
  auto four_of = [&](int col) {
    const Place p = place(col);
    const bool there = p.j < a.shards && p.valid > 0;
    const FourColumns four = four_columns(p.at, r.per);
    const int j = there ? p.j : 0;
    return Four{j, there ? four.at : 0, j * r.per_cols + four.at, four.others, there};
  };
  typedef float any_float4 __attribute__((ext_vector_type(4), aligned(4)));

  // ---- this wave's token's targets, two a lane: on their way first
  const int g = first + wave, token_shard = g / r.per_shard, token = g - token_shard * r.per_shard;
  const bool has_token = g < r.tokens;
  const GSPMD_KERNARG TokenShard& s = r.shard[has_token ? token_shard : 0];
  float q[2];
  int id[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int k = n * 64 + lane;
    id[n] = -1;
    q[n] = -INFINITY;
    if (has_token && k < K) {
      const int64_t at = static_cast<int64_t>(token) * K + k;
      const int here = ((GSPMD_GLOBAL const int32_t*)s.ids)[at];
      q[n] = teachers_logit(s, r.logits_bf16, at);
      if (here >= 0 && here < r.vocab) id[n] = here;
      else q[n] = -INFINITY;
    }
  }

  // ---- logits: groups of 64 columns; fewer groups than waves: several waves share a group's sum, whose parts meet in LDS
  int splits = 1;
  while (splits * 2 * groups <= kWaves && splits * 2 * kStep <= M) splits *= 2;
  {
    const int each = ((M + splits - 1) / splits + kStep - 1) / kStep * kStep;
    GSPMD_GLOBAL const T* const x = x_row(first + n16);
    for (int item = wave; item < groups * splits; item += kWaves) {
      const int split = item / groups, group = item - split * groups, begin = split * each, end = min(begin + each, M);
      const Four four = four_of(group * 64 + 4 * n16);
      float4_t acc[4] = {};
      constexpr int U = 2;
      const int its = (end - begin + U * kStep - 1) / (U * kStep);
      if constexpr (ORDER == 0) {
        GSPMD_GLOBAL const T* w[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const Place p = place(group * 64 + c * 16 + n16);
          w[c] = (GSPMD_GLOBAL const T*)a.w[p.valid > 0 ? p.j : 0] + (p.valid > 0 ? p.at * a.ldw : 0);
        }
#pragma unroll 1
        for (int it = 0; it < its; ++it) {
          const int k0 = turned(it, its, begin, U * kStep);
          few_raw<T> fa[U], fb[U][4];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int k = k0 + u * kStep + quad * V, here = k0 + u * kStep < end ? k : M + V;
            fa[u] = small_along<T>(x, here, M);
#pragma unroll
            for (int c = 0; c < 4; ++c) fb[u][c] = small_along<T>(w[c], here, M);
          }
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < 4; ++c) small_multiply<T>(acc[c], fa[u], fb[u][c]);
        }
      } else {
        GSPMD_GLOBAL const T* const w = (GSPMD_GLOBAL const T*)a.w[four.j] + four.at;
#pragma unroll 1
        for (int it = 0; it < its; ++it) {
          const int k0 = turned(it, its, begin, U * kStep);
          few_raw<T> fa[U];
          small_four<T> raw[U][V];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int k = k0 + u * kStep + quad * V, here = k0 + u * kStep < end ? k : M + V;
            fa[u] = small_along<T>(x, here, M);
#pragma unroll
            for (int i = 0; i < V; ++i) {
              raw[u][i] = *(GSPMD_GLOBAL const small_four<T>*)(w + min(here + i, M - 1) * a.ldw);
              if (here + i >= M) raw[u][i] = 0;
            }
          }
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              few_raw<T> fb;
#pragma unroll
              for (int i = 0; i < V; ++i) fb[i] = raw[u][i][c];
              small_multiply<T>(acc[c], fa[u], fb);
            }
        }
      }
      float* const out = logits + (split * kSmallTokens + quad * 4) * ld + group * 64;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (ORDER == 0) {
#pragma unroll
          for (int c = 0; c < 4; ++c) out[i * ld + c * 16 + n16] = acc[c][i];
        } else {
          // (without those of another lane, whose wave may have begun the sum elsewhere and round otherwise: with two writers the bits would be those of the later one)
          float* const to = logits + (split * kSmallTokens + quad * 4 + i) * ld + four.col;
          if (four.there && four.others == 0) {
            *reinterpret_cast<any_float4*>(to) = float4_t{acc[0][i], acc[1][i], acc[2][i], acc[3][i]};
          } else if (four.there) {
#pragma unroll
            for (int e = 1; e < 4; ++e)
              if (e >= four.others) to[e] = acc[e][i];
          }
        }
      }
    }
  }
  __syncthreads();

  // ---- the softmax and D: a wave's token
  const bool has_grad = a.dx[0] != nullptr || DW || r.z != nullptr;
  const float inv_tau = r.inv_tau, c = inv_tau * kLog2e;
  float* const z = logits + wave * ld;
  if (!has_token) {                             // padding of the last shards, or none of theirs
    if (has_grad)
      for (int col = lane; col < groups * 64; col += 64) z[col] = 0.f;
    if (lane == 0 && slice == 0 && g < a.token_shards * r.per_shard) {
      r.shard[token_shard].loss[token] = 0.f;
      if (r.shard[token_shard].lse) r.shard[token_shard].lse[token] = 0.f;
    }
  } else {
    float m = -INFINITY;
#pragma unroll 1
    for (int col = lane; col < groups * 64; col += 64) {
      float v = z[col];
#pragma unroll 4
      for (int p = 1; p < splits; ++p) v += z[p * kSmallTokens * ld + col];
      if (place(col).valid <= 0) v = -INFINITY;
      z[col] = v;
      m = fmaxf(m, v);
    }
    m = over_wave(m, [](float x, float y) { return fmaxf(x, y); });
    const float finite_m = m == -INFINITY ? 0.f : m;
    float total = 0.f;
#pragma unroll 1
    for (int col = lane; col < groups * 64; col += 64) total += __builtin_amdgcn_exp2f((z[col] - finite_m) * c);
    total = over_wave(total, [](float x, float y) { return x + y; });
    const float u_most = m * inv_tau, log_total = logf(total);
    staged_in_order();                          // (the row is this wave's own)
    float u[2], p[2] = {0.f, 0.f};
    int column[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int j = id[n] / r.per;
      column[n] = id[n] >= 0 ? j * r.per_cols + (id[n] - j * r.per) : -1;
      u[n] = column[n] >= 0 ? z[column[n]] * inv_tau : 0.f;
    }
    const TargetSums of = over_targets(K, inv_tau, [&](int k) { return k < 64 ? q[0] : q[1]; }, [&](int k) { return k < 64 ? u[0] : u[1]; }, [&](int k, float share) { (k < 64 ? p[0] : p[1]) = share; });
    if (lane == 0 && slice == 0) {
      s.loss[token] = of.any ? of.sum + u_most + log_total : 0.f;
      if (s.lse) s.lse[token] = u_most + log_total;
    }
    if (has_grad) {
      const float weight = s.weights ? s.weights[token] : 1.f, scale = of.any ? weight * inv_tau : 0.f, factor = scale / total;
      // a target given twice: its shares are added in the targets' order by each of them
      float* const shares = part + wave * 2 * kSmallTargets;
      int32_t* const ids = reinterpret_cast<int32_t*>(shares + kSmallTargets);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        shares[n * 64 + lane] = p[n];
        ids[n * 64 + lane] = id[n];
      }
      staged_in_order();
      float share[2] = {0.f, 0.f};
#pragma unroll 1
      for (int k = 0; k < K; ++k) {
        const int here = ids[k];
        const float of_it = shares[k];
#pragma unroll
        for (int n = 0; n < 2; ++n) share[n] += here == id[n] ? of_it : 0.f;
      }
#pragma unroll 1
      for (int col = lane; col < groups * 64; col += 64) z[col] = scale == 0.f ? 0.f : __builtin_amdgcn_exp2f((z[col] - finite_m) * c) * factor;
      staged_in_order();
#pragma unroll
      for (int n = 0; n < 2; ++n)
        if (scale != 0.f && column[n] >= 0) z[column[n]] = scale * (__builtin_amdgcn_exp2f(((u[n] - u_most) - log_total) * kLog2e) - share[n]);
      staged_in_order();
      if (r.z != nullptr && slice == 0) {       // for the product that makes dw
        GSPMD_GLOBAL T* const d = (GSPMD_GLOBAL T*)reinterpret_cast<T*>(r.z + g * r.ldz);
        GSPMD_GLOBAL T* const d_lost = (GSPMD_GLOBAL T*)reinterpret_cast<T*>(r.z + (r.lost + g) * r.ldz);
#pragma unroll 1
        for (int col = lane; col < cols; col += 64) {
          const float v = z[col];
          const T rounded = small_round<T>(v);
          d[col] = rounded;
          if constexpr (sizeof(T) == 2)
            if (a.lost) d_lost[col] = small_round<T>(v - bf16_to_float(rounded));
        }
        if (r.x_copies != nullptr) {
          GSPMD_GLOBAL const T* const x = x_row(g);
          GSPMD_GLOBAL T* const to = (GSPMD_GLOBAL T*)reinterpret_cast<T*>(r.x_copies) + g * r.ld_copy;
#pragma unroll 1
          for (int e = lane; e < M; e += 64) {
            const T v = x[e];
            to[e] = v;
            if (a.lost) to[r.lost * r.ld_copy + e] = v;
          }
        }
      }
    }
  }
  if (a.dx[0] == nullptr && !DW) return;
  __syncthreads();

  auto m_of = [&](int group) { return min(group * 64 + 4 * n16, M - 4); };       // the first of a lane's four of M

  const int across = (M + 63) >> 6, mine_first = across * slice / slices, mine_end = a.dx[0] != nullptr ? across * (slice + 1) / slices : mine_first;       // groups of 64 of M

  // ---- dw, of 16 tokens in all: one instruction's sum (bfloat16: D in two parts, each times x).  Made by waves that have nothing of dx's sums, or before these are joined.
  constexpr int kTokensOf = sizeof(T) == 2 ? 1 : 3;       // a lane's V terms are tokens (quad & this) * V and following
  const int t_of = (quad & kTokensOf) * V;
  const bool second = sizeof(T) == 2 && quad >= 2;        // the part that D's rounding lost
  const int stored_cols = a.shards * r.per_cols;          // shards without an entry get zeros
  // rows of the result: entries ([V, M]) or M; columns in fours
  const int tiles = ORDER == 0 ? (stored_cols + 15) / 16 : (M + 15) / 16, fours = ORDER == 0 ? across : (stored_cols + 63) / 64;
  // A unit: one group of 64 columns and every `step`-th tile of rows, from the waves on that have none of dx's sums first.
  auto make_dw = [&](int busy) {
    const int units = slices * kWaves, unit = slice * kWaves + ((wave - busy) & (kWaves - 1));
    const int step = max(1, units / fours);
#pragma unroll 1
    for (int n = unit; n < fours * step; n += units) {
      const int four = n % fours, phase = n / fours;
      const int col = four * 64 + 4 * n16, m0 = m_of(four);
      const Place here = place(col);              // [M, V]: four columns of one shard, moved back as in four_of
      const int back = max(here.at - (r.per - 4), 0), entries = here.valid + back, col0 = col - back;
      few_raw<T> fb[4];
      if constexpr (ORDER == 0) {
        small_four<T> raw[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          raw[i] = *(GSPMD_GLOBAL const small_four<T>*)(x_row(t_of + i) + m0);
          if (t_of + i >= r.tokens) raw[i] = 0;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < V; ++i) fb[e][i] = raw[i][e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float d[V];
#pragma unroll
          for (int i = 0; i < V; ++i) d[i] = entries > 0 ? logits[(t_of + i) * ld + col0 + e] : 0.f;
          few_raw<T> hi, lo;
          small_operand<T>(d, hi, lo);
          fb[e] = second ? lo : hi;
        }
      }
#pragma unroll 1
      for (int tile = phase; tile < tiles; tile += step) {
        few_raw<T> fa;
        if constexpr (ORDER == 0) {
          const int entry = min(tile * 16 + n16, groups * 64 - 1);
          float d[V];
#pragma unroll
          for (int i = 0; i < V; ++i) d[i] = logits[(t_of + i) * ld + entry];
          few_raw<T> hi, lo;
          small_operand<T>(d, hi, lo);
          fa = second ? lo : hi;
        } else {
          const int m = min(tile * 16 + n16, M - 1);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            fa[i] = x_row(t_of + i)[m];
            if (t_of + i >= r.tokens) fa[i] = 0;
          }
        }
        float4_t acc[4] = {};
#pragma unroll
        for (int e = 0; e < 4; ++e) small_multiply<T>(acc[e], fa, fb[e]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = tile * 16 + quad * 4 + i;
          small_four<T> out;
#pragma unroll
          for (int e = 0; e < 4; ++e) out[e] = small_round<T>(acc[e][i]);
          if constexpr (ORDER == 0) {
            const Place p = place(row);
            if (p.valid <= 0) out = 0;
            if (row < stored_cols && p.stored > 0) *(GSPMD_GLOBAL small_four<T>*)((GSPMD_GLOBAL T*)a.dw[p.j] + p.at * a.lddw + m0) = out;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e >= entries) out[e] = 0;
            if (row < M && col < stored_cols) *(GSPMD_GLOBAL small_four<T>*)((GSPMD_GLOBAL T*)a.dw[here.j] + row * a.lddw + here.at - back) = out;
          }
        }
      }
    }
  };

  // ---- dx: sums over the columns, whose D is in LDS.  A round of the waves takes `at_once` groups of 64 of M, several waves sharing one's sum; their parts meet in LDS.
  int shares = 1;
  while (shares * 2 * max(mine_end - mine_first, 1) <= kWaves && shares * 2 * kStep <= groups * 64) shares *= 2;
  const int at_once = kWaves / shares, each = (groups * 64 / shares + kStep - 1) / kStep * kStep;
  bool dw_left = DW && blockIdx.x == 0;         // (others have padding rows of the shards only: 16 tokens in 3 shards are 18 rows)
  for (int from = mine_first; from < mine_end || dw_left; from += at_once) {
    const int share = wave / at_once, group = from + wave - share * at_once, begin = share * each, end = min(begin + each, groups * 64);
    float4_t acc[4] = {};
    if (group < mine_end) {
      constexpr int U = DW && sizeof(T) == 2 && ORDER == 1 ? 1 : 2;       // (with 2 there, three registers spill)
      const int its = (end - begin + U * kStep - 1) / (U * kStep);
#pragma unroll 1
      for (int it = 0; it < its; ++it) {
        const int k0 = turned(it, its, begin, U * kStep);
        few_raw<T> fb[U][4];
        small_four<T> raw[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int k = k0 + u * kStep + quad * V;
          const Place p = place(k);           // (V columns of one shard)
          const int valid = k0 + u * kStep < end ? p.valid : 0;
          GSPMD_GLOBAL const T* const w = (GSPMD_GLOBAL const T*)a.w[valid > 0 ? p.j : 0];
          if constexpr (ORDER == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) raw[u][i] = *(GSPMD_GLOBAL const small_four<T>*)(w + (i < valid ? p.at + i : 0) * a.ldw + m_of(group));       // (times a D of 0)
          } else {
#pragma unroll
            for (int n = 0; n < 4; ++n) fb[u][n] = small_keep<T>(small_along<T>(w + min(group * 64 + n * 16 + n16, M - 1) * a.ldw, valid > 0 ? p.at : 0, r.per), valid);
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (k0 + u * kStep >= end) break;
          float d[V];
#pragma unroll
          for (int i = 0; i < V; i += 4) {
            const float4_t four = *reinterpret_cast<const float4_t*>(logits + n16 * ld + k0 + u * kStep + quad * V + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) d[i + e] = four[e];
          }
          few_raw<T> hi, lo;
          small_operand<T>(d, hi, lo);
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            few_raw<T> b;
            if constexpr (ORDER == 0) {
#pragma unroll
              for (int i = 0; i < V; ++i) b[i] = raw[u][i][n];
            } else {
              b = fb[u][n];
            }
            small_multiply<T>(acc[n], hi, b);
            if constexpr (sizeof(T) == 2) small_multiply<T>(acc[n], lo, b);
          }
        }
      }
      float* const out = part + (wave * kSmallTokens + quad * 4) * kPartLd + 4;       // (a lane's four may be moved back to before the group)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (ORDER == 0) {
          *reinterpret_cast<any_float4*>(out + i * kPartLd + m_of(group) - group * 64) = float4_t{acc[0][i], acc[1][i], acc[2][i], acc[3][i]};
        } else {
#pragma unroll
          for (int n = 0; n < 4; ++n) out[i * kPartLd + n * 16 + n16] = acc[n][i];
        }
      }
    }
    if constexpr (DW) {
      if (dw_left) make_dw(min(mine_end - from, at_once) * shares & (kWaves - 1));
      dw_left = false;
      if (from >= mine_end) break;              // (dw alone)
    }
    __syncthreads();
    for (int n = t0; n < at_once * kSmallTokens * 64; n += kSmallThreads) {
      const int which = n >> 10, tl = (n >> 6) & 15, m = (from + which) * 64 + (n & 63), g = first + tl;
      if (from + which >= mine_end || m >= M || g >= a.token_shards * r.per_shard) continue;
      float sum = 0.f;
#pragma unroll 4
      for (int p = 0; p < shares; ++p) sum += part[((p * at_once + which) * kSmallTokens + tl) * kPartLd + 4 + (n & 63)];
      const int i = g / r.per_shard;
      ((GSPMD_GLOBAL T*)a.dx[i])[static_cast<int64_t>(g - i * r.per_shard) * a.lddx + m] = small_round<T>(g < r.tokens ? sum : 0.f);
    }
    __syncthreads();
  }
}

}  // namespace gspmd
