// The choice of experts and the exchange of rows with them (gspmd_route, gspmd_dispatch, gspmd_combine and their gradients).
//
// Routing: sixteen lanes have a token, each R neighbouring experts in registers.  The largest logit is found k times over: every lane's own, a maximum over the sixteen by rotations
// within their row of the wave, and of those that have it the lowest lane, whose experts are the lowest.  It is bound by those instructions, some 20 + 3 R a choice, not by the logits (16384 tokens of 128 experts, 8 chosen: 8.4 us,
// of which the 8.4 MB would take 2).  Logits are compared as whole numbers: a maximum of floats is two instructions where a NaN may be about.
// Exchange: bound by memory, rows copied or added up 16 bytes a lane.  Every row has one writer (or two with the same bits, kernels_rows.h); a token's rows are added in the order of its choices.
// 8192 tokens of 4096, 4 choices: combine_kernel 79 us (336 MB, 4.2 TB/s), combine_grad_kernel 109 (604 MB, 5.5 TB/s); 2048 of 2048, 2 choices: dispatch_kernel 10.0,
// combine_kernel 6.1.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels_basic.h"
#include "kernels_embed.h"
#include "kernels_rows.h"
#include "mfma_common.h"
#include "order.h"
#include "ragged.h"

namespace gspmd {

constexpr int kRouteLanes = 16, kMostExperts = GSPMD_MAX_EXPERTS, kMostChoices = GSPMD_MAX_CHOICES;
static_assert(kMostChoices <= kRouteLanes, "a lane for every choice");

struct RouteSizes {
  int32_t T, ts, shards, E, k, ld, ld_d;
  int32_t normalise;
  int32_t* experts;                // [T][k]
  float* weights;                  // [T][k]
  const float* dweights;           // the gradient's
};
struct RouteShard {
  const void* logits;
  void* dlogits;                   // null: none to be written
};
template <int SHARDS>
struct RouteArgsOf : RouteSizes {  // (the first of a kernel's arguments: shards are read there)
  RouteShard shard[SHARDS];
};
typedef RouteArgsOf<kTokenShards> RouteArgs;

// v combined over the sixteen lanes of a row, in all of them.  (Rotations: every lane adds in another order, but of max and of the two-by-two sums the bits are the same.)
template <typename Op>
__device__ __forceinline__ float over_row(float v, Op op) {
  auto turned = [](float x, auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true)); };
  v = op(v, turned(v, std::integral_constant<int, 0x128>{}));      // row_ror:8
  v = op(v, turned(v, std::integral_constant<int, 0x124>{}));
  v = op(v, turned(v, std::integral_constant<int, 0x122>{}));
  return op(v, turned(v, std::integral_constant<int, 0x121>{}));
}
__device__ __forceinline__ float row_max(float v) { return over_row(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float row_sum(float v) { return over_row(v, [](float a, float b) { return a + b; }); }
// of those lanes of this one's row of sixteen that say yes, a mask
__device__ __forceinline__ uint32_t row_ballot(bool yes, int lane) { return static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(yes) >> (lane & 48)) & 0xffffu; }

// This lane's experts' logits, -infinity where there are none; NaN as -infinity, and whether there was one among the token's.
template <typename T, int R>
__device__ __forceinline__ bool route_load(const T* z, int E, int of_row, int lane, float (&v)[R]) {
  bool strange = false;
  constexpr int n = Sixteen<T>::n;
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = -INFINITY;
  if (z != nullptr && (of_row + 1) * R <= E) {
    const T* const from = z + of_row * R;
    if constexpr (R % n == 0) {
      u32x4_t w[R / n];
#pragma unroll
      for (int i = 0; i < R / n; ++i) w[i] = load16(from + i * n);
#pragma unroll
      for (int i = 0; i < R / n; ++i) {
        float f[n];
        Sixteen<T>::open(w[i], f);
#pragma unroll
        for (int e = 0; e < n; ++e) v[i * n + e] = f[e];
      }
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r) v[r] = load_as_float<T>(from + r);
    }
  } else if (z != nullptr && of_row * R < E) {
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = load_as_float<T>(z + min(of_row * R + r, E - 1));      // (no branch: a load under one is waited for there)
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (of_row * R + r >= E) v[r] = -INFINITY;
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (v[r] != v[r]) {
      strange = true;
      v[r] = -INFINITY;
    }
  return row_ballot(strange, lane) != 0;
}

// The sum of exp(logit - most) over a token's experts; NaN where a logit is.
template <int R>
__device__ __forceinline__ float route_total(const float (&v)[R], float most, bool strange) {
  float sum = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) sum += expf(v[r] - most);
  sum = row_sum(sum);
  return strange ? NAN : sum;
}

// Logits as whole numbers in the same order (a zero has one sign; -infinity, which is never chosen, the lowest of all), and back: the same steps.
constexpr int32_t kNoLogit = INT32_MIN;
__device__ __forceinline__ int32_t order_of_logit(float f) {
  const int32_t i = __float_as_int(f + 0.f);
  return f == -INFINITY ? kNoLogit : i ^ ((i >> 31) & INT32_MAX);
}
__device__ __forceinline__ float logit_of_order(int32_t i) { return i == kNoLogit ? -INFINITY : __int_as_float(i ^ ((i >> 31) & INT32_MAX)); }
__device__ __forceinline__ int32_t row_most(int32_t v) {
  auto turned = [](int32_t x, auto ctrl) { return __builtin_amdgcn_update_dpp(0, x, decltype(ctrl)::value, 0xf, 0xf, true); };
  v = max(v, turned(v, std::integral_constant<int, 0x128>{}));      // row_ror:8
  v = max(v, turned(v, std::integral_constant<int, 0x124>{}));
  v = max(v, turned(v, std::integral_constant<int, 0x122>{}));
  return max(v, turned(v, std::integral_constant<int, 0x121>{}));
}

// The sixteen lanes' choices: lane i of them has the i-th, its expert (-1: none) and weight.  `chosen`: LDS, a word for each lane of the wave.
template <typename T, int R, typename A>
__device__ __forceinline__ void route_choose(const A& a, int token, int lane, int32_t* chosen, int* chosen_expert, float* weight) {
  const int of_row = lane & 15;
  const T* z = nullptr;
  if (token < a.T) {
    const int shard = embed_shard(token, a.ts, a.shards);
    z = static_cast<const T*>(a.shards == 1 ? a.shard[0].logits : first_kernel_argument<A>()->shard[shard].logits) + static_cast<int64_t>(token - shard * a.ts) * a.ld;
  }
  float v[R];
  const bool strange = route_load<T, R>(z, a.E, of_row, lane, v);
  int32_t order[R];
#pragma unroll
  for (int r = 0; r < R; ++r) order[r] = order_of_logit(v[r]);
  auto lanes_most = [&] {
    int32_t best = order[0];
#pragma unroll
    for (int r = 1; r < R; ++r) best = max(best, order[r]);
    return best;
  };
  chosen[lane] = -1;
  staged_in_order();
  int32_t best = lanes_most(), here = row_most(best), mine = kNoLogit;
  const float most = logit_of_order(here);
  float total = a.normalise ? 0.f : route_total<R>(v, most, strange);
  for (int i = 0;;) {
    // the lowest lane of each row of sixteen that has the largest (one has), and the lowest of its experts that do
    const uint64_t having = __builtin_amdgcn_ballot_w64(best == here), lowest = having & ~(having - 0x0001000100010001ull);
    bool looking = ((lowest >> lane) & 1) != 0 && here != kNoLogit;
    const bool winner = looking;
    int at = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool it = looking && order[r] == here;
      looking = looking && !it;
      order[r] = it ? kNoLogit : order[r];
      at = it ? r : at;
    }
    if (winner) chosen[(lane & 48) + i] = of_row * R + at;
    mine = of_row == i ? here : mine;
    if (++i == a.k) break;
    best = lanes_most();
    here = row_most(best);
  }
  staged_in_order();
  const int expert = chosen[lane];
  const float share = expert >= 0 ? expf(logit_of_order(mine) - most) : 0.f;
  if (a.normalise) total = row_sum(share);
  *chosen_expert = expert;
  *weight = expert >= 0 ? share / total : 0.f;
}

// The choices of sixty-four tokens, and how many of them each expert has: counts [tile][E].  (With them a routing takes two launches; ordering the choices as order_kernel does takes three.)
constexpr int kFewRouted = kOrderThreads / kRouteLanes, kTileTokens = kFewRouted;
template <typename T, int R, typename A>
__global__ __launch_bounds__(kOrderThreads) void route_kernel(const A a, int32_t* counts) {
  __shared__ int32_t here[kMostExperts], chosen[kOrderThreads];
  const int t = threadIdx.x, lane = t & 63, of_row = lane & 15, token = blockIdx.x * kTileTokens + t / kRouteLanes;
  if (t < a.E) here[t] = 0;
  int expert;
  float weight;
  route_choose<T, R>(a, token, lane, chosen + (t & ~63), &expert, &weight);
  __syncthreads();
  if (token < a.T && of_row < a.k) {
    a.experts[static_cast<int64_t>(token) * a.k + of_row] = expert;
    a.weights[static_cast<int64_t>(token) * a.k + of_row] = weight;
    if (expert >= 0) atomicAdd(&here[expert], 1);
  }
  __syncthreads();
  if (t < a.E) counts[static_cast<int64_t>(blockIdx.x) * a.E + t] = here[t];
}
static_assert(kMostExperts <= kOrderThreads, "a thread for every expert");

// Where a tile's choices begin, of every expert: the choices of lower experts, and those of its own in earlier tiles.  With few tiles a workgroup adds them up itself (route_places_kernel); with many, one
// for every expert turns the tiles' counts into sums of the earlier ones, and its total.  What the first reads grows with the square of the tiles, the second is a launch more (the whole routing, us, first /
// second; tokens x experts, choices: 8192 x 64, 2 9.2 / 11.4; 16384 x 16, 2 8.9 / 11.7, x 128, 8 14.6 / 15.2, x 256, 2 16.3 / 15.6, x 512, 2 27.8 / 25.1; 32768 x 8, 2 9.6 / 11.2, x 64, 2 13.7 / 13.2, x 128, 8
// 23.9 / 21.0, x 256, 2 29.1 / 21.7; 65536 x 8, 2 16.3 / 16.1, x 64, 2 27.5 / 20.6).  512 tiles, of 64 tokens, are where they cross with 64 experts; with more of them it is earlier, which the rule does not follow.
constexpr int kTilesSummed = 512;
__global__ __launch_bounds__(kOrderThreads) static void route_sums_kernel(int32_t* counts, int tiles, int E, int32_t* totals) {
  __shared__ uint32_t sums[kOrderWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, e = blockIdx.x;
  int before = 0;
  for (int base = 0; base < tiles; base += kOrderThreads) {
    int32_t* const at = counts + static_cast<int64_t>(base + t) * E + e;
    const int n = base + t < tiles ? *at : 0, to_here = wave_sum_to_here(n);
    if (lane == 63) sums[wave] = static_cast<uint32_t>(to_here);
    __syncthreads();
    int sum = before + to_here - n;
    for (int w = 0; w < kOrderWaves; ++w) {
      if (w < wave) sum += static_cast<int>(sums[w]);
      before += static_cast<int>(sums[w]);
    }
    if (base + t < tiles) *at = sum;
    __syncthreads();
  }
  if (t == 0) totals[e] = before;
}

// The places of up to a workgroup's 1024 keys, each below 1 << bits, among them, those of equal keys in the order of the threads: lanes with equal keys are found by a ballot for each bit, and
// sums over [keys][waves] are places.  `counts`: LDS, [1 << bits][waves]; returns with where each key's run begins in counts[key][0].
__device__ __forceinline__ int place_of_mine(uint32_t key, int bits, uint16_t* counts, uint32_t* sums) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, entries = kOrderWaves << bits;
  for (int i = t; i < entries / 2; i += kOrderThreads) reinterpret_cast<uint32_t*>(counts)[i] = 0;
  __syncthreads();
  uint64_t same = ~uint64_t(0);
  for (int b = 0; b < bits; ++b) {
    const bool on = (key >> b) & 1;
    const uint64_t with = __builtin_amdgcn_ballot_w64(on);
    same &= on ? with : ~with;
  }
  const int rank = __builtin_popcountll(same & ((uint64_t(1) << lane) - 1));
  uint16_t* const mine = counts + key * kOrderWaves + wave;
  if (rank == 0) *mine = static_cast<uint16_t>(__builtin_popcountll(same));
  __syncthreads();
  const int each = (entries + kOrderThreads - 1) / kOrderThreads, first = t * each;
  int sum = 0;
  for (int i = 0; i < each; ++i) sum += first + i < entries ? counts[first + i] : 0;
  const int to_here = wave_sum_to_here(sum);
  if (lane == 63) sums[wave] = static_cast<uint32_t>(to_here);
  __syncthreads();
  int at = to_here - sum;
  for (int w = 0; w < wave; ++w) at += static_cast<int>(sums[w]);
  for (int i = 0; i < each; ++i)
    if (first + i < entries) {
      const int n = counts[first + i];
      counts[first + i] = static_cast<uint16_t>(at);
      at += n;
    }
  __syncthreads();
  return rank + *mine;
}

// Slots of a tile's choices, a choice a thread.  Bound by waits: 256 tiles' counts of 128 experts come in four rounds (7.4 us).  `totals`: null where counts are the tiles' own (kTilesSummed).
__global__ __launch_bounds__(kOrderThreads) static void route_places_kernel(const int32_t* experts, const int32_t* counts, const int32_t* totals, int n, int each, int E, int tiles, int bits, int32_t* slots,
                                                                         int32_t* order, int32_t* sizes) {
  __shared__ uint16_t of_tile[kOrderWaves << kMostRange];
  __shared__ uint32_t sums[kOrderWaves];
  __shared__ int32_t begins[kMostExperts], parts[2][kOrderThreads];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, tile = blockIdx.x, at = tile * each + t;
  const bool mine = t < each && at < n;
  const int expert = mine ? experts[at] : -1;
  const uint32_t key = mine ? static_cast<uint32_t>(min(static_cast<uint32_t>(expert), static_cast<uint32_t>(E))) : (1u << bits) - 1;
  // of expert t % E: choices of all tiles and of the earlier ones, a share of the tiles a thread
  int total = 0, earlier = 0;
  const int shares = min(kOrderThreads / E, 32);
  if (totals == nullptr) {
    const int share = t / E, e = t - share * E;
    if (share < shares) {
      const int per = (tiles + shares - 1) / shares, first = share * per, end = min(first + per, tiles);
      GSPMD_GLOBAL const int32_t* from = (GSPMD_GLOBAL const int32_t*)counts + static_cast<int64_t>(first) * E + e;
      int i = first;
      for (; i + 8 <= end; i += 8, from += 8 * static_cast<int64_t>(E)) {
        int32_t v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = from[u * static_cast<int64_t>(E)];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          total += v[u];
          earlier += i + u < tile ? v[u] : 0;
        }
      }
      for (; i < end; ++i, from += E) {
        total += *from;
        earlier += i < tile ? *from : 0;
      }
    }
    parts[0][t] = total;
    parts[1][t] = earlier;
    __syncthreads();
    total = earlier = 0;
    if (t < E)
      for (int s = 0; s < shares; ++s) {
        total += parts[0][s * E + t];
        earlier += parts[1][s * E + t];
      }
  } else if (t < E) {
    total = totals[t];
    earlier = counts[static_cast<int64_t>(tile) * E + t];
  }
  const int to_here = wave_sum_to_here(total);
  if (lane == 63) sums[wave] = static_cast<uint32_t>(to_here);
  __syncthreads();
  int lower = to_here - total, all = 0;
  for (int w = 0; w < kOrderWaves; ++w) {
    if (w < wave) lower += static_cast<int>(sums[w]);
    all += static_cast<int>(sums[w]);
  }
  if (t < E) {
    begins[t] = lower + earlier;
    if (tile == 0) sizes[t] = total;
  }
  __syncthreads();                              // (sums are used again)
  const int place = place_of_mine(key, bits, of_tile, sums);
  if (mine) {
    const bool there = key < static_cast<uint32_t>(E);
    const int slot = there ? begins[key] + place - of_tile[key * kOrderWaves] : -1;
    slots[at] = slot;
    if (there) order[slot] = at;
    if (at >= all) order[at] = -1;              // behind the last slot
  }
}

// A routing of a few tokens, with its order, by one workgroup.
template <typename T, int R, typename A>
__global__ __launch_bounds__(kOrderThreads) void route_few_kernel(const A a, int bits, int32_t* slots, int32_t* order, int32_t* sizes) {
  __shared__ uint16_t counts[kOrderWaves << kMostRange];
  __shared__ uint32_t keys[kOrderThreads], sums[kOrderWaves];
  __shared__ int32_t chosen[kOrderThreads];
  const int t = threadIdx.x, lane = t & 63, of_row = lane & 15, token = t / kRouteLanes, n = a.T * a.k;
  int expert;
  float weight;
  route_choose<T, R>(a, token, lane, chosen + (t & ~63), &expert, &weight);
  if (token < a.T && of_row < a.k) {
    a.experts[token * a.k + of_row] = expert;
    a.weights[token * a.k + of_row] = weight;
    keys[token * a.k + of_row] = static_cast<uint32_t>(expert >= 0 ? expert : a.E);
  }
  __syncthreads();
  const uint32_t key = t < n ? keys[t] : (1u << bits) - 1;   // behind all others, or among those without an expert and behind them
  const int place = place_of_mine(key, bits, counts, sums);
  const bool there = key < static_cast<uint32_t>(a.E);
  if (t < n) {
    slots[t] = there ? place : -1;
    order[place] = there ? t : -1;
  }
  for (int e = t; e < a.E; e += kOrderThreads) sizes[e] = counts[(e + 1) * kOrderWaves] - counts[e * kOrderWaves];
}

// dlogits: of weights from all experts p (g - sum p g), g zero where not chosen; from the chosen ones the same among them, zeros elsewhere.  What the choices add is put where their experts are in LDS.
template <typename T, int R, typename A>
__global__ __launch_bounds__(256) void route_grad_kernel(const A a) {
  __shared__ __attribute__((aligned(16))) float added[256 / kRouteLanes][kRouteLanes * R];
  const int lane = threadIdx.x & 63, of_row = lane & 15, token = (blockIdx.x * 256 + threadIdx.x) / kRouteLanes;
  float* const add = added[threadIdx.x / kRouteLanes];
  const bool in = token < a.ts * a.shards, live = token < a.T;
  const int shard = in ? embed_shard(token, a.ts, a.shards) : 0, within = token - shard * a.ts;
  const T* z = live && !a.normalise ? static_cast<const T*>(first_kernel_argument<A>()->shard[shard].logits) + static_cast<int64_t>(within) * a.ld : nullptr;
  T* const d = in ? static_cast<T*>(first_kernel_argument<A>()->shard[shard].dlogits) : nullptr;
  const int64_t at = static_cast<int64_t>(token) * a.k + of_row;
  const bool mine = live && of_row < a.k;
  const int expert = mine ? a.experts[at] : -1;
  const bool chosen = expert >= 0 && expert < a.E;
  const float w = chosen ? a.weights[at] : 0.f, g = chosen ? a.dweights[at] : 0.f;
  float v[R];
  if (a.normalise) {
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = 0.f;
  } else {
    const bool strange = route_load<T, R>(z, a.E, of_row, lane, v);
    float best = v[0];
#pragma unroll
    for (int r = 1; r < R; ++r) best = fmaxf(best, v[r]);
    const float most = row_max(best), each = 1.f / route_total<R>(v, most, strange);
    const bool none = row_ballot(chosen, lane) == 0 || (most == -INFINITY && !strange);        // a token without experts has no gradient, whatever its logits hold
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = none ? 0.f : expf(v[r] - most) * each;
  }
  const float mean = row_sum(w * g), own = a.normalise ? w * (g - mean) : w * g, all = a.normalise ? 0.f : -mean;      // (what is not chosen: zeros, also where the mean is not finite)
#pragma unroll
  for (int r = 0; r < R; ++r) add[of_row * R + r] = 0.f;
  staged_in_order();
  if (chosen) add[expert] = __int_as_float(of_row);
  staged_in_order();
  const bool alone = !chosen || __float_as_int(add[expert]) == of_row;
  staged_in_order();
  if (__builtin_amdgcn_ballot_w64(!alone) == 0) {
    if (chosen) add[expert] = own;
  } else {                                       // an expert twice (no routing of gspmd_route's): one choice after the other
    if (chosen) add[expert] = 0.f;
    staged_in_order();
    for (int i = 0; i < a.k; ++i) {
      if (chosen && of_row == i) add[expert] += own;
      staged_in_order();
    }
  }
  staged_in_order();
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = fmaf(v[r], all, add[of_row * R + r]);
  if (d == nullptr) return;
  constexpr int n = Sixteen<T>::n;
  if constexpr (R % n == 0) {
    if ((of_row + 1) * R <= a.E) {
      T* const to = d + static_cast<int64_t>(within) * a.ld_d + of_row * R;
#pragma unroll
      for (int i = 0; i < R / n; ++i) {
        float f[n];
#pragma unroll
        for (int e = 0; e < n; ++e) f[e] = live ? v[i * n + e] : 0.f;
        store16(to + i * n, Sixteen<T>::close(f));
      }
      return;
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (of_row * R + r < a.E) store_from_float<T>(d + static_cast<int64_t>(within) * a.ld_d + of_row * R + r, live ? v[r] : 0.f);
}

// ---- the exchange
constexpr int kExpertShards = 64;
struct ExchangeArgs {
  void* tokens[kTokenShards];      // rows by token: x, y or dy; null: none to be written.  (These three first in the kernel's arguments: read there.)
  void* rows[kExpertShards];       // by slot, of the experts' shards
  void* drows[kExpertShards];
  int32_t T, ts, token_shards, k, E, es, expert_shards, M;
  int64_t ld_tokens, ld_rows, ld_drows;
  const int32_t *experts, *slots;
  const float* weights;            // null: all 1
  float* dweights;
};
__device__ __forceinline__ const GSPMD_KERNARG ExchangeArgs* exchange_arguments() { return first_kernel_argument<ExchangeArgs>(); }
// (one shard: an address that is read with the other arguments, not once its number is known)
__device__ __forceinline__ void* tokens_of(const ExchangeArgs& a, int shard) { return a.token_shards == 1 ? a.tokens[0] : exchange_arguments()->tokens[shard]; }
__device__ __forceinline__ void* rows_of(const ExchangeArgs& a, int part) { return a.expert_shards == 1 ? a.rows[0] : exchange_arguments()->rows[part]; }

// The shard of choice `o`'s expert, or -1 if it has none.
__device__ __forceinline__ int expert_shard(const ExchangeArgs& a, int o) {
  if (a.expert_shards == 1) return 0;
  const uint32_t e = static_cast<uint32_t>(((GSPMD_GLOBAL const int32_t*)a.experts)[o]);
  return e < static_cast<uint32_t>(a.E) ? static_cast<int>(e / static_cast<uint32_t>(a.es)) : -1;
}

// rows[slot] = x[token of the slot]: a wave has a piece of a token's row, or a few tokens' short rows, which it reads once and writes to each of their slots.  (Slot by slot, a row read
// for each of them: 16384 tokens of 1024, 8 choices, with combine_kernel 127 us, so 113.)
constexpr int kExchangeUnroll = 4;
template <typename T, int LINES>
__global__ __launch_bounds__(256) void dispatch_kernel(const ExchangeArgs a, int log_lanes, int pieces) {
  constexpr int n = Sixteen<T>::n;
  const int log = LINES == kWide ? 6 : log_lanes, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = blockIdx.x / pieces, piece = blockIdx.x - group * pieces;       // (neighbouring pieces of rows together)
  const int token = of_row<LINES>(((group * 4 + wave) << (6 - log)) + (lane >> log));
  if (token >= a.T) return;
  const int shard = of_row<LINES>(embed_shard(token, a.ts, a.token_shards));
  const T* const x = static_cast<const T*>(tokens_of(a, shard)) + (token - shard * a.ts) * a.ld_tokens;
  const int col0 = (((piece * kExchangeUnroll) << log) + (lane & ((1 << log) - 1))) * n, step = n << log;
  // its slot, or -1, and where that lies
  auto slot_of = [&](int o, int* part) {
    const int slot = ((GSPMD_GLOBAL const int32_t*)a.slots)[o];
    *part = expert_shard(a, o);
    return static_cast<uint32_t>(slot) < static_cast<uint32_t>(a.T * a.k) && *part >= 0 ? slot : -1;
  };
  int part = 0;
  static_assert(kMostChoices <= 64, "a lane for every choice");
  const int slots = LINES == kWide ? slot_of(token * a.k + min(lane, a.k - 1), &part) : 0, parts = part;      // (of a wave's one token: a choice a lane)
  u32x4_t v[kExchangeUnroll];
#pragma unroll
  for (int u = 0; u < kExchangeUnroll; ++u) v[u] = load_line<LINES, T>(x, line_at<LINES, T>(col0 + u * step, a.M), a.M);
  for (int i = 0; i < a.k; ++i) {
    int slot;
    if constexpr (LINES == kWide) {
      slot = __builtin_amdgcn_readlane(slots, i);
      part = __builtin_amdgcn_readlane(parts, i);
    } else {
      slot = slot_of(token * a.k + i, &part);
    }
    if (slot < 0) continue;
    T* to = static_cast<T*>(rows_of(a, part));
    if (to == nullptr) continue;
    to += slot * a.ld_rows;
#pragma unroll
    for (int u = 0; u < kExchangeUnroll; ++u)
      if (col0 + u * step < a.M) store_line<LINES, T>(to, line_at<LINES, T>(col0 + u * step, a.M), a.M, v[u]);
  }
}

// y[t] = sum over t's choices of weight * rows[slot], in float32, in their order; what has no slot adds nothing.
constexpr int kCombineAhead = 4, kCombineUnroll = 2;
template <typename T, int LINES>
__global__ __launch_bounds__(256) void combine_kernel(const ExchangeArgs a, int log_lanes, int pieces) {
  constexpr int n = Sixteen<T>::n;
  const int log = LINES == kWide ? 6 : log_lanes, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = blockIdx.x / pieces, piece = blockIdx.x - group * pieces;
  const int token = of_row<LINES>(((group * 4 + wave) << (6 - log)) + (lane >> log));
  if (token >= a.ts * a.token_shards) return;
  const int shard = of_row<LINES>(embed_shard(token, a.ts, a.token_shards)), col0 = (((piece * kCombineUnroll) << log) + (lane & ((1 << log) - 1))) * n, step = n << log;
  T* y = static_cast<T*>(tokens_of(a, shard));
  if (y == nullptr || col0 >= a.M) return;
  y += (token - shard * a.ts) * a.ld_tokens;
  float sum[kCombineUnroll][n];
#pragma unroll
  for (int p = 0; p < kCombineUnroll; ++p)
#pragma unroll
    for (int e = 0; e < n; ++e) sum[p][e] = 0.f;
  if (token < a.T) {
#pragma unroll 1
    for (int i = 0; i < a.k; i += kCombineAhead) {
      u32x4_t v[kCombineAhead][kCombineUnroll];
      float w[kCombineAhead];
      // choices beyond the last are the last again, those without a slot the first row, with a weight of 0 and zeros for a row: no branch, a load in one is waited for there
      int slot[kCombineAhead], part[kCombineAhead];
#pragma unroll
      for (int u = 0; u < kCombineAhead; ++u) {
        const int o = token * a.k + min(i + u, a.k - 1);
        slot[u] = of_row<LINES>(((GSPMD_GLOBAL const int32_t*)a.slots)[o]);
        part[u] = a.expert_shards == 1 ? 0 : of_row<LINES>(((GSPMD_GLOBAL const int32_t*)a.experts)[o]);
        w[u] = a.weights ? ((GSPMD_GLOBAL const float*)a.weights)[o] : 1.f;
      }
      bool there[kCombineAhead];
#pragma unroll
      for (int u = 0; u < kCombineAhead; ++u) {
        there[u] = i + u < a.k && static_cast<uint32_t>(slot[u]) < static_cast<uint32_t>(a.T * a.k) && (a.expert_shards == 1 || static_cast<uint32_t>(part[u]) < static_cast<uint32_t>(a.E));
        const int of = there[u] && a.expert_shards != 1 ? of_row<LINES>(static_cast<int>(static_cast<uint32_t>(part[u]) / static_cast<uint32_t>(a.es))) : 0;
        const T* const from = static_cast<const T*>(rows_of(a, of)) + (there[u] ? slot[u] : 0) * a.ld_rows;
#pragma unroll
        for (int p = 0; p < kCombineUnroll; ++p) v[u][p] = load_line<LINES, T>(from, line_at<LINES, T>(col0 + p * step, a.M), a.M);
      }
#pragma unroll
      for (int u = 0; u < kCombineAhead; ++u) {
        if (!there[u]) continue;
#pragma unroll
        for (int p = 0; p < kCombineUnroll; ++p) {
          float f[n];
          Sixteen<T>::open(v[u][p], f);
#pragma unroll
          for (int e = 0; e < n; ++e) sum[p][e] = fmaf(w[u], f[e], sum[p][e]);
        }
      }
    }
  }
#pragma unroll
  for (int p = 0; p < kCombineUnroll; ++p)
    if (col0 + p * step < a.M) store_line<LINES, T>(y, line_at<LINES, T>(col0 + p * step, a.M), a.M, Sixteen<T>::close(sum[p]));
}

// drows[slot] = weight * dy[t] and dweight = the product of dy[t] and rows[slot], a wave for a choice (or a few with short rows).
template <typename T, int LINES>
__global__ __launch_bounds__(256) void combine_grad_kernel(const ExchangeArgs a, int log_lanes) {
  constexpr int n = Sixteen<T>::n, kAhead = 2;
  const int log = LINES == kWide ? 6 : log_lanes, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lanes = 1 << log;
  const int o = of_row<LINES>(((blockIdx.x * 4 + wave) << (6 - log)) + (lane >> log));
  const bool in = o < a.T * a.k;
  const int slot = in ? of_row<LINES>(((GSPMD_GLOBAL const int32_t*)a.slots)[o]) : -1, part = in ? of_row<LINES>(expert_shard(a, o)) : -1;
  const bool there = static_cast<uint32_t>(slot) < static_cast<uint32_t>(a.T * a.k) && part >= 0;
  float dot = 0.f;
  if (there) {
    const int token = of_row<LINES>(static_cast<int>(static_cast<uint32_t>(o) / static_cast<uint32_t>(a.k))), shard = of_row<LINES>(embed_shard(token, a.ts, a.token_shards));
    const T* const dy = static_cast<const T*>(tokens_of(a, shard)) + (token - shard * a.ts) * a.ld_tokens;
    const T* const row = static_cast<const T*>(rows_of(a, part)) + slot * a.ld_rows;
    T* drow = static_cast<T*>(exchange_arguments()->drows[part]);
    const bool wanted = drow != nullptr;
    if (wanted) drow += slot * a.ld_drows;
    const float w = ((GSPMD_GLOBAL const float*)a.weights)[o];
    const int step = n << log;
#pragma unroll 1
    for (int col0 = (lane & (lanes - 1)) * n; col0 < a.M; col0 += kAhead * step) {
      u32x4_t g[kAhead], v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int at = line_at<LINES, T>(col0 + u * step, a.M);
        g[u] = load_line<LINES, T>(dy, at, a.M);
        v[u] = load_line<LINES, T>(row, at, a.M);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int col = col0 + u * step, at = line_at<LINES, T>(col, a.M);
        if (col >= a.M) continue;
        float p[n], q[n], r[n];
        Sixteen<T>::open(g[u], p);
        Sixteen<T>::open(v[u], q);
#pragma unroll
        for (int e = 0; e < n; ++e) r[e] = p[e] * w;
        if (wanted) store_line<LINES, T>(drow, at, a.M, Sixteen<T>::close(r));
        if (LINES != kExact && at < col) {      // what the neighbour has of the product
#pragma unroll
          for (int e = 0; e < n; ++e)
            if (at + e < col) p[e] = q[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < n; ++e) dot = fmaf(p[e], q[e], dot);
      }
    }
  }
  for (int by = 1; by < lanes; by *= 2) dot += __shfl_xor(dot, by);
  if (in && (lane & (lanes - 1)) == 0) a.dweights[o] = there ? dot : 0.f;
}

}  // namespace gspmd
