// Tokens ordered by an index of theirs, the vocabulary entry, and, of one index, as they come.
//
// A workgroup has a range of the indexes, looks through ALL keys and takes those of its range: how many are below it is where its own begin, so the workgroups need nothing of each
// other, and one launch orders any number of keys of any size.  Each reads every key twice, from L2; a sort by digits reads them fewer times but has a chain of launches, or of one workgroup's
// rounds (us, digits / this: 2048 keys below 32000 10.3 / 4.3, 9999 27.8 / 8.3).
// Its sixteen waves have a part of the keys each.  First they count, by index and wave, with atomics in LDS whose order does not matter; sums over the counts are places.  Then every wave goes
// through its part again, sixty-four keys at a time, in order: lanes with the same index are found, and take consecutive places.  Of sixty-four keys a range has hardly any but for an index that many keys
// have: the first lane's index, those that have it, the next lane's that is left ..., and for what is left after kLeaders of them a ballot for each bit (ballots alone, us: 9999 keys below 32000,
// a tenth of them one, 12.9; 32768, 30.1).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels_basic.h"
#include "kernels_rows.h"
#include "mfma_common.h"
#include "order.h"
#include "ragged.h"

namespace gspmd {

constexpr int kLeaders = 4;
template <int SHARDS>
struct OrderWork {
  OrderKeysOf<SHARDS> in;
  OrderOut out;
  ZeroRowsOf<SHARDS> zero;
  int32_t log_range, groups;                    // of workgroups that order; those behind them zero rows
  int32_t zero_log, zero_pieces;                // lanes of a row, as a power of two; pieces of kZeroUnroll x 16 bytes a lane
};

// Rows zeroed, beside the order, whose time it hides (131 MB with the order of 2048 tokens 20 us, 6.5 TB/s): a workgroup has a piece of every so-many-th row, a wave one row (or a few short ones) at a time.
constexpr int kZeroUnroll = 4;
template <int SHARDS>
__device__ __forceinline__ void zero_rows(const OrderWork<SHARDS>& w) {
  typedef bf16_bits half;
  constexpr int n = Sixteen<half>::n;
  const ZeroRowsOf<SHARDS>& z = w.zero;
  const int block = blockIdx.x - w.groups, of = gridDim.x - w.groups, piece = block % w.zero_pieces, log = w.zero_log, side = 6 - log;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), count = z.per * z.shards - z.from;
  const int col0 = (((piece * kZeroUnroll) << log) + (lane & ((1 << log) - 1))) * n, turn = (of / w.zero_pieces * kOrderWaves) << side;
  for (int64_t base = static_cast<int64_t>(block / w.zero_pieces * kOrderWaves + wave) << side; base < count; base += turn) {
    const int row = static_cast<int>(base) + (lane >> log) + z.from;
    if (row - z.from >= count) break;
    int shard = z.shards == 1 ? 0 : static_cast<int>(static_cast<uint32_t>(row) / static_cast<uint32_t>(z.per));
    if (log == 6) shard = __builtin_amdgcn_readfirstlane(shard);
    half* const to = static_cast<half*>(z.shards == 1 ? z.shard[0] : first_kernel_argument<OrderWork<SHARDS>>()->zero.shard[shard]);
    if (to == nullptr) continue;
    half* const at = to + static_cast<int64_t>(row - shard * z.per) * z.stride;
    const u32x4_t zeros = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int u = 0; u < kZeroUnroll; ++u) {
      const int col = col0 + ((u << log) * n);
      if (col < z.halves) {
        if (z.halves >= n) store_line<kNarrow, half>(at, line_at<kNarrow, half>(col, z.halves), z.halves, zeros);
        else store_some(at, zeros, z.halves);
      }
    }
  }
}

template <int SHARDS>
__global__ __launch_bounds__(kOrderThreads) void order_kernel(const OrderWork<SHARDS> w) {
  extern __shared__ __attribute__((aligned(16))) int32_t counts[];      // [range][waves]
  __shared__ int32_t sums[kOrderWaves], below[kOrderWaves];
  __shared__ const int32_t* from[SHARDS];
  if (static_cast<int>(blockIdx.x) >= w.groups) {
    zero_rows(w);
    return;
  }
  const OrderKeysOf<SHARDS>& in = w.in;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), log_range = w.log_range, entries = kOrderWaves << log_range;
  const int lo = blockIdx.x << log_range, range = min(1 << log_range, in.keys - lo);
  const int part = ((in.count + kOrderWaves - 1) / kOrderWaves + 63) & ~63, first = min(wave * part, in.count), end = min(first + part, in.count);
  if (in.shards > 1 && t < in.shards) from[t] = first_kernel_argument<OrderWork<SHARDS>>()->in.shard[t];
  for (int i = t; i < entries; i += kOrderThreads) counts[i] = 0;
  __syncthreads();
  constexpr int kAhead = 4;
  int key[kAhead];
  // this lane's of 64 x kAhead keys from `base` on, INT32_MAX behind the wave's last; what is no key is `keys`.  (No branch: a load in one is waited for there.)
  auto load = [&](int base) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = min(base + u * 64 + lane, end - 1);
      if (in.shards == 1) {
        key[u] = ((GSPMD_GLOBAL const int32_t*)in.shard[0])[i];
      } else {
        const int s = static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(in.per));
        key[u] = ((GSPMD_GLOBAL const int32_t*)from[s])[i - s * in.per];
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      key[u] = base + u * 64 + lane >= end ? INT32_MAX : static_cast<int>(min(static_cast<uint32_t>(key[u]), static_cast<uint32_t>(in.keys)));
  };
  int less = 0;
  for (int base = first; base < end; base += 64 * kAhead) {
    load(base);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      less += key[u] < lo;
      if (key[u] >= lo && key[u] < lo + range) atomicAdd(&counts[(key[u] - lo) * kOrderWaves + wave], 1);
    }
  }
  less = wave_sum_to_here(less);
  if (lane == 63) below[wave] = less;
  __syncthreads();
  // places: exclusive sums over [range][waves], a run of entries a thread, from the number of keys below the range on
  const int each = (entries + kOrderThreads - 1) / kOrderThreads, mine = t * each;
  int sum = 0;
  for (int i = 0; i < each; ++i) sum += mine + i < entries ? counts[mine + i] : 0;
  const int to_here = wave_sum_to_here(sum);
  if (lane == 63) sums[wave] = to_here;
  __syncthreads();
  const int of_waves = wave_sum_to_here(lane < kOrderWaves ? sums[lane] : 0), all_below = wave_sum_to_here(lane < kOrderWaves ? below[lane] : 0);
  const int lower = __builtin_amdgcn_readlane(all_below, kOrderWaves - 1);
  int at = lower + to_here - sum + (wave > 0 ? __builtin_amdgcn_readlane(of_waves, max(wave - 1, 0)) : 0);
  for (int i = 0; i < each; ++i)
    if (mine + i < entries) {
      const int n = counts[mine + i];
      counts[mine + i] = at;
      at += n;
    }
  __syncthreads();
  for (int i = t; i < range; i += kOrderThreads) w.out.begins[lo + i] = counts[i * kOrderWaves];
  if (lo + range == in.keys && t == 0) w.out.begins[in.keys] = lower + __builtin_amdgcn_readlane(of_waves, kOrderWaves - 1);
  __syncthreads();                              // (what was read there changes below)
  const uint64_t before = (uint64_t(1) << lane) - 1;
  for (int base = first; base < end; base += 64 * kAhead) {
    if (end - first > 64 * kAhead) load(base);  // (else they are there)
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int index = key[u] - lo;
      uint64_t left = __builtin_amdgcn_ballot_w64(key[u] >= lo && index < range);
      auto place_of = [&](bool mine, uint64_t same) {              // the lanes `same`, those of this lane's index, if it is `mine`
        if (mine) {
          int32_t* const next = counts + index * kOrderWaves + wave;
          const int place = *next + __builtin_popcountll(same & before);
          staged_in_order();                    // all have read before the first of each counts them
          if ((same & before) == 0) *next += __builtin_popcountll(same);
          w.out.order[place] = base + u * 64 + lane;
          w.out.entries[place] = key[u];
        }
        staged_in_order();
      };
#pragma unroll 1
      for (int turn = 0; left != 0 && turn < kLeaders; ++turn) {
        const int leader = __builtin_amdgcn_readlane(index, __builtin_ctzll(left));
        const uint64_t same = __builtin_amdgcn_ballot_w64(index == leader);
        place_of(index == leader, same);
        left &= ~same;
      }
      if (left != 0) {
        const bool here = (left >> lane) & 1;
        uint64_t same = left;
#pragma unroll 1
        for (int b = 0; b < log_range; ++b) {
          const bool on = (index >> b) & 1;
          const uint64_t with = __builtin_amdgcn_ballot_w64(here && on);
          same &= on ? with : ~with;
        }
        place_of(here, same);
      }
    }
  }
}

}  // namespace gspmd
