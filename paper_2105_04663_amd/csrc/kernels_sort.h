// Stable sorting of tokens by an index of theirs -- vocabulary entries, experts -- by digits of up to ten bits, the lowest first.
//
// A workgroup sorts up to 12288 keys by itself, in registers and LDS, all digits in one launch; more go in tiles of 8192, three launches a digit (counts of every tile, their sums, places).
// A digit: every wave goes through its keys sixty-four at a time, in order.  Which lanes have the same digit is found by a ballot for each of its bits; a key's rank is how many
// of its wave had its digit before, counted in LDS, so nothing depends on the order in which atomics arrive.  Counts by digit and, within, by wave are then added up to places.
// What bounds it is the length of that chain: twelve rounds of nine ballots and an LDS round trip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels_basic.h"
#include "mfma_common.h"
#include "ragged.h"

namespace gspmd {

constexpr int kSortShards = 64;
constexpr int kSortThreads = 1024, kSortMost = 12288, kSortTile = 8192;
constexpr int kSortDigit = 10;                  // bits of a digit, at most

// Where keys come from: arrays one after the other, `per` keys in each; what is not in 0 .. keys - 1 is `keys`.  The first thing in a kernel's arguments.
struct SortKeys {
  const int32_t* shard[kSortShards];
  int32_t per, shards, count, keys;
  __device__ __forceinline__ uint32_t at(int i) const {
    const int s = shards == 1 ? 0 : i / per;
    const int32_t* const from = shards == 1 ? shard[0] : first_kernel_argument<SortKeys>()->shard[s];
    const uint32_t key = static_cast<uint32_t>(((GSPMD_GLOBAL const int32_t*)from)[i - s * per]);
    return key < static_cast<uint32_t>(keys) ? key : static_cast<uint32_t>(keys);
  }
};

// Where a sorted key goes.  `sorted` nullable.  Of a routing (`slots` not null): the order of keys that are none is -1, as is their place; `sizes` the count of every key.
struct SortOut {
  int32_t *sorted, *order, *slots, *sizes;
  __device__ __forceinline__ void put(int place, uint32_t key, int from, int keys) const {
    const bool there = key < static_cast<uint32_t>(keys);
    if (sorted) sorted[place] = static_cast<int32_t>(key);
    order[place] = slots && !there ? -1 : from;
    if (slots) slots[from] = there ? place : -1;
  }
};

// One digit of a workgroup's keys: the place of each among all of them in the lower half of `place`, whose upper half is left alone.  Item i of a lane is the (wave * ITEMS + i) * 64 + lane-th key.  `count`: LDS, [digits][waves].
template <int THREADS, int ITEMS>
__device__ __forceinline__ void sort_digit(const uint32_t (&key)[ITEMS], int shift, int bits, uint16_t* count, uint32_t* sums, uint32_t (&place)[ITEMS]) {
  constexpr int kWaves = THREADS / 64;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, entries = kWaves << bits;
  for (int i = t; i < entries / 2; i += THREADS) reinterpret_cast<uint32_t*>(count)[i] = 0;      // (entries are even: a digit has a bit)
  __syncthreads();
  const uint64_t below = (uint64_t(1) << lane) - 1;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const uint32_t digit = (key[i] >> shift) & ((1u << bits) - 1);
    uint64_t same = ~uint64_t(0);
    for (int b = 0; b < bits; ++b) {
      const bool on = (digit >> b) & 1;
      const uint64_t with = __builtin_amdgcn_ballot_w64(on);
      same &= on ? with : ~with;
    }
    uint16_t* const mine = count + digit * kWaves + wave;
    const int before = *mine;
    staged_in_order();                          // all lanes have read before the first of each digit counts them
    place[i] = (place[i] & 0xffff0000u) | static_cast<uint32_t>(before + __builtin_popcountll(same & below));
    if ((same & below) == 0) *mine = static_cast<uint16_t>(before + __builtin_popcountll(same));
    staged_in_order();
    __builtin_amdgcn_sched_barrier(0);          // (one after the other: registers for twelve keys, not for what finding their places takes)
  }
  __syncthreads();
  // exclusive sums over [digits][waves], a run of entries a thread
  const int each = (entries + THREADS - 1) / THREADS, first = t * each;
  int sum = 0;
  for (int i = 0; i < each; ++i) sum += first + i < entries ? count[first + i] : 0;
  const int to_here = wave_sum_to_here(sum);
  if (lane == 63) sums[wave] = to_here;
  __syncthreads();
  int at = to_here - sum;
  for (int w = 0; w < wave; ++w) at += sums[w];
  for (int i = 0; i < each; ++i)
    if (first + i < entries) {
      const int n = count[first + i];
      count[first + i] = static_cast<uint16_t>(at);
      at += n;
    }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    uint32_t again = key[i];                    // (its counter's place worked out again, not kept in a register from above)
    asm volatile("" : "+v"(again));
    place[i] += count[((again >> shift) & ((1u << bits) - 1)) * kWaves + wave];
  }
}

// LDS: keys, where they come from, counts, sums.
template <int THREADS, int ITEMS> constexpr int sort_lds(int bits) { return THREADS * ITEMS * 6 + ((THREADS / 64) << bits) * 2 + 64; }

// All digits of up to THREADS * ITEMS keys by one workgroup.
template <int THREADS, int ITEMS>
__global__ __launch_bounds__(THREADS) void sort_block_kernel(const SortKeys in, const SortOut out, int bits, int digit) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int kAll = THREADS * ITEMS;
  uint32_t* const keys = reinterpret_cast<uint32_t*>(smem);
  uint16_t* const froms = reinterpret_cast<uint16_t*>(smem + kAll * 4);
  uint16_t* const count = froms + kAll;
  uint32_t* const sums = reinterpret_cast<uint32_t*>(count + ((THREADS / 64) << digit));
  const int t = threadIdx.x, first = (t >> 6) * ITEMS * 64 + (t & 63);
  uint32_t key[ITEMS];
  uint32_t place[ITEMS];                        // and, in the upper half, where the key comes from
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int from = first + i * 64;
    place[i] = static_cast<uint32_t>(from) << 16;
    key[i] = from < in.count ? in.at(from) : ~0u;             // behind all others: all ones in every digit, and last before the first
    if (i % 4 == 3) asm volatile("" ::: "memory");            // (registers for the addresses of four)
  }
  for (int shift = 0; shift < bits; shift += digit) {
    const int here = min(digit, bits - shift);
    sort_digit<THREADS, ITEMS>(key, shift, here, count, sums, place);
    if (out.sizes && shift + here >= bits) {                  // a routing has one digit
      for (int k = t; k < in.keys; k += THREADS) {
        constexpr int kWaves = THREADS / 64;
        out.sizes[k] = count[(k + 1) * kWaves] - count[k * kWaves];      // (k + 1 <= in.keys is a digit)
      }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      keys[place[i] & 0xffff] = key[i];
      froms[place[i] & 0xffff] = static_cast<uint16_t>(place[i] >> 16);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      key[i] = keys[first + i * 64];
      place[i] = static_cast<uint32_t>(froms[first + i * 64]) << 16;
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (first + i * 64 < in.count) out.put(first + i * 64, key[i], static_cast<int>(place[i] >> 16), in.keys);
    if (i % 4 == 3) asm volatile("" ::: "memory");
  }
}

// One digit of many tiles.  What has been sorted by lower digits: `keys` and `froms` (null for the first: the keys as they come).
struct SortTiles {
  SortKeys in;
  const uint32_t* keys;
  const int32_t* froms;
  uint32_t* counts;            // [digits][tiles]
  uint32_t* to_keys;           // where the digit is not the last
  int32_t* to_froms;
  SortOut out;                 // where it is
  int32_t tiles, shift, bits, last;
};

template <int ITEMS>
__device__ __forceinline__ void sort_tile_load(const SortTiles& a, uint32_t (&key)[ITEMS], int (&from)[ITEMS], int first, int base) {
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int at = base + first + i * 64;
    const bool there = at < a.in.count;
    key[i] = !there ? ~0u : a.keys ? a.keys[at] : a.in.at(at);
    from[i] = !there ? 0 : a.froms ? a.froms[at] : at;
  }
}

// 0: counts.  2: places.
template <int STEP>
__global__ __launch_bounds__(kSortThreads) void sort_tiles_kernel(const SortTiles a) {
  constexpr int ITEMS = kSortTile / kSortThreads, kWaves = kSortThreads / 64;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  uint32_t* const keys = reinterpret_cast<uint32_t*>(smem);
  int32_t* const froms = reinterpret_cast<int32_t*>(smem + kSortTile * 4);
  uint16_t* const count = reinterpret_cast<uint16_t*>(smem + kSortTile * 8);
  uint32_t* const sums = reinterpret_cast<uint32_t*>(count + (kWaves << a.bits));
  const int t = threadIdx.x, first = (t >> 6) * ITEMS * 64 + (t & 63), tile = blockIdx.x, base = tile * kSortTile, digits = 1 << a.bits;
  uint32_t key[ITEMS];
  int from[ITEMS];
  uint32_t place[ITEMS] = {};
  sort_tile_load<ITEMS>(a, key, from, first, base);
  sort_digit<kSortThreads, ITEMS>(key, a.shift, a.bits, count, sums, place);
  const int here = min(kSortTile, a.in.count - base);
  auto begin = [&](int d) { return static_cast<int>(count[d * kWaves]); };
  if constexpr (STEP == 0) {
    // (what lies beyond the last key is among the last digit's, behind its keys)
    for (int d = t; d < digits; d += kSortThreads) a.counts[static_cast<int64_t>(d) * a.tiles + tile] = (d + 1 < digits ? min(begin(d + 1), here) : here) - min(begin(d), here);
  } else {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      keys[place[i]] = key[i];
      froms[place[i]] = from[i];
    }
    __syncthreads();
    for (int at = t; at < here; at += kSortThreads) {         // neighbours of one digit go side by side
      const uint32_t k = keys[at];
      const int d = (k >> a.shift) & (digits - 1), to = static_cast<int>(a.counts[static_cast<int64_t>(d) * a.tiles + tile]) + at - begin(d);
      if (a.last) {
        a.out.put(to, k, froms[at], a.in.keys);
      } else {
        a.to_keys[to] = k;
        a.to_froms[to] = froms[at];
      }
    }
  }
}

// Exclusive sums over the counts, by one workgroup; of a routing also every key's size.
__global__ __launch_bounds__(kSortThreads) static void sort_sums_kernel(uint32_t* counts, int entries, int tiles, int32_t* sizes, int keys, int total) {
  __shared__ uint32_t sums[kSortThreads / 64];
  constexpr int kEach = 8;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t before = 0;
  for (int base = 0; base < entries; base += kSortThreads * kEach) {
    uint32_t n[kEach];
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = base + t * kEach + i;
      n[i] = at < entries ? counts[at] : 0;
      sum += static_cast<int>(n[i]);
    }
    const int to_here = wave_sum_to_here(sum);
    if (lane == 63) sums[wave] = static_cast<uint32_t>(to_here);
    __syncthreads();
    uint32_t at_sum = before + static_cast<uint32_t>(to_here - sum);
    for (int w = 0; w < kSortThreads / 64; ++w) {
      if (w < wave) at_sum += sums[w];
      before += sums[w];
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = base + t * kEach + i;
      if (at < entries) counts[at] = at_sum;
      at_sum += n[i];
    }
    __syncthreads();
  }
  if (sizes == nullptr) return;
  __threadfence_block();
  __syncthreads();
  for (int k = t; k < keys; k += kSortThreads) {
    const int next = (k + 1) * tiles;
    sizes[k] = static_cast<int32_t>((next < entries ? counts[next] : static_cast<uint32_t>(total)) - counts[k * tiles]);
  }
}

}  // namespace gspmd
