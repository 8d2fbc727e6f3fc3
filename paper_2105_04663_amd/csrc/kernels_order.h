// Tokens ordered by an index of theirs -- vocabulary entries, experts -- and, of one index, as they come.
//
// A workgroup has a range of the indexes, looks through ALL keys and takes those of its range: how many are below it is where its own begin, so the workgroups need nothing of each
// other, and one launch orders any number of keys of any size.  Each reads every key twice, from L2; a sort by digits reads them fewer times but has a chain of launches, or of one workgroup's
// rounds (us, digits / this: 2048 keys below 32000 10.3 / 5.2, 9999 27.8 / 7.6, 131072 below 128, three launches, 32 / 15).
// Its sixteen waves have a part of the keys each.  First they count, by index and wave, with atomics in LDS whose order does not matter; sums over the counts are places.  Then every wave goes
// through its part again, sixty-four keys at a time, in order: lanes with the same index are found by a ballot for each of its bits, and take consecutive places.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels_basic.h"
#include "mfma_common.h"
#include "order.h"
#include "ragged.h"

namespace gspmd {

__global__ __launch_bounds__(kOrderThreads) void order_kernel(const OrderKeys in, const OrderOut out, int log_range) {
  extern __shared__ __attribute__((aligned(16))) int32_t counts[];      // [range][waves]
  __shared__ int32_t sums[kOrderWaves], below[kOrderWaves];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), entries = kOrderWaves << log_range;
  const int lo = blockIdx.x << log_range, range = min(1 << log_range, in.keys - lo);
  const int part = ((in.count + kOrderWaves - 1) / kOrderWaves + 63) & ~63, first = min(wave * part, in.count), end = min(first + part, in.count);
  for (int i = t; i < entries; i += kOrderThreads) counts[i] = 0;
  __syncthreads();
  constexpr int kAhead = 16;
  int less = 0;
  for (int base = first; base < end; base += 64 * kAhead) {
    int key[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) key[u] = in.at(min(base + u * 64 + lane, end - 1));      // (no branch: a load under one is waited for there)
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (base + u * 64 + lane >= end) key[u] = INT32_MAX;
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
  int at = to_here - sum, total = 0;
  for (int w = 0; w < kOrderWaves; ++w) {
    at += below[w] + (w < wave ? sums[w] : 0);
    total += below[w] + sums[w];
  }
  for (int i = 0; i < each; ++i)
    if (mine + i < entries) {
      const int n = counts[mine + i];
      counts[mine + i] = at;
      at += n;
    }
  __syncthreads();
  for (int i = t; i < range; i += kOrderThreads) out.begins[lo + i] = counts[i * kOrderWaves];
  if (lo + range == in.keys && t == 0) out.begins[in.keys] = total;
  __syncthreads();                              // (what was read there changes below)
  const uint64_t before = (uint64_t(1) << lane) - 1;
  for (int base = first; base < end; base += 64 * kAhead) {
    int key[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) key[u] = in.at(min(base + u * 64 + lane, end - 1));      // (no branch: a load under one is waited for there)
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (base + u * 64 + lane >= end) key[u] = INT32_MAX;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int index = key[u] - lo;
      const bool here = key[u] >= lo && index < range;
      uint64_t same = __builtin_amdgcn_ballot_w64(here);
      if (same == 0) continue;
      for (int b = 0; b < log_range; ++b) {
        const bool on = (index >> b) & 1;
        const uint64_t with = __builtin_amdgcn_ballot_w64(here && on);
        same &= on ? with : ~with;
      }
      if (here) {
        int32_t* const next = counts + index * kOrderWaves + wave;
        const int place = *next + __builtin_popcountll(same & before);
        staged_in_order();                      // all have read before the first of each counts them
        if ((same & before) == 0) *next += __builtin_popcountll(same);
        out.order[place] = base + u * 64 + lane;
      }
      staged_in_order();
    }
  }
}

}  // namespace gspmd
