// Tokens ordered by an index of theirs (kernels_order.h).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/gspmd.h"
#include "kernels_basic.h"

namespace gspmd {

constexpr int kKeyShards = 64;
constexpr int kOrderThreads = 1024, kOrderWaves = kOrderThreads / 64;
constexpr int kMostRange = 10;                  // indexes of a workgroup's range, at most, as a power of two: 64 KiB of counts

// Where keys come from: arrays one after the other, `per` keys in each; what is not in 0 .. keys - 1 is `keys`.  The first thing in a kernel's arguments.
struct OrderKeys {
  const int32_t* shard[kKeyShards];
  int32_t per, shards, count, keys;
  __device__ __forceinline__ int at(int i) const {
    const int s = shards == 1 ? 0 : static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(per));
    const int32_t* const from = shards == 1 ? shard[0] : first_kernel_argument<OrderKeys>()->shard[s];
    const uint32_t key = static_cast<uint32_t>(((GSPMD_GLOBAL const int32_t*)from)[i - s * per]);
    return static_cast<int>(min(key, static_cast<uint32_t>(keys)));
  }
};

// order: of every place the key's number, up to the last that is one; begins [keys + 1]: where each index's run begins.
struct OrderOut {
  int32_t *order, *begins;
};

// One launch; nothing else is needed.
int32_t run_order(const OrderKeys& in, const OrderOut& out, hipStream_t stream);

}  // namespace gspmd
