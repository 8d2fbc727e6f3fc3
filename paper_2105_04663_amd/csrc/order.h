// Tokens ordered by an index of theirs (kernels_order.h).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/gspmd.h"
#include "kernels_basic.h"

namespace gspmd {

constexpr int kKeyShards = 64, kFewKeyShards = 8;
constexpr int kOrderThreads = 1024, kOrderWaves = kOrderThreads / 64;
constexpr int kMostRange = 10;                  // indexes of a workgroup's range, at most, as a power of two: 64 KiB of counts

// Where keys come from: arrays one after the other, `per` keys in each; what is not in 0 .. keys - 1 is `keys`.  The first thing in a kernel's arguments.
template <int SHARDS>
struct OrderKeysOf {
  const int32_t* shard[SHARDS];
  int32_t per, shards, count, keys;
};
typedef OrderKeysOf<kKeyShards> OrderKeys;

// order, entries: of every place the key's number and the key, up to the last that is one; begins [keys + 1]: where each index's run begins.
struct OrderOut {
  int32_t *order, *entries, *begins;
};

// Rows to be zeroed by the same launch, in workgroups of their own: `per` rows in each shard (null: none), row numbers from `from` on through all of them.
template <int SHARDS>
struct ZeroRowsOf {
  void* shard[SHARDS];
  int32_t per, shards, from;
  int32_t halves;              // 2-byte units of a row
  int64_t stride;              // of them
};
typedef ZeroRowsOf<kKeyShards> ZeroRows;

// One launch; nothing else is needed.  No keys: rows are zeroed only; no rows, no shards: keys are ordered only.
int32_t run_order(const OrderKeys& in, const OrderOut& out, const ZeroRows& zero, hipStream_t stream);

}  // namespace gspmd
