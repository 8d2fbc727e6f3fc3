// Tokens ordered by an index (kernels_order.h): the launch.
#include "order.h"

#include <algorithm>

#include "kernels_order.h"
#include "tokens.h"

namespace gspmd {

// Ranges for about a workgroup on every compute unit: with more, the keys are read more often, with fewer, longer.
constexpr int kOrderGroups = 256;

// Workgroups that zero rows, at most: two on every compute unit are there at a time.
constexpr int kZeroGroups = 1024;

template <int SHARDS>
int32_t launch_order(const OrderKeys& in, const OrderOut& out, const ZeroRows& zero, hipStream_t stream) {
  OrderWork<SHARDS> w{};
  std::copy_n(in.shard, SHARDS, w.in.shard);
  w.in.per = in.per;
  w.in.shards = in.shards;
  w.in.count = in.count;
  w.in.keys = in.keys;
  w.out = out;
  std::copy_n(zero.shard, SHARDS, w.zero.shard);
  w.zero.per = zero.per;
  w.zero.shards = zero.shards;
  w.zero.from = zero.from;
  w.zero.halves = zero.halves;
  w.zero.stride = zero.stride;
  if (in.count > 0) {
    while (w.log_range < kMostRange && (static_cast<int64_t>(kOrderGroups) << w.log_range) < in.keys) ++w.log_range;
    w.groups = static_cast<int32_t>((static_cast<int64_t>(in.keys) + (int64_t(1) << w.log_range) - 1) >> w.log_range);
  }
  int64_t groups = 0;
  const int64_t rows = static_cast<int64_t>(zero.per) * zero.shards - zero.from;
  if (rows > 0 && zero.halves > 0) {
    constexpr int n = Sixteen<bf16_bits>::n;
    w.zero_log = row_lanes_log(zero.halves, n);
    const int64_t piece = static_cast<int64_t>(kZeroUnroll) * n << w.zero_log, at_once = static_cast<int64_t>(kOrderWaves) << (6 - w.zero_log);
    w.zero_pieces = static_cast<int32_t>((zero.halves + piece - 1) / piece);
    groups = std::min<int64_t>((rows + at_once - 1) / at_once, std::max<int64_t>(1, kZeroGroups / w.zero_pieces)) * w.zero_pieces;
  }
  groups += w.groups;
  if (groups == 0) return GSPMD_OK;
  if (groups > INT32_MAX) return GSPMD_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((order_kernel<SHARDS>), dim3(static_cast<unsigned>(groups)), dim3(kOrderThreads), static_cast<size_t>(kOrderWaves << w.log_range) * 4, stream, w);
  return launched();
}

int32_t run_order(const OrderKeys& in, const OrderOut& out, const ZeroRows& zero, hipStream_t stream) {
  return std::max(in.shards, zero.shards) <= kFewKeyShards ? launch_order<kFewKeyShards>(in, out, zero, stream) : launch_order<kKeyShards>(in, out, zero, stream);
}

}  // namespace gspmd
