// Tokens ordered by an index (kernels_order.h): the launch.
#include "order.h"

#include <algorithm>

#include "kernels_order.h"
#include "tokens.h"

namespace gspmd {

// Ranges for about a workgroup on every compute unit: with more, the keys are read more often, with fewer, longer (the gradient of rows of 8, us, 64 / 128 / 256 / 512 / 1024 workgroups: 2048 tokens, 32000
// entries 17.9 / 15.2 / 14.7 / 15.8 / 18.4; 9999 tokens, 32003 27.8 / 24.4 / 23.6 / 25.5 / 31.4, 128000 34.5 / 34.5 / 26.6 / 26.4 / 32.1; 32768 tokens, 1000 39.1 / 37.3 / 36.3 / 41.9 / 54.2).
constexpr int kOrderGroups = 256;

// Workgroups that zero rows, at most: two on every compute unit are there at a time.  It hardly matters (the gradient, us, 256 / 512 / 1024 / 2048 / 4096: 2048 tokens of 2048, 32000 entries 28.9 / 28.5 / 28.3 / 28.9 /
// 28.9; of 8192, 8000 35.0 / 34.5 / 34.3 / 35.2 / 35.3; of 513, 50000 19.4 / 19.3 / 20.7 / 23.3 / 25.1; 9999 of 2048, 128000 117.3 / 117.1 / 117.4 / 115.8 / 118.1).
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
