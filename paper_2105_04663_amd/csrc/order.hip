// Tokens ordered by an index (kernels_order.h): the launch.
#include "order.h"

#include "kernels_order.h"
#include "tokens.h"

namespace gspmd {

// Ranges for about a workgroup on every compute unit: with more, the keys are read more often, with fewer, longer.
constexpr int kOrderGroups = 256;

int32_t run_order(const OrderKeys& in, const OrderOut& out, hipStream_t stream) {
  int log = 0;
  while (log < kMostRange && (static_cast<int64_t>(kOrderGroups) << log) < in.keys) ++log;
  const unsigned groups = static_cast<unsigned>((static_cast<int64_t>(in.keys) + (int64_t(1) << log) - 1) >> log);
  hipLaunchKernelGGL(order_kernel, dim3(groups), dim3(kOrderThreads), static_cast<size_t>(kOrderWaves << log) * 4, stream, in, out, log);
  return launched();
}

}  // namespace gspmd
