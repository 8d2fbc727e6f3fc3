// dot_mfma_kernel ending in a softmax's statistics (kernels_stats.h) for one operand layout (GSPMD_TU_LAYOUT: K-contiguous lhs): compiled once per layout.
#include "kernels_mfma.h"
#include "kernels_stats.h"

namespace gspmd {

template <int LAYOUT>
bool launch_dot_stats_layout(const MfmaLaunch& l, const SoftmaxFinish& finish, hipStream_t stream) {
  static std::once_flag once[kMaxDevices];
  static bool ok[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return false;
  std::call_once(once[dev], [dev] {
    ok[dev] = hipFuncSetAttribute(reinterpret_cast<const void*>(&dot_mfma_kernel<float, LAYOUT, false, SoftmaxFinish>),
                                  hipFuncAttributeMaxDynamicSharedMemorySize, kMfmaLds) == hipSuccess;
  });
  if (!ok[dev]) return false;
  hipLaunchKernelGGL((dot_mfma_kernel<float, LAYOUT, false, SoftmaxFinish>), dim3(static_cast<unsigned>(l.tiles)), dim3(kMfmaThreads), kMfmaLds, stream, *l.inl, l.tab, l.n_prob,
                     GSPMD_EPILOGUE_NONE, nullptr, nullptr, nullptr, 0, finish);
  return hipGetLastError() == hipSuccess;
}

template bool launch_dot_stats_layout<GSPMD_TU_LAYOUT>(const MfmaLaunch& l, const SoftmaxFinish& finish, hipStream_t stream);

}  // namespace gspmd
