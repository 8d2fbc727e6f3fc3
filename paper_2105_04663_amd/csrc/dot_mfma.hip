// dot_mfma_kernel for one operand layout (GSPMD_TU_LAYOUT, GSPMD_LAYOUT_* bits): compiled once per layout.
#include "kernels_mfma.h"

namespace gspmd {

template bool launch_dot_mfma_layout<GSPMD_TU_LAYOUT>(const MfmaLaunch& l, int32_t out_dtype, bool staged, hipStream_t stream);
#if GSPMD_TU_LAYOUT == 0 || GSPMD_TU_LAYOUT == 2
template bool launch_dot_stats_layout<GSPMD_TU_LAYOUT>(const MfmaLaunch& l, const SoftmaxFinish& finish, hipStream_t stream);
#endif

}  // namespace gspmd
