// dot_mfma_kernel over experts' packed rows (ragged.h) for one operand layout (GSPMD_TU_LAYOUT): compiled once per layout.
#include "kernels_mfma.h"

namespace gspmd {

template <int LAYOUT>
bool launch_ragged_mfma_layout(const MfmaLaunch& l, int32_t out_dtype, hipStream_t stream) {
  return out_dtype == GSPMD_F32 ? launch_dot_mfma_as<float, LAYOUT, false, true>(l, stream) : launch_dot_mfma_as<bf16_bits, LAYOUT, false, true>(l, stream);
}

template bool launch_ragged_mfma_layout<GSPMD_TU_LAYOUT>(const MfmaLaunch&, int32_t, hipStream_t);

}  // namespace gspmd
