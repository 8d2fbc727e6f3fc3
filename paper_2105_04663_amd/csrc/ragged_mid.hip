// dot_mid_kernel and dot_pair_kernel over experts' packed rows (ragged.h) for one operand layout (GSPMD_TU_LAYOUT): compiled once per layout.
#include "kernels_mid.h"
#include "kernels_pair.h"

namespace gspmd {

// Workgroups that a compute unit has: by the launch's bound on its tiles, of which there may be fewer.
template <int LAYOUT>
bool launch_ragged_mid_layout(const MfmaLaunch& l, int32_t out_dtype, bool staged, hipStream_t stream) {
  if (staged)
    return out_dtype == GSPMD_F32 ? launch_dot_mid_as<float, LAYOUT, false, 2, true, true>(l, stream) : launch_dot_mid_as<bf16_bits, LAYOUT, false, 2, true, true>(l, stream);
  if (l.tiles <= kMidAlone)
    return out_dtype == GSPMD_F32 ? launch_dot_mid_as<float, LAYOUT, false, 1, false, true>(l, stream) : launch_dot_mid_as<bf16_bits, LAYOUT, false, 1, false, true>(l, stream);
  return out_dtype == GSPMD_F32 ? launch_dot_mid_as<float, LAYOUT, false, 2, false, true>(l, stream) : launch_dot_mid_as<bf16_bits, LAYOUT, false, 2, false, true>(l, stream);
}

template <int LAYOUT>
bool launch_ragged_pair_layout(const MfmaLaunch& l, int32_t out_dtype, hipStream_t stream) {
  if (out_dtype == GSPMD_F32) return launch_dot_pair_as<LAYOUT, float, false, true>(l, stream);
  return l.past ? launch_dot_pair_as<LAYOUT, bf16_bits, true, true>(l, stream) : launch_dot_pair_as<LAYOUT, bf16_bits, false, true>(l, stream);
}

template bool launch_ragged_mid_layout<GSPMD_TU_LAYOUT>(const MfmaLaunch&, int32_t, bool, hipStream_t);
template bool launch_ragged_pair_layout<GSPMD_TU_LAYOUT>(const MfmaLaunch&, int32_t, hipStream_t);

}  // namespace gspmd
