// dot_split_kernel over experts' packed rows (ragged.h) for one operand layout (GSPMD_TU_LAYOUT): compiled once per layout.
#include "kernels_split.h"

namespace gspmd {

template <int LAYOUT>
bool launch_ragged_split_layout(const MfmaLaunch& l, int32_t out_dtype, int row_blocks, int col_blocks, hipStream_t stream) {
  return out_dtype == GSPMD_F32 ? launch_dot_split_out<LAYOUT, float, true>(l, row_blocks, col_blocks, stream)
                                : launch_dot_split_out<LAYOUT, bf16_bits, true>(l, row_blocks, col_blocks, stream);
}

template bool launch_ragged_split_layout<GSPMD_TU_LAYOUT>(const MfmaLaunch&, int32_t, int, int, hipStream_t);

}  // namespace gspmd
