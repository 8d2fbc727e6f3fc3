// Products for other sources: what gspmd.hip launches for lists of strided GEMMs, and sums of fp32 partials.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <vector>

#include "plan.h"

namespace gspmd {

constexpr int64_t kWsAlign = 256;          // of every workspace and of the pieces in it

// All of `ps` (one layout, one pair of types) in one launch; `tables`: device memory of `table_bytes`, kTableBytesPerProblem per problem.
int32_t run_dots(std::vector<Problem>& ps, int32_t layout, int32_t in_dtype, int32_t out_dtype, void* tables, int64_t table_bytes, hipStream_t stream);

// Which kernel a launch of such problems takes (by the rule on their sizes and alignments, or a test's pin), for launches that are made elsewhere.
struct DotChoice {
  int32_t kernel = 0;                      // GSPMD_TESTING_* (testing.h)
  int row_blocks = 0, col_blocks = 0;      // dot_split_kernel
  bool staged = false;                     // dot_mid_kernel: operands through registers
  bool moves_back = false;                 // rhs rows may need kProblemMovesBack
  bool past = false;                       // dot_mid_kernel, dot_pair_kernel: bf16 outputs past all caches
  bool f32_wide = false, f32_lean = false; // dot_f32_kernel's variants
  int bm = 0, bn = 0;                      // its tiles
};
DotChoice choose_dot(const std::vector<Problem>& ps, int32_t layout, int32_t in_dtype);      // (never dot_mfma_kernel through registers)

struct SoftmaxFinish;
// Products of bfloat16 operands that end in `finish` (kernels_stats.h) instead of outputs, for launches that takes_stats() names: those that go to 256 x 256 tiles with direct
// loads anyhow, and with long_outputs those whose outputs rather than products make them go to another kernel.
bool takes_stats(const std::vector<Problem>& ps, int32_t layout, bool long_outputs);
int32_t run_stats(std::vector<Problem>& ps, int32_t layout, const SoftmaxFinish& finish, void* tables, int64_t table_bytes, hipStream_t stream);

// out[r, c] = partials[0][r, c] + partials[1][r, c] + .., ascending, in fp32; any number of partials (all but the first of 16 at a time add to
// partials[0], which is overwritten where there are more than that).
int32_t run_sum(const std::vector<float*>& partials, int64_t rows, int64_t cols, int64_t ld_in, void* out, int64_t ld_out, int32_t out_dtype, hipStream_t stream);

// A test has pinned this thread's calls to end before their launches (testing.h).
bool launches_are_dry();
// A test has pinned the kernel of this thread's products: there have to be some.
bool a_product_is_pinned();

}  // namespace gspmd
