// The host's side of kernels_sort.h: workspace and launches.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "dots.h"
#include "plan.h"

namespace gspmd {

struct SortKeys;
struct SortOut;
// Bytes of workspace to sort `count` keys below `keys` (0 where one workgroup does).
int64_t sort_bytes(int64_t count, int64_t keys);
// `workspace`: kWsAlign-aligned.  A routing (out.sizes) has keys of one digit.
int32_t run_sort(const SortKeys& in, const SortOut& out, void* workspace, hipStream_t stream);

}  // namespace gspmd
