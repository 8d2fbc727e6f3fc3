// What the entry points that choose by a token's index share on the host: buffers of a tensor whose dimension 0 is split, by shard and replica.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <vector>

#include "../../include/gspmd.h"
#include "plan.h"

namespace gspmd {

constexpr int64_t kMostGroups = UINT32_MAX / 256;      // workgroups of 256 along one dimension of a launch, whose threads are counted in 32 bits

inline int32_t launched() { return hipGetLastError() == hipSuccess ? GSPMD_OK : GSPMD_ERR_DEVICE; }

// The mesh dimension that splits a tensor's dimension (one of size 1 splits nothing), or -1.
inline int split_axis(const gspmd_mesh* mesh, const gspmd_sharding* sh, int dim) {
  const int a = sh->dims_mapping[dim];
  return a >= 0 && mesh->shape[a] > 1 ? a : -1;
}

// Type, row stride (the same for all of a tensor's shards) and alignment of a shard buffer.
inline int32_t check_rows(const gspmd_shard_buf& b, int32_t dtype, int64_t cols, bool elements, int64_t* ld) {
  if (b.dtype != dtype) return GSPMD_ERR_UNSUPPORTED;
  const int64_t stride = b.row_stride > 0 ? b.row_stride : cols;
  if (b.row_stride < 0 || stride < cols || stride > INT32_MAX) return GSPMD_ERR_BAD_BUFFER;
  if (*ld >= 0 && *ld != stride) return GSPMD_ERR_BAD_BUFFER;
  *ld = stride;
  if (elements && !b.data) return GSPMD_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(b.data) & (dtype == GSPMD_BF16 ? 1 : 3)) return GSPMD_ERR_BAD_BUFFER;
  return GSPMD_OK;
}

// The distinct buffers of every shard: which[r][s] is shard s's r-th one, null where it has fewer.
struct Replicas {
  std::vector<std::vector<void*>> which;
  int64_t shards;
  explicit Replicas(int64_t n) : shards(n) {}
  void add(int64_t shard, void* data) {
    for (auto& level : which) {
      void*& here = level[static_cast<size_t>(shard)];
      if (here == data) return;
      if (here == nullptr) {
        here = data;
        return;
      }
    }
    which.emplace_back(static_cast<size_t>(shards), nullptr);
    which.back()[static_cast<size_t>(shard)] = data;
  }
};

}  // namespace gspmd
