// Products grouped by expert whose sizes only the device knows (gspmd_ragged_dot): how a workgroup of a contraction kernel finds its output tile.
//
// The experts' rows ("slots") lie packed, one expert's after the other's.  What a launch's table in the kernel arguments holds is then not the problems themselves but the
// parts of the experts that lie in one buffer each; every wave reads the sizes, a lane an expert, and adds them up: which expert its tile belongs to, where that one's rows begin
// and how many there are.  Against a table of problems made by a launch of its own this costs a wave some 0.7 us before its first load, once, and no launch (4 us) nor search of
// the table (log2 of the experts loads, one after the other).
// Sizes are not trusted: negative ones are 0, and the sum ends at the slots there are, so no value of theirs leads out of the buffers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels_basic.h"
#include "plan.h"
#include "tile_index.h"

namespace gspmd {

constexpr int32_t kMostSlots = 1 << 24;       // 64 sizes of at most so many add up in 32 bits

// Sum over lanes 0 .. this one.
__device__ __forceinline__ int wave_sum_to_here(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);      // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);      // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);      // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast:15 to rows 1, 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // row_bcast:31 to rows 2, 3
  return v;
}

struct RaggedSizes {           // of experts base .. base + 63, this lane's
  int begin, count;            // first slot and how many
  int tiles_to_here, tiles;    // row tiles of the launch's experts among them up to and with this lane's; of all of them
};

// The table in the kernel arguments holds up to kRaggedParts parts -- A, B, C of the first of the part's experts (of packed rows: of slot 0), the leading dimensions, the extents that
// are the same for all experts, and join_first, join_count: the first expert and how many -- and in its last entry's place what is the same for all of them.
struct RaggedRows {
  const int32_t* sizes;        // [experts], device
  int32_t experts, slots;      // slots at most kMostSlots
  int32_t first, last;         // rows of the output ragged: experts that this launch computes, parts in their order, none twice
  int32_t contracting;         // the slots contract: one output block for each of a part's join_count experts; those at `experts` and beyond have no slots
  int32_t rows;                // static rows of an expert's block in the operand or output that is not packed
};
static_assert(sizeof(RaggedRows) <= sizeof(Problem) && sizeof(RaggedRows) % 8 == 0, "");

// A workgroup's tile and the problem that it belongs to.
struct RaggedTile {
  int tile;
  Problem problem;

  // false if there is no tile left for workgroup `block`
  template <int BM, int BN>
  __device__ __forceinline__ bool find(int n_parts, size_t in_size, size_t out_size, int block, int blocks) {
    const int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    const GSPMD_KERNARG Problem* const parts = first_kernel_argument<Problem>();
    const RaggedRows r = copy_from_kernarg((const GSPMD_KERNARG RaggedRows*)(parts + kRaggedParts));
    GSPMD_GLOBAL const int32_t* const of = (GSPMD_GLOBAL const int32_t*)r.sizes;
    Problem& P = problem;
    auto size_of = [&](int e) { return e < r.experts ? min(max(of[e], 0), r.slots) : 0; };
    if (r.contracting) {
      P = copy_from_kernarg(parts);
      const int tiles_n = (P.Nv + BN - 1) / BN, each = ((P.Mv + BM - 1) / BM) * tiles_n;
      tile = logical_tile(block, blocks);
      const int which = tile / each, of_part = P.join_count, part = which / of_part, local = which - part * of_part;
      P = copy_from_kernarg(parts + part);
      const int e = P.join_first + local;
      int begin = 0;
      for (int base = 0; base < min(e, r.experts); base += 64) {
        const int sum = wave_sum_to_here(base + lane < e ? size_of(base + lane) : 0);
        begin = min(begin + __builtin_amdgcn_readlane(sum, 63), r.slots);
      }
      const int count = min(__builtin_amdgcn_readfirstlane(size_of(e)), r.slots - begin);
      P.A = static_cast<const char*>(P.A) + static_cast<int64_t>(begin) * P.lda * in_size;
      P.B = static_cast<const char*>(P.B) + static_cast<int64_t>(begin) * P.ldb * in_size;
      P.C = static_cast<char*>(P.C) + static_cast<int64_t>(local) * r.rows * P.ldc * out_size;
      P.Kv = count;
      P.tile_begin = which * each;
      P.tiles_n = tiles_n;
      P.join_count = 0;
      return true;
    }
    const int tiles_n = (parts->Nv + BN - 1) / BN;
    auto look = [&](int base, int before) {       // `before`: the first of these experts' first slot
      RaggedSizes s;
      const int e = base + lane, size = size_of(e), to_here = wave_sum_to_here(size);
      s.begin = min(before + to_here - size, r.slots);
      s.count = min(before + to_here, r.slots) - s.begin;
      s.tiles_to_here = wave_sum_to_here(e >= r.first && e < r.last ? (s.count + BM - 1) / BM : 0);
      s.tiles = __builtin_amdgcn_readlane(s.tiles_to_here, 63);
      return s;
    };
    auto next_slot = [](const RaggedSizes& s) { return __builtin_amdgcn_readlane(s.begin + s.count, 63); };
    const RaggedSizes lowest = look(0, 0);
    int total = lowest.tiles;
    for (int base = 64, before = next_slot(lowest); base < r.last; base += 64) {
      const RaggedSizes s = look(base, before);
      total += s.tiles;
      before = next_slot(s);
    }
    if (block >= total * tiles_n) return false;
    tile = logical_tile(block, total * tiles_n);
    const int row_tile = tile / tiles_n;
    RaggedSizes s = lowest;
    int base = 0, seen = 0;
    while (row_tile >= seen + s.tiles && base + 64 < r.last) {
      seen += s.tiles;
      base += 64;
      s = look(base, next_slot(s));
    }
    if (row_tile >= seen + s.tiles) return false; // (sizes that have changed meanwhile)
    const int owner = __builtin_ctzll(__builtin_amdgcn_ballot_w64(seen + s.tiles_to_here > row_tile));
    const int e = base + owner, begin = __builtin_amdgcn_readlane(s.begin, owner), count = __builtin_amdgcn_readlane(s.count, owner);
    const int tiles_before = seen + __builtin_amdgcn_readlane(s.tiles_to_here, owner) - (count + BM - 1) / BM;
    static_assert(kRaggedParts <= 64, "a lane for every part");
    const int starts = parts[min(lane, n_parts - 1)].join_first;
    const int part = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < n_parts && starts <= e)) - 1;
    P = copy_from_kernarg(parts + part);
    P.A = static_cast<const char*>(P.A) + static_cast<int64_t>(begin) * P.lda * in_size;
    P.B = static_cast<const char*>(P.B) + static_cast<int64_t>(e - P.join_first) * r.rows * P.ldb * in_size;
    P.C = static_cast<char*>(P.C) + static_cast<int64_t>(begin) * P.ldc * out_size;
    P.Mv = P.Ms = count;
    P.tile_begin = tiles_before * tiles_n;
    P.tiles_n = tiles_n;
    P.join_count = 0;
    return true;
  }
};

}  // namespace gspmd
