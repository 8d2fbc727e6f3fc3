// Logits that are not kept: dot_mfma_kernel's tiles reduced, where their accumulators are, to what a softmax needs of them -- of each row of a wave's 64 columns the
// maximum and the sum of exp(z - maximum) -- and to the logits of the tokens' targets.  512 bytes of a tile row of 256 logits become 32.
// The K loop bounds it as ever; a tile's end takes 128 exponentials a lane in place of 256 KiB of stores.  Measured: 16384 x 2048 x 32000 1.62 ms with all of the call (1.32 PFLOP/s); 1024 x 1024 x
// 128000 277 us, 35 us a round of tiles of which the K loop is 26, with 100 targets a token 314; 1024 x 64 x 128000 12 us a round, what a tile costs beside its K loop.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mfma_common.h"
#include "plan.h"
#include "tile_index.h"

namespace gspmd {

// What the launch's problems stand for: join_first is the problem's first row among the piece's, join_slot the column of a row of logits where its columns start (a multiple of
// 64); C the table of pairs [column / 64][row], ldc its rows.
struct SoftmaxFinish {
  const int32_t* columns;        // [rows][targets]: the target's column in a row of logits; what is none is no target
  float* logits;                 // [rows][targets], out
  int32_t targets;
  float c;                       // log2(e) / tau

  // Targets that a thread has in registers: the next ones are on their way while what is found among these is stored (1024 tokens of 100 targets, 1024 x 128000: a load and a barrier after the
  // other, eight at a time, 393 us; 32 held 328; 56, all of a tile's 25600 at once, 314; more than 112 targets a token take a second round).
  static constexpr int kHeld = 56, kAtOnce = kHeld * 512;

  __device__ __forceinline__ void operator()(float16_t (&acc)[8], const Problem& P, TileRows own, int n0, unsigned char* smem) const {
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), wm = wave >> 2, wn = wave & 3;
    const int quad = lane >> 4, r16 = lane & 15, col0 = n0 + wn * 64, first = P.join_first + own.first;
    typedef __attribute__((ext_vector_type(2))) float float2_t;
    GSPMD_GLOBAL const int32_t* const mine = (GSPMD_GLOBAL const int32_t*)columns + static_cast<int64_t>(first) * targets;
    const int total = own.rows * targets, tile_col = P.join_slot + n0, cols = min(P.Nv - n0, 256);
    int held[kHeld];
    auto fetch = [&](int from) {
#pragma unroll
      for (int n = 0; n < kHeld; ++n) {
        const int i = from + n * 512 + t;
        held[n] = -1;
        if (i < total) held[n] = mine[i];
      }
    };
    fetch(0);
    // ---- maximum and sum.  A lane holds 16 of a row's 64 columns, the four lanes beside it in steps of 16 the others.
    if (col0 < P.Nv) {
      GSPMD_GLOBAL float2_t* const out = (GSPMD_GLOBAL float2_t*)P.C + static_cast<int64_t>((P.join_slot + col0) >> 6) * P.ldc + first;
      const bool inside = col0 + 64 <= P.Nv;
#pragma unroll
      for (int bm = 0; bm < 8; ++bm) {
        float v[16], m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          v[e] = acc[bm][e];
          if (!inside && col0 + (e >> 2) * 16 + quad * 4 + (e & 3) >= P.Nv) v[e] = -INFINITY;
          m = fmaxf(m, v[e]);
        }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f((v[e] - from) * c);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        const int row = wm * 128 + bm * 16 + r16;
        if (quad == 0 && row < own.rows) out[row] = float2_t{m, sum};
      }
    }
    // ---- the targets in this tile: found by all threads, a list of them in LDS, each stored by the lane that holds it
    uint32_t* const count = reinterpret_cast<uint32_t*>(smem);
    uint32_t* const list = reinterpret_cast<uint32_t*>(smem + 64);
    for (int from = 0; from < total; from += kAtOnce) {
      __syncthreads();                           // every wave's LDS reads are over: the last tile's fragments, the list before
      if (t == 0) *count = 0;
      __syncthreads();
#pragma unroll
      for (int n = 0; n < kHeld; ++n) {
        if (from + n * 512 >= total) break;
        const int col = held[n] - tile_col;      // (of no target far below 0)
        if (static_cast<uint32_t>(col) >= static_cast<uint32_t>(cols)) continue;
        const int i = from + n * 512 + t, row = i / targets;
        list[atomicAdd(count, 1u)] = static_cast<uint32_t>(row | col << 8 | (i - row * targets) << 16);
      }
      fetch(from + kAtOnce);
      __syncthreads();
      const int found = __builtin_amdgcn_readfirstlane(*count);
      for (int h = 0; h < found; h += 64) {
        const uint32_t here = h + lane < found ? list[h + lane] : 0u;
        for (uint64_t left = __builtin_amdgcn_ballot_w64(h + lane < found && ((here >> 7) & 1) == static_cast<uint32_t>(wm) && ((here >> 14) & 3) == static_cast<uint32_t>(wn)); left != 0;
             left &= left - 1) {                 // those of this wave
          const uint32_t entry = __builtin_amdgcn_readlane(here, __builtin_ctzll(left));
          const int row = entry & 255, col = (entry >> 8) & 255, k = entry >> 16, bm_of = (row >> 4) & 7, e_of = ((col >> 4) & 3) * 4 + (col & 3);
          float v = 0.f;
#pragma unroll
          for (int bm = 0; bm < 8; ++bm)
            if (bm == bm_of)
#pragma unroll
              for (int e = 0; e < 16; ++e)
                if (e == e_of) v = acc[bm][e];
          if (lane == ((col >> 2) & 3) * 16 + (row & 15)) ((GSPMD_GLOBAL float*)logits)[static_cast<int64_t>(first + row) * targets + k] = v;
        }
      }
    }
  }
};

}  // namespace gspmd
