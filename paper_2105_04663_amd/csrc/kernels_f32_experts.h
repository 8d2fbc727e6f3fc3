// float32 products of experts' packed rows (ragged.h) of a few rows each, which leave dot_f32_kernel's tiles of 64 x 64 mostly empty: 16 x 64 a workgroup.
//
// Operands go from memory into registers, where v_mfma_f32_16x16x4_f32 takes them as they lie, 16 bytes a lane along whatever is contiguous.  A K-contiguous operand gives a lane four k of a row, one for
// each of four MFMAs; a K-major one four neighbouring columns of a k, one for each of four blocks of sixteen, whose columns are then every fourth.  No LDS and no barrier in the loop: each of the four waves has 16
// of every 64 k, kF32ExpertsAhead such steps on their way, and their sums meet in LDS once, in the order of the waves.  Sums are folded by 32 products, as dot_f32_kernel's by 96
// or 64 (relative to float64, rows of 2240 1.4e-7, of 4096 1.5e-7).
// Bound by the matrices, read once where an expert has up to 16 rows (us, dot_f32_kernel / this: 35 experts of 3 rows, 3378 x 2950 286 / 247; 77 of
// 1.5, 320 x 4096 60 / 41; 5 of 6, 1024 x 640 18.4 / 10.2).  Two steps ahead and four workgroups on a compute unit: with four and three 45 for the second, 6 and two 50.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels_basic.h"
#include "kernels_f32.h"
#include "mfma_common.h"
#include "plan.h"
#include "ragged.h"

namespace gspmd {

constexpr int kF32ExpertsRows = 16, kF32ExpertsCols = 64, kF32ExpertsStep = 16, kF32ExpertsAhead = 2;
constexpr int64_t kF32ExpertsStride = 1 << 23;           // elements: a tile's rows stay within 32-bit offsets (of bytes)

template <int LAYOUT>
__global__ __launch_bounds__(256, 4) void dot_f32_experts_kernel(const RaggedParts inl, int n_prob, int epilogue) {
  constexpr bool BKC = (LAYOUT & GSPMD_LAYOUT_RHS_K_CONTIGUOUS) != 0;
  static_assert(!(LAYOUT & GSPMD_LAYOUT_LHS_K_MAJOR), "experts' rows");
  typedef GSPMD_GLOBAL const float* gfloats;
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  RaggedTile ragged;
  if (!ragged.find<kF32ExpertsRows, kF32ExpertsCols>(n_prob, sizeof(float), sizeof(float), blockIdx.x, gridDim.x)) return;
  const Problem P = ragged.problem;
  // the row index runs fastest: tiles that are in flight together share the matrix
  const int local = ragged.tile - P.tile_begin, tiles_m = (P.Mv + kF32ExpertsRows - 1) / kF32ExpertsRows;
  const int m0 = local % tiles_m * kF32ExpertsRows, n0 = local / tiles_m * kF32ExpertsCols;
  // A lane's bytes from a tile's first row (K-contiguous) or the step's first k (K-major) on.  Rows and columns beyond the valid ones are the last ones: what they give is not stored.
  const gfloats A = (gfloats)P.A, B = (gfloats)P.B;
  const bool whole = BKC || n0 + kF32ExpertsCols <= P.Nv;          // (columns in chunks of four that are all there)
  auto row_offset = [&](int first, int block, int valid, int64_t ld) { return static_cast<uint32_t>(min(16 * block + l16, valid - 1 - first) * ld + 4 * g) * 4u; };
  const uint32_t a_off = row_offset(m0, 0, P.Mv, P.lda);
  uint32_t b_off[BKC ? 4 : 1];
  if constexpr (BKC) {
#pragma unroll
    for (int i = 0; i < 4; ++i) b_off[i] = row_offset(n0, i, P.Nv, P.ldb);
  } else {
    b_off[0] = static_cast<uint32_t>(4 * g * static_cast<int64_t>(P.ldb)) * 4u;
  }
  auto four = [&](gfloats base, uint32_t off) -> f32x4 { return *(GSPMD_GLOBAL const f32x4_any*)((GSPMD_GLOBAL const char*)base + off); };
  struct Step {
    f32x4 a, b[4];                              // b: by block (K-contiguous) or by k
  };
  auto load = [&](Step& s, int k) {             // k .. k + 15 are there
    s.a = four(A + static_cast<int64_t>(m0) * P.lda + k, a_off);
    const gfloats at = BKC ? B + static_cast<int64_t>(n0) * P.ldb + k : B + static_cast<int64_t>(k) * P.ldb;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BKC) {
        s.b[i] = four(at, b_off[i]);
      } else {
        const gfloats row = at + i * static_cast<int64_t>(P.ldb);
        if (whole) {
          s.b[i] = four(row, b_off[0] + static_cast<uint32_t>(n0 + 4 * l16) * 4u);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) s.b[i][e] = *(gfloats)((GSPMD_GLOBAL const char*)row + b_off[0] + static_cast<uint32_t>(min(n0 + 4 * l16 + e, P.Nv - 1)) * 4u);
        }
      }
    }
  };
  auto load_last = [&](Step& s, int k) {        // what is left of K, zeros beyond in both operands
    auto element = [&](gfloats base, int64_t ld, bool kmajor, int x, int at) { return base[kmajor ? min(at, P.Kv - 1) * ld + x : x * ld + min(at, P.Kv - 1)]; };
    const int m = min(m0 + l16, P.Mv - 1);
#pragma unroll
    for (int e = 0; e < 4; ++e) s.a[e] = element(A, P.lda, false, m, k + 4 * g + e);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s.b[i][e] = BKC ? element(B, P.ldb, false, min(n0 + 16 * i + l16, P.Nv - 1), k + 4 * g + e) : element(B, P.ldb, true, min(n0 + 4 * l16 + e, P.Nv - 1), k + 4 * g + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s.a[e] = k + 4 * g + e < P.Kv ? s.a[e] : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) s.b[i][e] = k + 4 * g + (BKC ? e : i) < P.Kv ? s.b[i][e] : 0.f;
    }
  };
  f32x4 acc[4], sum[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = sum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const Step& s) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(BKC ? s.b[j][k] : s.b[k][j], s.a[k], acc[j], 0, 0, 0);
  };
  auto fold = [&] {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sum[j] += acc[j];
      acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  const int steps = P.Kv / kF32ExpertsStep, mine = (steps + 3 - wave) / 4, first = wave * kF32ExpertsStep;        // this wave's whole steps, its first k
  if (mine > 0) {
    Step s[kF32ExpertsAhead];
    auto k_of = [&](int i) { return first + min(i, mine - 1) * 4 * kF32ExpertsStep; };     // (beyond the last: the last again, not used)
#pragma unroll
    for (int d = 0; d < kF32ExpertsAhead; ++d) load(s[d], k_of(d));
#pragma unroll 1
    for (int i = 0; i < mine; i += kF32ExpertsAhead) {
#pragma unroll
      for (int d = 0; d < kF32ExpertsAhead; ++d) {
        if (i + d < mine) multiply(s[d]);
        load(s[d], k_of(i + d + kF32ExpertsAhead));
      }
      fold();                                   // (32 products)
    }
  }
  if (steps * kF32ExpertsStep < P.Kv && wave == (steps & 3)) {
    Step s;
    load_last(s, steps * kF32ExpertsStep);
    multiply(s);
    fold();
  }
  // Four neighbouring columns a store, a wave a quarter of them: with a K-major rhs those of the four blocks, else four results of one.
  __shared__ float parts[4][4][4][64];          // [wave][group of columns][column][lane]
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int e = 0; e < 4; ++e) parts[wave][q][e][lane] = BKC ? sum[q][e] : sum[e][q];
  __syncthreads();
  const int m = m0 + l16, n = BKC ? n0 + 16 * wave + 4 * g : n0 + 16 * g + 4 * wave;
  if (m >= P.Mv) return;
  f32x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = apply_epilogue(((parts[0][wave][e][lane] + parts[1][wave][e][lane]) + parts[2][wave][e][lane]) + parts[3][wave][e][lane], epilogue);
  GSPMD_GLOBAL float* const c = (GSPMD_GLOBAL float*)P.C + static_cast<int64_t>(m) * P.ldc + n;
  if (n + 4 <= P.Nv) *(GSPMD_GLOBAL f32x4_any*)c = o;
  else
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < P.Nv) c[e] = o[e];
}

}  // namespace gspmd
