// gspmd_ragged_dot (include/gspmd.h): the host's part, and the float32 kernel over experts' packed rows.  How a workgroup finds its tile: ragged.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <vector>

#include "../../include/gspmd.h"
#include "dots.h"
#include "kernels_basic.h"
#include "kernels_f32.h"
#include "kernels_f32_experts.h"
#include "launch.h"
#include "plan.h"
#include "ragged.h"
#include "testing.h"

namespace gspmd {
namespace {

// One product: out[s] = lhs[s] w[expert of s] (rows), or out[e] = lhs[e's rows]^T rhs[e's rows] (contracting).
struct Ragged {
  int64_t E = 0, S = 0, M = 0, N = 0, K = 0;      // experts, slots; extents of an output row block (contracting: M x N a matrix of the output), K of rows
  int64_t es = 0, w_rows = 0;                     // static experts of a shard, rows of an expert's matrix
  bool contracting = false;
  int32_t layout = 0;
};

bool whole(const gspmd_mesh* mesh, const gspmd_sharding* sh, int dim) {
  const int a = sh->dims_mapping[dim];
  return a < 0 || mesh->shape[a] == 1;
}

int32_t analyse(const gspmd_mesh* mesh, const gspmd_dot_dims* dims, const gspmd_sharding* lhs_sh, const gspmd_sharding* rhs_sh, const gspmd_sharding* out_sh, Ragged* g) {
  DotRoles roles;
  int32_t cls[kMaxRank];
  int32_t st = analyse_dot(mesh, dims, lhs_sh, rhs_sh, out_sh, &roles, cls);
  if (st != GSPMD_OK) return st;
  if (lhs_sh->rank != 3 || rhs_sh->rank != 3 || roles.nb != 1 || roles.nc != 1 || roles.lhs_batch[0] != 0 || roles.rhs_batch[0] != 0) return GSPMD_ERR_UNSUPPORTED;
  g->contracting = roles.lhs_contract[0] == 1;
  if (g->contracting && roles.rhs_contract[0] != 1) return GSPMD_ERR_UNSUPPORTED;
  for (int i = 1; i < 3; ++i)
    if (!whole(mesh, lhs_sh, i) || !whole(mesh, rhs_sh, i) || !whole(mesh, out_sh, i)) return GSPMD_ERR_NEEDS_RESHARD;
  g->E = lhs_sh->global_shape[0];
  g->S = lhs_sh->global_shape[1];
  const int64_t features = lhs_sh->global_shape[2];
  if (g->contracting) {
    g->M = features;
    g->N = rhs_sh->global_shape[2];
    g->K = g->S;
    g->w_rows = g->M;
    g->layout = GSPMD_LAYOUT_LHS_K_MAJOR;
  } else {
    const bool transposed = roles.rhs_contract[0] == 2;
    g->M = g->S;
    g->K = features;
    g->N = rhs_sh->global_shape[transposed ? 1 : 2];
    g->w_rows = rhs_sh->global_shape[1];
    g->layout = transposed ? GSPMD_LAYOUT_RHS_K_CONTIGUOUS : 0;
  }
  if (g->E > (1 << 20) || g->S > kMostSlots || std::max(g->M, std::max(g->N, g->K)) > INT32_MAX / 2) return GSPMD_ERR_UNSUPPORTED;
  return GSPMD_OK;
}

// What a kernel is chosen by: rows that spread evenly between half and one and a half times the mean (experts are never liked alike).
std::vector<Problem> likely(const Ragged& g, const Problem& part, int64_t experts, int32_t in_dtype) {
  const int64_t size = in_dtype == GSPMD_BF16 ? 2 : 4;
  const int64_t rows = std::max<int64_t>(1, g.E > 0 ? g.S * std::min(experts, g.E) / g.E : g.S), n = std::max<int64_t>(1, std::min<int64_t>({experts, g.contracting ? experts : rows, 4096}));
  std::vector<Problem> ps(static_cast<size_t>(n), part);
  int64_t at = 0;
  for (int64_t i = 0; i < n; ++i) {
    Problem& p = ps[static_cast<size_t>(i)];
    const double share = n == 1 ? 1.0 : 0.5 + static_cast<double>(i) / static_cast<double>(n - 1);
    const int32_t own = static_cast<int32_t>(std::max<int64_t>(1, static_cast<int64_t>(static_cast<double>(rows) * share / static_cast<double>(n))));
    p.A = static_cast<const char*>(p.A) + at * p.lda * size;
    p.B = static_cast<const char*>(p.B) + (g.contracting ? at * p.ldb : i * g.w_rows * p.ldb) * size;
    if (g.contracting) p.Kv = own;
    else p.Mv = p.Ms = own;
    p.join_count = p.join_first = p.join_slot = 0;
    at += own;
  }
  return ps;
}

template <bool LEAN, bool WIDE>
void launch_f32(const InlineProblems& inl, int n, unsigned tiles, int32_t layout, int32_t epilogue, hipStream_t stream) {
  const dim3 grid(tiles), block(kF32Threads);
  switch (layout) {
    case 0: hipLaunchKernelGGL((dot_f32_kernel<0, LEAN, WIDE, true>), grid, block, 0, stream, table_of<true>(inl), nullptr, n, epilogue); break;
    case 1: hipLaunchKernelGGL((dot_f32_kernel<1, LEAN, WIDE, true>), grid, block, 0, stream, table_of<true>(inl), nullptr, n, epilogue); break;
    default: hipLaunchKernelGGL((dot_f32_kernel<2, LEAN, WIDE, true>), grid, block, 0, stream, table_of<true>(inl), nullptr, n, epilogue);
  }
}

// Whether experts' float32 rows are few enough for dot_f32_experts_kernel (us, dot_f32_kernel / it): K-major matrices 52 experts of 14 rows, 1216 x 4800 311 / 257; 18 of 20, 1024 x 7040 152 / 132; 23 of 29, 416 x 1142
// 17 / 28; K-contiguous ones 27 of 8, 576 x 896 21 / 15; 12 of 12, 576 x 1088 12.6 / 14.6; 18 of 20, 7040 x 1024 202 / 233.
constexpr int64_t kFewF32Rows = 20, kFewF32RowsKContiguous = 10;
bool few_f32_rows(const Ragged& g, const std::vector<Problem>& parts) {
  if (g.contracting || g.E == 0) return false;
  for (const auto& p : parts)
    if (std::max(p.lda, p.ldb) > kF32ExpertsStride) return false;
  const int64_t rows = g.S / std::max<int64_t>(1, std::min(g.E, g.S));       // of an expert that has any
  return rows <= (g.layout & GSPMD_LAYOUT_RHS_K_CONTIGUOUS ? kFewF32RowsKContiguous : kFewF32Rows);
}

int32_t launch_parts(const Ragged& g, std::vector<Problem>& parts, const int32_t* sizes, int32_t first, int32_t last, int32_t in_dtype, int32_t out_dtype, int32_t epilogue, hipStream_t stream) {
  if (parts.empty()) return GSPMD_OK;
  int64_t experts = last - first;
  if (g.contracting) experts = static_cast<int64_t>(parts.size()) * g.es;
  std::vector<Problem> ps;
  for (const auto& part : parts) {              // every part's alignment counts
    auto some = likely(g, part, std::max<int64_t>(1, experts / static_cast<int64_t>(parts.size())), in_dtype);
    ps.insert(ps.end(), some.begin(), some.end());
  }
  DotChoice c = choose_dot(ps, g.layout, in_dtype);
  if (in_dtype == GSPMD_BF16 && c.kernel == GSPMD_TESTING_SCALAR) return GSPMD_ERR_UNSUPPORTED;      // rows beyond 32-bit offsets inside a tile
  if (c.moves_back)
    for (auto& p : parts)
      if ((reinterpret_cast<uintptr_t>(p.B) & 15) || (p.ldb & 7)) p.flags |= kProblemMovesBack;
  const bool few = in_dtype == GSPMD_F32 && few_f32_rows(g, parts);
  if (few) {
    c.bm = kF32ExpertsRows;
    c.bn = kF32ExpertsCols;
  }
  const int64_t tiles_n = (g.N + c.bn - 1) / c.bn;
  const int64_t row_tiles = g.contracting ? experts * ((g.M + c.bm - 1) / c.bm) : g.S / c.bm + std::min(experts, g.S);
  if (row_tiles * tiles_n > INT32_MAX) return GSPMD_ERR_UNSUPPORTED;
  if (launches_are_dry()) return GSPMD_OK;
  InlineProblems inl;
  std::memset(&inl, 0, sizeof(inl));
  std::memcpy(inl.p, parts.data(), parts.size() * sizeof(Problem));
  const int n = static_cast<int>(parts.size());
  RaggedRows r{};
  r.sizes = sizes;
  r.experts = static_cast<int32_t>(g.E);
  r.slots = static_cast<int32_t>(g.S);
  r.first = first;
  r.last = last;
  r.contracting = g.contracting;
  r.rows = static_cast<int32_t>(g.w_rows);
  std::memcpy(&inl.p[kRaggedParts], &r, sizeof(r));
  const unsigned tiles = static_cast<unsigned>(row_tiles * tiles_n);
  if (tiles == 0) return GSPMD_OK;
  MfmaLaunch l{&inl, nullptr, n, static_cast<int>(tiles), epilogue, nullptr, nullptr, nullptr, 0};
  l.past = c.past;
  auto by_layout = [&](auto go) {
    switch (g.layout) {
      case 0: return go(std::integral_constant<int, 0>{});
      case 1: return go(std::integral_constant<int, 1>{});
      default: return go(std::integral_constant<int, 2>{});
    }
  };
  bool ok = true;
  switch (c.kernel) {
    case GSPMD_TESTING_SPLIT: ok = by_layout([&](auto layout) { return launch_ragged_split_layout<decltype(layout)::value>(l, out_dtype, c.row_blocks, c.col_blocks, stream); }); break;
    case GSPMD_TESTING_MID: ok = by_layout([&](auto layout) { return launch_ragged_mid_layout<decltype(layout)::value>(l, out_dtype, c.staged, stream); }); break;
    case GSPMD_TESTING_PAIR: ok = by_layout([&](auto layout) { return launch_ragged_pair_layout<decltype(layout)::value>(l, out_dtype, stream); }); break;
    case GSPMD_TESTING_MFMA: ok = by_layout([&](auto layout) { return launch_ragged_mfma_layout<decltype(layout)::value>(l, out_dtype, stream); }); break;
    default:
      if (few && g.layout == 0) hipLaunchKernelGGL((dot_f32_experts_kernel<0>), dim3(tiles), dim3(256), 0, stream, table_of<true>(inl), n, epilogue);
      else if (few) hipLaunchKernelGGL((dot_f32_experts_kernel<GSPMD_LAYOUT_RHS_K_CONTIGUOUS>), dim3(tiles), dim3(256), 0, stream, table_of<true>(inl), n, epilogue);
      else if (c.f32_wide) launch_f32<false, true>(inl, n, tiles, g.layout, epilogue, stream);
      else if (c.f32_lean) launch_f32<true, false>(inl, n, tiles, g.layout, epilogue, stream);
      else launch_f32<false, false>(inl, n, tiles, g.layout, epilogue, stream);
      ok = hipGetLastError() == hipSuccess;
  }
  return ok ? GSPMD_OK : GSPMD_ERR_DEVICE;
}

// A shard's leading dimension; 0 if the buffer cannot hold it.  `elements`: it has any.
int32_t check(const gspmd_shard_buf& b, int32_t dtype, int64_t cols, bool elements, int32_t* ld) {
  if (b.dtype != dtype) return GSPMD_ERR_UNSUPPORTED;
  if (b.row_stride < 0 || (b.row_stride > 0 && b.row_stride < cols)) return GSPMD_ERR_BAD_BUFFER;
  if (elements && !b.data) return GSPMD_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(b.data) & (dtype == GSPMD_F32 ? 3 : 1)) return GSPMD_ERR_BAD_BUFFER;
  const int64_t stride = b.row_stride > 0 ? b.row_stride : cols;
  if (stride > INT32_MAX) return GSPMD_ERR_UNSUPPORTED;
  *ld = static_cast<int32_t>(stride);
  return GSPMD_OK;
}

}  // namespace
}  // namespace gspmd

using namespace gspmd;

extern "C" {

int32_t gspmd_ragged_dot(const gspmd_mesh* mesh, const gspmd_dot_dims* dims, const gspmd_shard_buf* lhs_shards, const gspmd_sharding* lhs_sh, const gspmd_shard_buf* rhs_shards,
                         const gspmd_sharding* rhs_sh, const gspmd_shard_buf* out_shards, const gspmd_sharding* out_sh, const int32_t* sizes, int32_t epilogue, void* hip_stream) try {
  if (!lhs_shards || !rhs_shards || !out_shards) return GSPMD_ERR_NULL;
  Ragged g;
  int32_t st = analyse(mesh, dims, lhs_sh, rhs_sh, out_sh, &g);
  if (st != GSPMD_OK) return st;
  if (epilogue != GSPMD_EPILOGUE_NONE && epilogue != GSPMD_EPILOGUE_RELU) return GSPMD_ERR_UNSUPPORTED;
  int64_t P = 1;
  for (int i = 0; i < mesh->rank; ++i) P *= mesh->shape[i];
  const int32_t in_dtype = lhs_shards[0].dtype, out_dtype = out_shards[0].dtype;
  if ((in_dtype != GSPMD_F32 && in_dtype != GSPMD_BF16) || (out_dtype != GSPMD_F32 && out_dtype != GSPMD_BF16) || (in_dtype == GSPMD_F32 && out_dtype != GSPMD_F32)) return GSPMD_ERR_UNSUPPORTED;
  const bool nothing = g.E == 0 || g.N == 0 || g.M == 0;           // no element of the output
  const bool lhs_some = g.S > 0 && (g.contracting ? g.M : g.K) > 0, rhs_some = g.contracting ? g.S > 0 && g.N > 0 : g.N > 0 && g.K > 0;
  if (!nothing && !sizes) return GSPMD_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(sizes) & 3) return GSPMD_ERR_BAD_BUFFER;
  struct Part {
    int64_t shard;
    Problem p;
  };
  std::vector<Part> distinct;                   // output buffers, of each shard of the experts those of its own
  const int64_t features = lhs_sh->global_shape[2], rhs_cols = rhs_sh->global_shape[2];
  for (int64_t p = 0; p < P; ++p) {
    Bounds b;
    if ((st = shard_bounds(mesh, out_sh, p, &b)) != GSPMD_OK) return st;
    g.es = b.shard[0];
    Part part{};
    Problem& q = part.p;
    if ((st = check(lhs_shards[p], in_dtype, features, g.E > 0 && lhs_some, &q.lda)) != GSPMD_OK) return st;
    if ((st = check(rhs_shards[p], in_dtype, rhs_cols, g.E > 0 && rhs_some, &q.ldb)) != GSPMD_OK) return st;
    if ((st = check(out_shards[p], out_dtype, g.N, !nothing, &q.ldc)) != GSPMD_OK) return st;
    if (nothing) continue;
    part.shard = b.shard[0] > 0 ? b.offset[0] / b.shard[0] : 0;
    if (b.valid[0] == 0 && !g.contracting) continue;
    if (std::any_of(distinct.begin(), distinct.end(), [&](const Part& d) { return d.shard == part.shard && d.p.C == out_shards[p].data; })) continue;
    q.A = lhs_shards[p].data;
    q.B = rhs_shards[p].data;
    q.C = out_shards[p].data;
    q.Mv = q.Ms = static_cast<int32_t>(g.M);
    q.Nv = q.Ns = static_cast<int32_t>(g.N);
    q.Kv = static_cast<int32_t>(g.K);
    q.join_first = static_cast<int32_t>(b.offset[0]);
    q.join_count = static_cast<int32_t>(b.shard[0]);
    part.p.join_slot = static_cast<int32_t>(b.offset[0] + b.valid[0]);      // (its last expert's successor; not read by the kernels)
    distinct.push_back(part);
  }
  if (distinct.empty()) return GSPMD_OK;
  std::stable_sort(distinct.begin(), distinct.end(), [](const Part& a, const Part& b) { return a.shard < b.shard; });
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  // A launch has up to kRaggedParts parts; of rows each expert once, in order and without gaps.
  std::vector<bool> done(distinct.size(), false);
  for (size_t left = distinct.size(); left > 0;) {
    std::vector<Problem> parts;
    int32_t first = 0, last = 0;
    for (size_t i = 0; i < distinct.size() && parts.size() < static_cast<size_t>(kRaggedParts); ++i) {
      if (done[i]) continue;
      const Problem& q = distinct[i].p;
      if (!g.contracting && !parts.empty() && q.join_first != last) continue;
      if (parts.empty()) first = q.join_first;
      last = q.join_slot;
      parts.push_back(q);
      done[i] = true;
      --left;
    }
    if ((st = launch_parts(g, parts, sizes, first, last, in_dtype, out_dtype, epilogue, stream)) != GSPMD_OK) return st;
  }
  return GSPMD_OK;
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

}  // extern "C"
