// Losses over a split vocabulary (include/gspmd.h: gspmd_softmax_xent, gspmd_softmax_distill).
//
// The logits of a piece of tokens (some rows of every token shard, all of the vocabulary) go to the workspace as float32, one product per pair of token shard and vocabulary
// shard; softmax_rows_kernel makes of each row the token's loss and, in place, D, the gradient with respect to the logits; two more products make of D the piece's rows of dx
// and its share of dw.  Sums over shards (dx over the vocabulary's, dw over the tokens') and over pieces (dw) are float32 partials, added up in ascending order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <map>
#include <vector>

#include "../../include/gspmd.h"
#include "dots.h"
#include "kernels_softmax.h"
#include "plan.h"

namespace gspmd {
namespace {

// Logits of a piece, at most (float32; at least one row of every token shard): what the workspace query provides for.
constexpr int64_t kPieceBytes = int64_t(1) << 30;
constexpr int64_t kColumnAlign = 64;

struct Loss {
  const gspmd_mesh* mesh = nullptr;
  int64_t P = 0;
  int64_t T = 0, M = 0, V = 0;               // global extents
  int64_t na = 1, nb = 1, ts = 0, vs = 0;    // shards of the tokens and of the vocabulary, and their static extents
  int axis_t = -1, axis_v = -1;              // mesh dimensions; -1: not split
  int vocab_dim = 0;
  int32_t dtype = 0;
  bool dx = false, dw = false;
  int64_t esize() const { return dtype == GSPMD_BF16 ? 2 : 4; }
  int64_t valid_t(int64_t i) const { return std::max<int64_t>(0, std::min(ts, T - i * ts)); }
  int64_t valid_v(int64_t j) const { return std::max<int64_t>(0, std::min(vs, V - j * vs)); }
  // logits: the vocabulary shards that hold any entry, one after the other
  int64_t shards_v() const { return vs > 0 ? (V + vs - 1) / vs : 0; }
  int64_t per_cols() const { return round_up(std::max<int64_t>(vs, 1), kColumnAlign); }
  int64_t ldz() const { return std::max<int64_t>(shards_v(), 1) * per_cols(); }
  int64_t dw_rows() const { return vocab_dim == 0 ? vs : M; }
  int64_t dw_cols() const { return vocab_dim == 0 ? M : vs; }
  // fp32 partials: dx of each vocabulary shard, dw of each token shard and (several pieces) of the pieces before
  bool parts_dx() const { return dx && nb > 1; }
  int64_t dw_partials(bool pieces) const { return dw && (na > 1 || pieces) ? na + (pieces ? 1 : 0) : 0; }
  int64_t row_bytes() const {                // workspace per row of a token shard
    return na * (ldz() * 4 + (parts_dx() ? nb * round_up(M, 4) * 4 : 0));
  }
  int64_t dw_bytes(bool pieces) const { return dw_partials(pieces) * nb * round_up(dw_rows() * round_up(dw_cols(), 4) * 4, kWsAlign); }
  int64_t table_bytes() const { return round_up((na * nb * 2 + 1) * kTableBytesPerProblem, kWsAlign); }
  int64_t fixed_bytes(bool pieces) const { return table_bytes() + dw_bytes(pieces) + 4 * kWsAlign; }
  int64_t whole_rows() const { return std::min<int64_t>(ts, std::max<int64_t>(T, 0)); }
};

// Shapes, shardings and the extents that follow from them.
int32_t analyse(const gspmd_mesh* mesh, const gspmd_sharding* x_sh, const gspmd_sharding* w_sh, int32_t vocab_dim, Loss* l) {
  int32_t st = validate_mesh(mesh, &l->P);
  if (st != GSPMD_OK) return st;
  if ((st = validate_sharding(mesh, x_sh)) != GSPMD_OK || (st = validate_sharding(mesh, w_sh)) != GSPMD_OK) return st;
  if (x_sh->rank != 2 || w_sh->rank != 2 || (vocab_dim != 0 && vocab_dim != 1)) return GSPMD_ERR_BAD_DOT_DIMS;
  l->mesh = mesh;
  l->vocab_dim = vocab_dim;
  l->T = x_sh->global_shape[0];
  l->M = x_sh->global_shape[1];
  l->V = w_sh->global_shape[vocab_dim];
  if (w_sh->global_shape[1 - vocab_dim] != l->M || l->V < 1) return GSPMD_ERR_BAD_DOT_DIMS;
  auto axis = [&](const gspmd_sharding* sh, int dim) {       // a mesh dimension of size 1 splits nothing
    const int a = sh->dims_mapping[dim];
    return a >= 0 && mesh->shape[a] > 1 ? a : -1;
  };
  if (axis(x_sh, 1) >= 0 || axis(w_sh, 1 - vocab_dim) >= 0) return GSPMD_ERR_NEEDS_RESHARD;
  l->axis_t = axis(x_sh, 0);
  l->axis_v = axis(w_sh, vocab_dim);
  if (l->axis_t >= 0 && l->axis_t == l->axis_v) return GSPMD_ERR_NEEDS_RESHARD;
  l->na = l->axis_t >= 0 ? mesh->shape[l->axis_t] : 1;
  l->nb = l->axis_v >= 0 ? mesh->shape[l->axis_v] : 1;
  l->ts = (l->T + l->na - 1) / l->na;
  l->vs = (l->V + l->nb - 1) / l->nb;
  constexpr int64_t kMost = INT32_MAX >> 2;                  // of a padded row of logits as of every extent
  if (l->T > kMost || l->M > kMost || l->ldz() > kMost || l->na * l->nb > kMaxProblems / 2) return GSPMD_ERR_UNSUPPORTED;
  return GSPMD_OK;
}

struct Buffers {                             // the distinct ones of one position, the first of which is computed into
  gspmd_shard_buf first;
  std::vector<gspmd_shard_buf> others;
};

int32_t add_buffer(std::vector<Buffers>& at, int64_t pos, bool seen, const gspmd_shard_buf& b) {
  Buffers& here = at[static_cast<size_t>(pos)];
  if (!seen) {
    here.first = b;
    return GSPMD_OK;
  }
  if (b.data == here.first.data) return b.row_stride == here.first.row_stride ? GSPMD_OK : GSPMD_ERR_BAD_BUFFER;
  for (const auto& o : here.others) if (o.data == b.data) return GSPMD_OK;
  here.others.push_back(b);
  return GSPMD_OK;
}

// A shard's row stride in elements, or -1.
int64_t stride_of(const gspmd_shard_buf& b, int64_t cols) {
  const int64_t ld = b.row_stride > 0 ? b.row_stride : cols;
  return ld < cols || ld > INT32_MAX ? -1 : std::max<int64_t>(ld, 1);
}

// A group of products that add up to one output block.
struct Sum {
  std::vector<Problem> members;              // same valid output extents where they have any K; C is set by run_sums
  void* out;
  int32_t ld_out, rows, cols;                // static extents
  float* earlier = nullptr;                  // what pieces before have added up (dense, ld of the partials), and goes on in
  float* partials = nullptr;                 // room for the members, ld of the partials
};

int32_t run_sums(std::vector<Sum>& sums, int32_t layout, int32_t dtype, bool first, bool last, void* tables, int64_t table_bytes, hipStream_t stream) {
  std::vector<Problem> launch;
  size_t most = 0;
  for (auto& s : sums) most = std::max(most, static_cast<size_t>(std::count_if(s.members.begin(), s.members.end(), [](const Problem& p) { return p.Kv > 0; })));
  const bool direct = most <= 1 && first && last;
  auto add = [&](Problem p, void* c, int64_t ldc, const Sum& s) {
    p.C = c;
    p.ldc = static_cast<int32_t>(ldc);
    p.Ms = s.rows;
    p.Ns = s.cols;
    if (p.Mv == 0 || p.Nv == 0 || p.Kv == 0) p.Mv = p.Nv = p.Kv = 0;
    launch.push_back(p);
  };
  for (auto& s : sums) {
    std::stable_partition(s.members.begin(), s.members.end(), [](const Problem& p) { return p.Kv > 0; });
    const int64_t ld = round_up(s.cols, 4), size = static_cast<int64_t>(s.rows) * ld;
    if (direct) {
      add(s.members[0], s.out, s.ld_out, s);
    } else {
      for (size_t m = 0; m < s.members.size(); ++m)
        if (m == 0 || s.members[m].Kv > 0) add(s.members[m], s.partials + static_cast<int64_t>(m) * size, ld, s);
    }
  }
  int32_t st = run_dots(launch, layout, dtype, direct ? dtype : static_cast<int32_t>(GSPMD_F32), tables, table_bytes, stream);
  if (st != GSPMD_OK || direct) return st;
  for (auto& s : sums) {
    const int64_t ld = round_up(s.cols, 4), size = static_cast<int64_t>(s.rows) * ld;
    std::vector<float*> parts;
    if (!first) parts.push_back(s.earlier);
    for (size_t m = 0; m < s.members.size(); ++m)
      if (m == 0 || s.members[m].Kv > 0) parts.push_back(s.partials + static_cast<int64_t>(m) * size);
    if ((st = run_sum(parts, s.rows, s.cols, ld, last ? s.out : s.earlier, last ? s.ld_out : ld, last ? dtype : static_cast<int32_t>(GSPMD_F32), stream)) != GSPMD_OK) return st;
  }
  return GSPMD_OK;
}

template <typename T, bool GRAD>
void launch_rows_as(const SoftmaxRows& a, unsigned rows, hipStream_t stream) {
  const size_t lds = static_cast<size_t>(a.targets) * 12;
  if (a.cols <= 64 * 4 * 4) hipLaunchKernelGGL((softmax_rows_kernel<T, 64, 4, false, GRAD>), dim3(rows), dim3(64), lds, stream, a);
  else if (a.cols <= 256 * 4 * 8) hipLaunchKernelGGL((softmax_rows_kernel<T, 256, 8, false, GRAD>), dim3(rows), dim3(256), lds, stream, a);
  else if (a.cols <= 1024 * 4 * 8) hipLaunchKernelGGL((softmax_rows_kernel<T, 1024, 8, false, GRAD>), dim3(rows), dim3(1024), lds, stream, a);
  else if (a.cols <= 1024 * 4 * 12) hipLaunchKernelGGL((softmax_rows_kernel<T, 1024, 12, false, GRAD>), dim3(rows), dim3(1024), lds, stream, a);
  else hipLaunchKernelGGL((softmax_rows_kernel<T, 1024, 8, true, GRAD>), dim3(rows), dim3(1024), lds, stream, a);
}

int32_t copy_rows(const gspmd_shard_buf& from, const gspmd_shard_buf& to, int64_t rows, int64_t cols, int64_t ld_from, int64_t ld_to, hipStream_t stream) {
  if (rows == 0 || cols == 0) return GSPMD_OK;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((cols + 255) / 256, 64)), static_cast<unsigned>(std::min<int64_t>(rows, 4096)));
  if (from.dtype == GSPMD_BF16) hipLaunchKernelGGL((copy_rows_kernel<uint16_t>), grid, dim3(256), 0, stream, static_cast<const uint16_t*>(from.data), static_cast<uint16_t*>(to.data), rows, cols, ld_from, ld_to);
  else hipLaunchKernelGGL((copy_rows_kernel<uint32_t>), grid, dim3(256), 0, stream, static_cast<const uint32_t*>(from.data), static_cast<uint32_t*>(to.data), rows, cols, ld_from, ld_to);
  return hipGetLastError() == hipSuccess ? GSPMD_OK : GSPMD_ERR_DEVICE;
}

int32_t check_shard(const gspmd_shard_buf& b, int32_t dtype, int64_t rows, int64_t cols) {
  if (b.dtype != dtype) return GSPMD_ERR_UNSUPPORTED;
  if (b.row_stride < 0 || stride_of(b, cols) < 0) return GSPMD_ERR_BAD_BUFFER;
  if (!b.data && rows > 0 && cols > 0) return GSPMD_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(b.data) & (dtype == GSPMD_BF16 ? 1 : 3)) return GSPMD_ERR_BAD_BUFFER;
  return GSPMD_OK;
}

int32_t run_loss(const gspmd_mesh* mesh, const gspmd_shard_buf* x_shards, const gspmd_sharding* x_sh, const gspmd_shard_buf* w_shards, const gspmd_sharding* w_sh, int32_t vocab_dim,
                 const gspmd_token_buf* tokens, int32_t targets, float tau, bool teacher, const gspmd_shard_buf* dx_shards, const gspmd_shard_buf* dw_shards, void* workspace,
                 int64_t workspace_bytes, void* hip_stream) {
  Loss l;
  int32_t st = analyse(mesh, x_sh, w_sh, vocab_dim, &l);
  if (st != GSPMD_OK) return st;
  if (!x_shards || !w_shards || !tokens) return GSPMD_ERR_NULL;
  if (targets < 1 || targets > GSPMD_MAX_TARGETS) return GSPMD_ERR_UNSUPPORTED;
  if (!(tau > 0.f) || !std::isfinite(tau) || !std::isfinite(1.f / tau)) return GSPMD_ERR_UNSUPPORTED;
  l.dtype = x_shards[0].dtype;
  if (l.dtype != GSPMD_BF16 && l.dtype != GSPMD_F32) return GSPMD_ERR_UNSUPPORTED;
  l.dx = dx_shards != nullptr;
  l.dw = dw_shards != nullptr;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);

  // what each position along the two mesh dimensions has; of partitions that hold the same data the first in mesh order is read
  std::vector<Buffers> x(static_cast<size_t>(l.na)), w(static_cast<size_t>(l.nb)), dx(x), dw(w);
  std::vector<std::vector<gspmd_token_buf>> token(static_cast<size_t>(l.na));
  std::vector<char> seen_t(static_cast<size_t>(l.na), 0), seen_v(static_cast<size_t>(l.nb), 0);
  const int64_t w_rows = l.dw_rows(), w_cols = l.dw_cols();
  for (int64_t at = 0; at < l.P; ++at) {
    const int64_t p = mesh->device_ids[at];
    int64_t coords[kMaxRank];
    if ((st = mesh_coords(mesh, p, coords)) != GSPMD_OK) return st;
    const int64_t i = l.axis_t >= 0 ? coords[l.axis_t] : 0, j = l.axis_v >= 0 ? coords[l.axis_v] : 0;
    if ((st = check_shard(x_shards[p], l.dtype, l.ts, l.M)) != GSPMD_OK || (st = check_shard(w_shards[p], l.dtype, w_rows, w_cols)) != GSPMD_OK) return st;
    if (l.dx && (st = check_shard(dx_shards[p], l.dtype, l.ts, l.M)) != GSPMD_OK) return st;
    if (l.dw && (st = check_shard(dw_shards[p], l.dtype, w_rows, w_cols)) != GSPMD_OK) return st;
    const gspmd_token_buf& tb = tokens[p];
    if (l.ts > 0 && (!tb.ids || !tb.loss || (teacher && !tb.logits))) return GSPMD_ERR_NULL;
    if (teacher && tb.logits_dtype != GSPMD_F32 && tb.logits_dtype != GSPMD_BF16) return GSPMD_ERR_UNSUPPORTED;
    if (teacher && tb.logits_dtype != tokens[0].logits_dtype) return GSPMD_ERR_UNSUPPORTED;
    const bool ts = seen_t[static_cast<size_t>(i)], vs = seen_v[static_cast<size_t>(j)];
    if (!ts) x[static_cast<size_t>(i)].first = x_shards[p];
    if (!vs) w[static_cast<size_t>(j)].first = w_shards[p];
    if (l.dx && (st = add_buffer(dx, i, ts, dx_shards[p])) != GSPMD_OK) return st;
    if (l.dw && (st = add_buffer(dw, j, vs, dw_shards[p])) != GSPMD_OK) return st;
    auto& mine = token[static_cast<size_t>(i)];
    const bool known = std::any_of(mine.begin(), mine.end(), [&](const gspmd_token_buf& o) { return o.loss == tb.loss && o.lse == tb.lse; });
    if (!known) mine.push_back(tb);
    seen_t[static_cast<size_t>(i)] = seen_v[static_cast<size_t>(j)] = 1;
  }

  // (the first of a shard's is what the kernel writes: one with an lse, if any has)
  for (auto& list : token) std::stable_partition(list.begin(), list.end(), [](const gspmd_token_buf& tb) { return tb.lse != nullptr; });

  // ---- pieces: as many rows of every token shard as the workspace holds
  const int64_t whole = l.whole_rows();
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & (kWsAlign - 1))) return GSPMD_ERR_WORKSPACE;
  const int64_t in_piece = std::max<int64_t>(1, kPieceBytes / (l.na * l.ldz() * 4));       // (more workspace than the query asks for is not used)
  int64_t rows = std::min(whole, in_piece);
  if (l.fixed_bytes(rows < whole) + rows * l.row_bytes() > workspace_bytes)
    rows = std::min(rows, (workspace_bytes - l.fixed_bytes(true)) / l.row_bytes());
  if (whole > 0 && rows < 1) return GSPMD_ERR_WORKSPACE;
  if (l.fixed_bytes(false) > workspace_bytes) return GSPMD_ERR_WORKSPACE;
  int64_t pieces = whole > 0 ? (whole + rows - 1) / rows : 1;
  if (pieces > 1) {                           // even ones, in whole tiles where that does not make more of them
    rows = (whole + pieces - 1) / pieces;
    const int64_t up = round_up(rows, 256);
    if (l.fixed_bytes(true) + up * l.row_bytes() <= workspace_bytes && up <= in_piece) rows = up;
    pieces = (whole + rows - 1) / rows;
  }
  char* ws = static_cast<char*>(workspace);
  auto take = [&](int64_t bytes) {
    char* at = ws;
    ws += round_up(bytes, kWsAlign);
    return at;
  };
  void* const tables = take(l.table_bytes());
  const int64_t ldz = l.ldz(), per_cols = l.per_cols(), zs = l.shards_v();
  const int64_t dw_size = round_up(w_rows * round_up(w_cols, 4) * 4, kWsAlign) / 4;          // float32 elements of a partial
  float* const dw_parts = reinterpret_cast<float*>(take(l.dw_bytes(pieces > 1)));
  float* const z = reinterpret_cast<float*>(take(l.na * rows * ldz * 4));
  float* const dx_parts = l.parts_dx() ? reinterpret_cast<float*>(take(l.na * rows * l.nb * round_up(l.M, 4) * 4)) : nullptr;
  const int64_t e = l.esize(), ldd = ldz * 4 / e;
  const bool grad = l.dx || l.dw;

  for (int64_t piece = 0; piece < pieces; ++piece) {
    const int64_t first = piece * rows, held = std::min(rows, std::max<int64_t>(l.ts - first, 0));
    auto valid = [&](int64_t i) { return std::max<int64_t>(0, std::min(rows, l.valid_t(i) - first)); };
    auto z_at = [&](int64_t i, int64_t j, int64_t size) { return reinterpret_cast<char*>(z + i * rows * ldz) + j * per_cols * size; };
    auto x_at = [&](int64_t i) { return static_cast<char*>(x[static_cast<size_t>(i)].first.data) + first * stride_of(x[static_cast<size_t>(i)].first, l.M) * e; };
    auto problem = [](const void* a, int64_t lda, const void* b, int64_t ldb, int64_t m, int64_t n, int64_t k) {
      Problem p;
      std::memset(&p, 0, sizeof(p));
      p.A = a;
      p.B = b;
      p.lda = static_cast<int32_t>(lda);
      p.ldb = static_cast<int32_t>(ldb);
      p.Mv = static_cast<int32_t>(m);
      p.Nv = static_cast<int32_t>(n);
      p.Kv = static_cast<int32_t>(k);
      return p;
    };
    // ---- logits
    std::vector<Problem> ps;
    for (int64_t i = 0; i < l.na; ++i)
      for (int64_t j = 0; j < zs; ++j) {
        const gspmd_shard_buf &xb = x[static_cast<size_t>(i)].first, &wb = w[static_cast<size_t>(j)].first;
        Problem p = problem(x_at(i), stride_of(xb, l.M), wb.data, stride_of(wb, w_cols), valid(i), l.valid_v(j), l.M);
        p.C = z_at(i, j, 4);
        p.ldc = static_cast<int32_t>(ldz);
        p.Ms = p.Mv;
        p.Ns = p.Nv;
        if (p.Kv == 0) p.Mv = p.Nv = 0;       // no hidden dimension: logits of 0, by the zero fill
        if (p.Ms > 0) ps.push_back(p);
      }
    if ((st = run_dots(ps, vocab_dim == 0 ? GSPMD_LAYOUT_RHS_K_CONTIGUOUS : 0, l.dtype, GSPMD_F32, tables, l.table_bytes(), stream)) != GSPMD_OK) return st;
    // ---- rows
    for (int64_t from = 0; held > 0 && from < l.na && !launches_are_dry(); from += kInlineTokenShards) {
      const int64_t n = std::min<int64_t>(kInlineTokenShards, l.na - from);
      SoftmaxRows a;
      std::memset(&a, 0, sizeof(a));
      for (int64_t i = 0; i < n; ++i) {
        const gspmd_token_buf& tb = token[static_cast<size_t>(from + i)][0];
        a.shard[i] = TokenShard{tb.ids, teacher ? tb.logits : nullptr, tb.weights, tb.loss, tb.lse, static_cast<int32_t>(l.valid_t(from + i)), 0};
      }
      a.z = z + from * rows * ldz;
      a.ldz = ldz;
      a.rows_per = static_cast<int32_t>(rows);
      a.first = static_cast<int32_t>(first);
      a.tokens = static_cast<int32_t>(l.ts);
      a.cols = static_cast<int32_t>((zs - 1) * per_cols + l.valid_v(zs - 1));
      a.vocab = static_cast<int32_t>(l.V);
      a.per = static_cast<int32_t>(l.vs);
      a.per_cols = static_cast<int32_t>(per_cols);
      a.by_cols = fast_div(static_cast<uint32_t>(per_cols));
      a.targets = targets;
      a.inv_tau = 1.f / tau;
      a.logits_bf16 = teacher && tokens[0].logits_dtype == GSPMD_BF16;
      const unsigned blocks = static_cast<unsigned>(n * rows);
      if (!grad) launch_rows_as<float, false>(a, blocks, stream);
      else if (l.dtype == GSPMD_BF16) launch_rows_as<bf16_bits, true>(a, blocks, stream);
      else launch_rows_as<float, true>(a, blocks, stream);
      if (hipGetLastError() != hipSuccess) return GSPMD_ERR_DEVICE;
    }
    // ---- dx: the piece's rows, summed over the vocabulary's shards
    if (l.dx && held > 0) {
      std::vector<Sum> sums(static_cast<size_t>(l.na));
      for (int64_t i = 0; i < l.na; ++i) {
        Sum& s = sums[static_cast<size_t>(i)];
        const gspmd_shard_buf& ob = dx[static_cast<size_t>(i)].first;
        s.ld_out = static_cast<int32_t>(stride_of(ob, l.M));
        s.out = static_cast<char*>(ob.data) + first * s.ld_out * e;
        s.rows = static_cast<int32_t>(held);
        s.cols = static_cast<int32_t>(l.M);
        s.partials = dx_parts ? dx_parts + i * rows * l.nb * round_up(l.M, 4) : nullptr;
        for (int64_t j = 0; j < zs; ++j) {
          const gspmd_shard_buf& wb = w[static_cast<size_t>(j)].first;
          s.members.push_back(problem(z_at(i, j, e), ldd, wb.data, stride_of(wb, w_cols), valid(i), l.M, valid(i) > 0 ? l.valid_v(j) : 0));
        }
      }
      if ((st = run_sums(sums, vocab_dim == 0 ? 0 : GSPMD_LAYOUT_RHS_K_CONTIGUOUS, l.dtype, true, true, tables, l.table_bytes(), stream)) != GSPMD_OK) return st;
    }
    // ---- dw: summed over the tokens' shards and the pieces
    if (l.dw) {
      std::vector<Sum> sums(static_cast<size_t>(l.nb));
      for (int64_t j = 0; j < l.nb; ++j) {
        Sum& s = sums[static_cast<size_t>(j)];
        const gspmd_shard_buf& ob = dw[static_cast<size_t>(j)].first;
        s.out = ob.data;
        s.ld_out = static_cast<int32_t>(stride_of(ob, w_cols));
        s.rows = static_cast<int32_t>(w_rows);
        s.cols = static_cast<int32_t>(w_cols);
        s.partials = dw_parts + j * l.dw_partials(pieces > 1) * dw_size;
        s.earlier = pieces > 1 ? s.partials + l.na * dw_size : nullptr;
        for (int64_t i = 0; i < l.na; ++i) {
          const gspmd_shard_buf& xb = x[static_cast<size_t>(i)].first;
          const int64_t k = l.valid_v(j) > 0 ? valid(i) : 0, ldx = stride_of(xb, l.M);
          s.members.push_back(vocab_dim == 0 ? problem(z_at(i, j, e), ldd, x_at(i), ldx, l.valid_v(j), l.M, k)
                                             : problem(x_at(i), ldx, z_at(i, j, e), ldd, l.M, l.valid_v(j), k));
        }
      }
      if ((st = run_sums(sums, GSPMD_LAYOUT_LHS_K_MAJOR, l.dtype, piece == 0, piece == pieces - 1, tables, l.table_bytes(), stream)) != GSPMD_OK) return st;
    }
  }
  // ---- partitions that hold the same results in buffers of their own
  if (launches_are_dry()) return GSPMD_OK;
  auto spread = [&](const std::vector<Buffers>& at, int64_t r, int64_t c) {
    for (const auto& b : at)
      for (const auto& o : b.others)
        if ((st = copy_rows(b.first, o, r, c, stride_of(b.first, c), stride_of(o, c), stream)) != GSPMD_OK) return st;
    return static_cast<int32_t>(GSPMD_OK);
  };
  if (l.dx && (st = spread(dx, l.ts, l.M)) != GSPMD_OK) return st;
  if (l.dw && (st = spread(dw, w_rows, w_cols)) != GSPMD_OK) return st;
  for (const auto& list : token)
    for (size_t k = 1; k < list.size(); ++k) {
      auto one = [&](float* from, float* to) {
        if (!from || !to || from == to) return static_cast<int32_t>(GSPMD_OK);
        return copy_rows(gspmd_shard_buf{from, GSPMD_F32, 0}, gspmd_shard_buf{to, GSPMD_F32, 0}, 1, l.ts, l.ts, l.ts, stream);
      };
      if ((st = one(list[0].loss, list[k].loss)) != GSPMD_OK || (st = one(list[0].lse, list[k].lse)) != GSPMD_OK) return st;
    }
  return GSPMD_OK;
}

}  // namespace
}  // namespace gspmd

using namespace gspmd;

extern "C" {

int32_t gspmd_softmax_workspace_bytes(const gspmd_mesh* mesh, const gspmd_sharding* x_sh, const gspmd_sharding* w_sh, int32_t vocab_dim, int32_t dtype, int32_t gradients,
                                      int64_t* bytes, int64_t* least) try {
  if (!bytes) return GSPMD_ERR_NULL;
  if (dtype != GSPMD_BF16 && dtype != GSPMD_F32) return GSPMD_ERR_UNSUPPORTED;
  Loss l;
  const int32_t st = analyse(mesh, x_sh, w_sh, vocab_dim, &l);
  if (st != GSPMD_OK) return st;
  l.dtype = dtype;
  l.dx = l.dw = gradients != 0;
  const int64_t whole = l.whole_rows(), rows = std::min(whole, std::max<int64_t>(1, kPieceBytes / (l.na * l.ldz() * 4)));
  *bytes = l.fixed_bytes(rows < whole) + rows * l.row_bytes();
  if (least) *least = std::min(*bytes, l.fixed_bytes(whole > 1) + std::min<int64_t>(whole, 1) * l.row_bytes());
  return GSPMD_OK;
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

int32_t gspmd_softmax_xent(const gspmd_mesh* mesh, const gspmd_shard_buf* x_shards, const gspmd_sharding* x_sh, const gspmd_shard_buf* w_shards, const gspmd_sharding* w_sh,
                           int32_t vocab_dim, const gspmd_token_buf* tokens, const gspmd_shard_buf* dx_shards, const gspmd_shard_buf* dw_shards, void* workspace,
                           int64_t workspace_bytes, void* hip_stream) try {
  return run_loss(mesh, x_shards, x_sh, w_shards, w_sh, vocab_dim, tokens, 1, 1.f, false, dx_shards, dw_shards, workspace, workspace_bytes, hip_stream);
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

int32_t gspmd_softmax_distill(const gspmd_mesh* mesh, const gspmd_shard_buf* x_shards, const gspmd_sharding* x_sh, const gspmd_shard_buf* w_shards, const gspmd_sharding* w_sh,
                              int32_t vocab_dim, const gspmd_token_buf* tokens, int32_t targets, float temperature, const gspmd_shard_buf* dx_shards,
                              const gspmd_shard_buf* dw_shards, void* workspace, int64_t workspace_bytes, void* hip_stream) try {
  return run_loss(mesh, x_shards, x_sh, w_shards, w_sh, vocab_dim, tokens, targets, temperature, true, dx_shards, dw_shards, workspace, workspace_bytes, hip_stream);
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

}  // extern "C"
