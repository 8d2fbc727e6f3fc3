// gspmd_embed, gspmd_embed_grad (include/gspmd.h): the host's part.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "../../include/gspmd.h"
#include "dots.h"
#include "kernels_embed.h"
#include "order.h"
#include "plan.h"
#include "tokens.h"

namespace gspmd {
namespace {

struct Embed {
  int64_t P = 0, T = 0, M = 0, V = 0;
  int64_t na = 1, nb = 1, ts = 0, vs = 0;       // shards of tokens and of the vocabulary, their static extents
  int axis_t = -1, axis_v = -1, vocab_dim = 0;
  int64_t chunk() const { return T <= kFewTokens ? kSmallChunk : kLargeChunk; }
  int64_t chunks() const { return (T + chunk() - 1) / chunk(); }
  // the workspace: the tokens' order and their entries in it, up to a chunk's end; where an entry's begin; chunks' sums, two of each; with dw [M, V] the sums of runs of two tokens and more
  int64_t order_bytes() const { return round_up(chunks() * chunk() * 4, kWsAlign); }
  int64_t begins_bytes() const { return round_up((V + 1) * 4, kWsAlign); }
  int64_t chunks_bytes() const { return round_up(chunks() * M * 4, kWsAlign); }
  bool columns_alone() const { return vocab_dim == 1 && T <= kAloneTokens; }        // (embed_grad_columns_kernel adds runs up itself)
  int64_t sums_bytes() const { return vocab_dim == 1 ? round_up(T / 2 * M * 4, kWsAlign) : 0; }
  int64_t bytes() const { return T == 0 ? 0 : 2 * order_bytes() + begins_bytes() + 2 * chunks_bytes() + sums_bytes(); }
};

int32_t analyse(const gspmd_mesh* mesh, const gspmd_sharding* rows_sh, const gspmd_sharding* w_sh, int32_t vocab_dim, Embed* e) {
  int32_t st = validate_mesh(mesh, &e->P);
  if (st != GSPMD_OK) return st;
  if ((st = validate_sharding(mesh, rows_sh)) != GSPMD_OK || (st = validate_sharding(mesh, w_sh)) != GSPMD_OK) return st;
  if (rows_sh->rank != 2 || w_sh->rank != 2 || (vocab_dim != 0 && vocab_dim != 1)) return GSPMD_ERR_BAD_DOT_DIMS;
  e->T = rows_sh->global_shape[0];
  e->M = rows_sh->global_shape[1];
  e->V = w_sh->global_shape[vocab_dim];
  e->vocab_dim = vocab_dim;
  if (w_sh->global_shape[1 - vocab_dim] != e->M || e->V < 1) return GSPMD_ERR_BAD_DOT_DIMS;
  if (split_axis(mesh, rows_sh, 1) >= 0 || split_axis(mesh, w_sh, 1 - vocab_dim) >= 0) return GSPMD_ERR_NEEDS_RESHARD;
  e->axis_t = split_axis(mesh, rows_sh, 0);
  e->axis_v = split_axis(mesh, w_sh, vocab_dim);
  if (e->axis_t >= 0 && e->axis_t == e->axis_v) return GSPMD_ERR_NEEDS_RESHARD;
  e->na = e->axis_t >= 0 ? mesh->shape[e->axis_t] : 1;
  e->nb = e->axis_v >= 0 ? mesh->shape[e->axis_v] : 1;
  e->ts = (e->T + e->na - 1) / e->na;
  e->vs = (e->V + e->nb - 1) / e->nb;
  constexpr int64_t kMost = INT32_MAX >> 2, kMostColumns = 1 << 21;
  if (e->na > kTokenShards || e->nb > kVocabShards || e->T > (1 << 24) || e->M > kMostColumns || e->V > kMost || e->ts * e->na > kMost || e->vs * e->nb > kMost) return GSPMD_ERR_UNSUPPORTED;
  return GSPMD_OK;
}

struct Shards {                                 // a call's arguments by shard
  std::vector<const int32_t*> ids;
  Replicas rows, vocab;
  int64_t ld_rows = -1, ld_vocab = -1;
};

int32_t collect(const gspmd_mesh* mesh, const Embed& e, const int32_t* const* ids, const gspmd_shard_buf* rows, const gspmd_shard_buf* vocab, Shards* s) {
  const int32_t dtype = rows[0].dtype;
  if (dtype != GSPMD_F32 && dtype != GSPMD_BF16) return GSPMD_ERR_UNSUPPORTED;
  s->ids.assign(static_cast<size_t>(e.na), nullptr);
  for (int64_t p = 0; p < e.P; ++p) {
    int64_t coords[kMaxRank];
    int32_t st = mesh_coords(mesh, p, coords);
    if (st != GSPMD_OK) return st;
    const int64_t i = e.axis_t >= 0 ? coords[e.axis_t] : 0, j = e.axis_v >= 0 ? coords[e.axis_v] : 0;
    if ((st = check_rows(rows[p], dtype, e.M, e.ts * e.M > 0, &s->ld_rows)) != GSPMD_OK) return st;
    if ((st = check_rows(vocab[p], dtype, e.vocab_dim == 0 ? e.M : e.vs, e.M > 0, &s->ld_vocab)) != GSPMD_OK) return st;
    if (e.ts > 0 && !ids[p]) return GSPMD_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(ids[p]) & 3) return GSPMD_ERR_BAD_BUFFER;
    if (!s->ids[static_cast<size_t>(i)]) s->ids[static_cast<size_t>(i)] = ids[p];
    s->rows.add(i, rows[p].data);
    s->vocab.add(j, vocab[p].data);
  }
  return GSPMD_OK;
}

EmbedArgs arguments(const Embed& e, const Shards& s, float scale) {
  EmbedArgs a{};
  for (int64_t i = 0; i < e.na; ++i) a.tokens[i] = TokenShard{s.ids[static_cast<size_t>(i)], s.rows.which[0][static_cast<size_t>(i)]};
  for (int64_t j = 0; j < e.nb; ++j) a.vocab[j] = s.vocab.which[0][static_cast<size_t>(j)];
  a.T = static_cast<int32_t>(e.T);
  a.ts = static_cast<int32_t>(e.ts);
  a.token_shards = static_cast<int32_t>(e.na);
  a.V = static_cast<int32_t>(e.V);
  a.vs = static_cast<int32_t>(e.vs);
  a.vocab_shards = static_cast<int32_t>(e.nb);
  a.M = static_cast<int32_t>(e.M);
  a.ld_rows = static_cast<int32_t>(s.ld_rows);
  a.ld_vocab = s.ld_vocab;
  a.scale = scale;
  return a;
}

// Launches with a table of as few shards as will do.
template <typename Go>
int32_t with_few_shards(const EmbedArgs& a, Go go) {
  if (std::max(a.token_shards, a.vocab_shards) > kFewShards) return go(a);
  EmbedArgsOf<kFewShards> few{};
  static_cast<EmbedSizes&>(few) = a;
  std::copy_n(a.tokens, kFewShards, few.tokens);
  std::copy_n(a.vocab, kFewShards, few.vocab);
  return go(few);
}

template <typename T, typename A>
int32_t launch_embed(const A& a, int vocab_dim, hipStream_t stream) {
  const int64_t rows = static_cast<int64_t>(a.ts) * a.token_shards;
  constexpr int n = Sixteen<T>::n;
  if (vocab_dim == 0) {
    const int log = row_lanes_log(a.M, n);
    const int64_t piece = static_cast<int64_t>(kEmbedUnroll) * n << log, per_group = int64_t(4) << (6 - log);
    const int64_t pieces = (a.M + piece - 1) / piece, groups = (rows + per_group - 1) / per_group * pieces;
    if (groups > kMostGroups) return GSPMD_ERR_UNSUPPORTED;
    const dim3 grid(static_cast<unsigned>(groups));
    return by_lines(lines_of<T>(a.M), [&](auto lines) {
      constexpr int L = decltype(lines)::value;
      if (a.scale == 1.f) hipLaunchKernelGGL((embed_rows_kernel<T, L, false, A>), grid, dim3(256), 0, stream, a, log, static_cast<int>(pieces));
      else hipLaunchKernelGGL((embed_rows_kernel<T, L, true, A>), grid, dim3(256), 0, stream, a, log, static_cast<int>(pieces));
    });
  }
  // blocks of tokens for eight XCDs along x (of 2^24 tokens 2^29 threads; a launch counts them in 32 bits along each dimension), and what each XCD takes one after the other along y
  const int64_t token_blocks = (rows + kColumnTokens - 1) / kColumnTokens, col_blocks = (a.M + kColumnCols - 1) / kColumnCols;
  const dim3 grid(static_cast<unsigned>(8 * token_blocks), static_cast<unsigned>((col_blocks + 7) / 8));
  hipLaunchKernelGGL((embed_columns_kernel<T, A>), grid, dim3(256), 0, stream, a, static_cast<int>(col_blocks));
  return launched();
}

// Sums over the runs of the order: rows of dw [V, M], or what embed_grad_columns_kernel reads.
template <typename T, int TO, int CHUNK, bool ALONE, typename A>
int32_t launch_chunks(const A& a, hipStream_t stream) {
  constexpr int n = Sixteen<T>::n;
  const int64_t chunks = (static_cast<int64_t>(a.T) + CHUNK - 1) / CHUNK;
  const Lines lines = TO == kAddedRows && a.M % n != 0 ? kExact : lines_of<T>(a.M);        // (nothing may be added twice)
  const int log = row_lanes_log(a.M, n);
  int across = 0;
  while (across < 2 && (static_cast<int64_t>(n) << (log + across)) < a.M) ++across;
  const int64_t piece = static_cast<int64_t>(n) << (log + across), units = int64_t(4) >> across << (6 - log);
  const dim3 grid(static_cast<unsigned>((chunks + units - 1) / units), static_cast<unsigned>((a.M + piece - 1) / piece));
  const int32_t st = by_lines(lines, [&](auto l) { hipLaunchKernelGGL((embed_runs_kernel<T, decltype(l)::value, TO, CHUNK, ALONE, A>), grid, dim3(256), 0, stream, a, log, across); });
  if (ALONE || st != GSPMD_OK || chunks < 2) return st;
  const dim3 joins(static_cast<unsigned>(chunks - 1), static_cast<unsigned>((a.M + 64 * n - 1) / (64 * n)));
  if (lines == kExact) hipLaunchKernelGGL((embed_joins_kernel<T, kExact, TO, CHUNK, A>), joins, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((embed_joins_kernel<T, kWide, TO, CHUNK, A>), joins, dim3(256), 0, stream, a);
  return launched();
}
template <typename T, typename A>
int32_t launch_runs(const Embed& e, const A& a, hipStream_t stream) {
  auto of_chunk = [&](auto to) {
    constexpr int TO = decltype(to)::value;
    if constexpr (TO != kSums)
      if (e.T <= kAloneTokens) return launch_chunks<T, TO, kSmallChunk, true>(a, stream);
    return e.chunk() == kSmallChunk ? launch_chunks<T, TO, kSmallChunk, false>(a, stream) : launch_chunks<T, TO, kLargeChunk, false>(a, stream);
  };
  if (e.vocab_dim == 1) return of_chunk(std::integral_constant<int, kSums>{});
  return a.accumulate ? of_chunk(std::integral_constant<int, kAddedRows>{}) : of_chunk(std::integral_constant<int, kRows>{});
}

template <typename T, typename A>
int32_t launch_turn(const Embed& e, const A& a, hipStream_t stream) {
  constexpr int n = Sixteen<T>::n, kRows = kTurnLanes * n;
  const int64_t across = (a.vs + kTurnEntries - 1) / kTurnEntries * static_cast<int64_t>(a.vocab_shards), tiles = across * ((a.M + kRows - 1) / kRows);
  if (tiles > kMostGroups) return GSPMD_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(tiles)), block(256);
  const int x = static_cast<int>(across);
  return by_lines(a.M < n ? kExact : kNarrow, [&](auto lines) {
    constexpr int L = decltype(lines)::value == kExact ? kExact : kNarrow;
    if (e.columns_alone()) {
      if (a.accumulate) hipLaunchKernelGGL((embed_grad_columns_kernel<T, L, float, true, A>), grid, block, 0, stream, a, x);
      else hipLaunchKernelGGL((embed_grad_columns_kernel<T, L, T, true, A>), grid, block, 0, stream, a, x);
    } else {
      if (a.accumulate) hipLaunchKernelGGL((embed_grad_columns_kernel<T, L, float, false, A>), grid, block, 0, stream, a, x);
      else hipLaunchKernelGGL((embed_grad_columns_kernel<T, L, T, false, A>), grid, block, 0, stream, a, x);
    }
  });
}

// The gradient: the tokens' order and zeros, the runs' sums, dw's columns.
template <typename T>
int32_t gradient(const Embed& e, const Shards& s, EmbedArgs a, char* workspace, hipStream_t stream) {
  int32_t st = GSPMD_OK;
  OrderKeys in{};
  OrderOut out{};
  if (e.T > 0) {
    char* at = workspace;
    auto take = [&at](int64_t bytes) { char* const here = at; at += bytes; return here; };
    out.order = reinterpret_cast<int32_t*>(take(e.order_bytes()));
    out.entries = reinterpret_cast<int32_t*>(take(e.order_bytes()));
    out.begins = reinterpret_cast<int32_t*>(take(e.begins_bytes()));
    a.heads = reinterpret_cast<float*>(take(e.chunks_bytes()));
    a.tails = reinterpret_cast<float*>(take(e.chunks_bytes()));
    a.sums = e.columns_alone() ? nullptr : reinterpret_cast<float*>(take(e.sums_bytes()));
    a.order = out.order;
    a.entries = out.entries;
    a.begins = out.begins;
    for (int64_t i = 0; i < e.na; ++i) in.shard[i] = s.ids[static_cast<size_t>(i)];
    in.per = a.ts;
    in.shards = a.token_shards;
    in.count = a.T;
    in.keys = a.V;
  }
  for (const auto& level : s.vocab.which) {
    for (int64_t j = 0; j < e.nb; ++j) a.vocab[j] = level[static_cast<size_t>(j)];
    ZeroRows zero{};
    if (e.vocab_dim == 0) {                     // rows without tokens, and the padding
      for (int64_t j = 0; j < e.nb; ++j) zero.shard[j] = level[static_cast<size_t>(j)];
      zero.per = a.vs;
      zero.shards = a.vocab_shards;
      zero.from = a.accumulate ? a.V : 0;
      zero.halves = a.M * static_cast<int32_t>(sizeof(T) / 2);
      zero.stride = a.ld_vocab * static_cast<int64_t>(sizeof(T) / 2);
    }
    if ((st = run_order(in, out, zero, stream)) != GSPMD_OK) return st;
    if (e.T > 0 && !e.columns_alone() && (e.vocab_dim == 0 || in.count > 0) && (st = with_few_shards(a, [&](const auto& b) { return launch_runs<T>(e, b, stream); })) != GSPMD_OK) return st;
    in.count = 0;                               // (ordered, for the next replicas; columns' sums are there, too)
    if (e.vocab_dim == 1 && (st = with_few_shards(a, [&](const auto& b) { return launch_turn<T>(e, b, stream); })) != GSPMD_OK) return st;
  }
  return st;
}

}  // namespace
}  // namespace gspmd

using namespace gspmd;

extern "C" {

int32_t gspmd_embed(const gspmd_mesh* mesh, const int32_t* const* ids, const gspmd_shard_buf* w_shards, const gspmd_sharding* w_sh, int32_t vocab_dim, float scale,
                    const gspmd_shard_buf* y_shards, const gspmd_sharding* y_sh, void* hip_stream) try {
  if (!ids || !w_shards || !y_shards) return GSPMD_ERR_NULL;
  Embed e;
  int32_t st = analyse(mesh, y_sh, w_sh, vocab_dim, &e);
  if (st != GSPMD_OK) return st;
  Shards s{{}, Replicas(e.na), Replicas(e.nb)};
  if ((st = collect(mesh, e, ids, y_shards, w_shards, &s)) != GSPMD_OK) return st;
  if (e.T == 0 || e.M == 0 || launches_are_dry()) return GSPMD_OK;
  EmbedArgs a = arguments(e, s, scale);
  for (const auto& level : s.rows.which) {
    for (int64_t i = 0; i < e.na; ++i) a.tokens[i].rows = level[static_cast<size_t>(i)];
    st = with_few_shards(a, [&](const auto& b) {
      return y_shards[0].dtype == GSPMD_BF16 ? launch_embed<bf16_bits>(b, vocab_dim, static_cast<hipStream_t>(hip_stream)) : launch_embed<float>(b, vocab_dim, static_cast<hipStream_t>(hip_stream));
    });
    if (st != GSPMD_OK) return st;
  }
  return GSPMD_OK;
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

int32_t gspmd_embed_grad_workspace_bytes(const gspmd_mesh* mesh, const gspmd_sharding* dy_sh, const gspmd_sharding* dw_sh, int32_t vocab_dim, int32_t dtype, int64_t* bytes) try {
  if (!bytes) return GSPMD_ERR_NULL;
  Embed e;
  const int32_t st = analyse(mesh, dy_sh, dw_sh, vocab_dim, &e);
  if (st != GSPMD_OK) return st;
  if (dtype != GSPMD_F32 && dtype != GSPMD_BF16) return GSPMD_ERR_UNSUPPORTED;
  *bytes = e.bytes();
  return GSPMD_OK;
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

int32_t gspmd_embed_grad(const gspmd_mesh* mesh, const int32_t* const* ids, const gspmd_shard_buf* dy_shards, const gspmd_sharding* dy_sh, const gspmd_shard_buf* dw_shards,
                         const gspmd_sharding* dw_sh, int32_t vocab_dim, float scale, int32_t accumulate, void* workspace, int64_t workspace_bytes, void* hip_stream) try {
  if (!ids || !dy_shards || !dw_shards) return GSPMD_ERR_NULL;
  Embed e;
  int32_t st = analyse(mesh, dy_sh, dw_sh, vocab_dim, &e);
  if (st != GSPMD_OK) return st;
  Shards s{{}, Replicas(e.na), Replicas(e.nb)};
  if ((st = collect(mesh, e, ids, dy_shards, dw_shards, &s)) != GSPMD_OK) return st;
  if (e.bytes() > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & (kWsAlign - 1)) || workspace_bytes < e.bytes())) return GSPMD_ERR_WORKSPACE;
  if (e.M == 0 || launches_are_dry()) return GSPMD_OK;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const bool bf16 = dy_shards[0].dtype == GSPMD_BF16;
  EmbedArgs a = arguments(e, s, scale);
  a.accumulate = accumulate != 0;
  return bf16 ? gradient<bf16_bits>(e, s, a, static_cast<char*>(workspace), stream) : gradient<float>(e, s, a, static_cast<char*>(workspace), stream);
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

}  // extern "C"
