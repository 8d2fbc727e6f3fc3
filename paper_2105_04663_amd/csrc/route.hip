// gspmd_route, gspmd_dispatch, gspmd_combine and their gradients (include/gspmd.h): the host's part.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>
#include <vector>

#include "../../include/gspmd.h"
#include "dots.h"
#include "kernels_route.h"
#include "plan.h"
#include "tokens.h"

namespace gspmd {
namespace {

constexpr int64_t kMostTokens = 1 << 24;        // choices of all tokens, too

struct Route {
  int64_t P = 0, T = 0, E = 0, k = 0, na = 1, ts = 0;
  int axis = -1;
  bool few() const { return T <= kFewRouted && T * k <= kOrderThreads; }
  int64_t tiles() const { return (T + kTileTokens - 1) / kTileTokens; }
  // the workspace: the tiles' counts, and with many tiles the experts' totals
  int64_t counts_bytes() const { return round_up(tiles() * E * 4, kWsAlign); }
  int64_t workspace() const { return few() ? 0 : counts_bytes() + (tiles() > kTilesSummed ? round_up(E * 4, kWsAlign) : 0); }
};

int32_t analyse(const gspmd_mesh* mesh, const gspmd_sharding* sh, int32_t choices, Route* r) {
  int32_t st = validate_mesh(mesh, &r->P);
  if (st != GSPMD_OK || (st = validate_sharding(mesh, sh)) != GSPMD_OK) return st;
  if (sh->rank != 2) return GSPMD_ERR_BAD_DOT_DIMS;
  r->T = sh->global_shape[0];
  r->E = sh->global_shape[1];
  r->k = choices;
  if (choices < 1 || choices > r->E) return GSPMD_ERR_BAD_DOT_DIMS;
  if (split_axis(mesh, sh, 1) >= 0) return GSPMD_ERR_NEEDS_RESHARD;
  r->axis = split_axis(mesh, sh, 0);
  r->na = r->axis >= 0 ? mesh->shape[r->axis] : 1;
  r->ts = (r->T + r->na - 1) / r->na;
  if (r->E > kMostExperts || choices > kMostChoices || r->na > kTokenShards || r->T > kMostTokens || r->ts * r->na > kMostTokens || r->T * choices > kMostTokens) return GSPMD_ERR_UNSUPPORTED;
  return GSPMD_OK;
}

int64_t coordinate(const gspmd_mesh* mesh, int64_t p, int axis) {
  int64_t coords[kMaxRank];
  mesh_coords(mesh, p, coords);                 // (a valid mesh, a partition of it)
  return axis >= 0 ? coords[axis] : 0;
}

bool loose(const void* p) { return reinterpret_cast<uintptr_t>(p) & 3; }

// The arrays of a routing that a call needs.
enum : int { kExperts = 1, kWeights = 2, kSlots = 4, kOrder = 8, kSizes = 16 };
int32_t check_route(const gspmd_route_buf* b, int need, bool elements) {
  if (!b) return GSPMD_ERR_NULL;
  const struct { int bit; const void* p; } all[] = {{kExperts, b->experts}, {kWeights, b->weights}, {kSlots, b->slots}, {kOrder, b->order}, {kSizes, b->sizes}};
  for (const auto& one : all) {
    if (!(need & one.bit)) continue;
    if (!one.p && (elements || one.bit == kSizes)) return GSPMD_ERR_NULL;
    if (loose(one.p)) return GSPMD_ERR_BAD_BUFFER;
  }
  return GSPMD_OK;
}

int32_t collect(const gspmd_mesh* mesh, const Route& r, const gspmd_shard_buf* logits, int32_t dtype, int64_t* ld, Replicas* out) {
  for (int64_t p = 0; p < r.P; ++p) {
    const int32_t st = check_rows(logits[p], dtype, r.E, r.ts > 0, ld);
    if (st != GSPMD_OK) return st;
    out->add(coordinate(mesh, p, r.axis), logits[p].data);
  }
  return GSPMD_OK;
}

// A lane's experts: a power of two of them.
template <typename Go>
void by_experts(int64_t E, Go go) {
  if (E <= 16) go(std::integral_constant<int, 1>{});
  else if (E <= 32) go(std::integral_constant<int, 2>{});
  else if (E <= 64) go(std::integral_constant<int, 4>{});
  else if (E <= 128) go(std::integral_constant<int, 8>{});
  else if (E <= 256) go(std::integral_constant<int, 16>{});
  else go(std::integral_constant<int, 32>{});
}
static_assert(kMostExperts == 32 * kRouteLanes, "");

RouteArgs arguments(const Route& r, const Replicas& logits, int64_t ld, const gspmd_route_buf& b, int32_t normalise) {
  RouteArgs a{};
  for (int64_t i = 0; i < r.na; ++i) a.shard[i].logits = logits.which[0][static_cast<size_t>(i)];
  a.T = static_cast<int32_t>(r.T);
  a.ts = static_cast<int32_t>(r.ts);
  a.shards = static_cast<int32_t>(r.na);
  a.E = static_cast<int32_t>(r.E);
  a.k = static_cast<int32_t>(r.k);
  a.ld = static_cast<int32_t>(ld);
  a.normalise = normalise != 0;
  a.experts = b.experts;
  a.weights = b.weights;
  return a;
}

// Launches with a table of as few shards as will do (kernels_embed.h).
template <typename Go>
int32_t with_few_shards(const RouteArgs& a, Go go) {
  if (a.shards > kFewShards) return go(a);
  RouteArgsOf<kFewShards> few{};
  static_cast<RouteSizes&>(few) = a;
  std::copy_n(a.shard, kFewShards, few.shard);
  return go(few);
}
// go(a lane's experts, the arguments): launches.
template <typename Go>
int32_t launch_route(int64_t E, const RouteArgs& a, Go go) {
  return with_few_shards(a, [&](const auto& b) {
    by_experts(E, [&](auto each) { go(each, b); });
    return launched();
  });
}

dim3 token_grid(int64_t tokens) { return dim3(static_cast<unsigned>((tokens * kRouteLanes + 255) / 256)); }

// ---- the exchange
struct Exchange {
  int64_t P = 0, T = 0, M = 0, E = 0, k = 0, na = 1, ts = 0, nb = 1, es = 0;
  int axis_t = -1, axis_e = -1;
};

int32_t analyse_exchange(const gspmd_mesh* mesh, const gspmd_sharding* x_sh, const gspmd_sharding* rows_sh, int32_t choices, Exchange* g) {
  int32_t st = validate_mesh(mesh, &g->P);
  if (st != GSPMD_OK) return st;
  if ((st = validate_sharding(mesh, x_sh)) != GSPMD_OK || (st = validate_sharding(mesh, rows_sh)) != GSPMD_OK) return st;
  if (x_sh->rank != 2 || rows_sh->rank != 3) return GSPMD_ERR_BAD_DOT_DIMS;
  g->T = x_sh->global_shape[0];
  g->M = x_sh->global_shape[1];
  g->E = rows_sh->global_shape[0];
  g->k = choices;
  if (rows_sh->global_shape[2] != g->M || choices < 1 || choices > g->E || rows_sh->global_shape[1] < g->T * choices) return GSPMD_ERR_BAD_DOT_DIMS;
  if (split_axis(mesh, x_sh, 1) >= 0 || split_axis(mesh, rows_sh, 1) >= 0 || split_axis(mesh, rows_sh, 2) >= 0) return GSPMD_ERR_NEEDS_RESHARD;
  g->axis_t = split_axis(mesh, x_sh, 0);
  g->axis_e = split_axis(mesh, rows_sh, 0);
  g->na = g->axis_t >= 0 ? mesh->shape[g->axis_t] : 1;
  g->nb = g->axis_e >= 0 ? mesh->shape[g->axis_e] : 1;
  g->ts = (g->T + g->na - 1) / g->na;
  g->es = (g->E + g->nb - 1) / g->nb;
  if (g->E > kMostExperts || choices > kMostChoices || g->na > kTokenShards || g->nb > kExpertShards || g->T > kMostTokens || g->ts * g->na > kMostTokens || g->T * choices > kMostTokens ||
      g->M > (INT32_MAX >> 2))
    return GSPMD_ERR_UNSUPPORTED;
  return GSPMD_OK;
}

// Buffers by the shard of the tokens (`of_tokens`) or of the experts.
int32_t collect(const gspmd_mesh* mesh, const Exchange& g, const gspmd_shard_buf* bufs, int32_t dtype, bool of_tokens, int64_t* ld, Replicas* out) {
  if (dtype != GSPMD_F32 && dtype != GSPMD_BF16) return GSPMD_ERR_UNSUPPORTED;
  for (int64_t p = 0; p < g.P; ++p) {
    const int32_t st = check_rows(bufs[p], dtype, g.M, g.T * g.M > 0, ld);
    if (st != GSPMD_OK) return st;
    out->add(coordinate(mesh, p, of_tokens ? g.axis_t : g.axis_e), bufs[p].data);
  }
  return GSPMD_OK;
}

ExchangeArgs arguments(const Exchange& g, const gspmd_route_buf& b) {
  ExchangeArgs a{};
  a.T = static_cast<int32_t>(g.T);
  a.ts = static_cast<int32_t>(g.ts);
  a.token_shards = static_cast<int32_t>(g.na);
  a.k = static_cast<int32_t>(g.k);
  a.E = static_cast<int32_t>(g.E);
  a.es = static_cast<int32_t>(g.es);
  a.expert_shards = static_cast<int32_t>(g.nb);
  a.M = static_cast<int32_t>(g.M);
  a.experts = b.experts;
  a.slots = b.slots;
  return a;
}

// Where all experts' rows are in one buffer nobody has to ask whose they are.
void one_buffer(ExchangeArgs* a, bool with_drows) {
  bool one = true;
  for (int j = 1; j < a->expert_shards; ++j) one = one && a->rows[j] == a->rows[0] && (!with_drows || a->drows[j] == a->drows[0]);
  if (one) a->expert_shards = 1;
}

static_assert(kTokenShards == kExpertShards, "one kind of table");
void set(void* (&table)[kTokenShards], const std::vector<void*>& level) {
  for (size_t i = 0; i < level.size(); ++i) table[i] = level[i];
}

enum Exchanged { kDispatch, kCombine, kCombineGrad };
template <typename T>
int32_t launch_exchange(Exchanged what, const ExchangeArgs& a, hipStream_t stream) {
  constexpr int n = Sixteen<T>::n;
  const int log = row_lanes_log(a.M, n);
  const int64_t side = int64_t(4) << (6 - log), rows = what == kCombine ? static_cast<int64_t>(a.ts) * a.token_shards : what == kDispatch ? a.T : static_cast<int64_t>(a.T) * a.k;
  const int64_t piece = (static_cast<int64_t>(n) << log) * (what == kDispatch ? kExchangeUnroll : kCombineUnroll);
  const int64_t pieces = what == kCombineGrad ? 1 : (a.M + piece - 1) / piece, groups = (rows + side - 1) / side * pieces;
  if (groups > kMostGroups) return GSPMD_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(groups));
  return by_lines(lines_of<T>(a.M), [&](auto lines) {
    constexpr int L = decltype(lines)::value;
    if (what == kDispatch) hipLaunchKernelGGL((dispatch_kernel<T, L>), grid, dim3(256), 0, stream, a, log, static_cast<int>(pieces));
    else if (what == kCombine) hipLaunchKernelGGL((combine_kernel<T, L>), grid, dim3(256), 0, stream, a, log, static_cast<int>(pieces));
    else hipLaunchKernelGGL((combine_grad_kernel<T, L>), grid, dim3(256), 0, stream, a, log);
  });
}
int32_t run_exchange(Exchanged what, int32_t dtype, ExchangeArgs a, void* stream) {
  one_buffer(&a, what == kCombineGrad);
  return dtype == GSPMD_BF16 ? launch_exchange<bf16_bits>(what, a, static_cast<hipStream_t>(stream)) : launch_exchange<float>(what, a, static_cast<hipStream_t>(stream));
}

}  // namespace
}  // namespace gspmd

using namespace gspmd;

extern "C" {

int32_t gspmd_route_workspace_bytes(const gspmd_mesh* mesh, const gspmd_sharding* logits_sh, int32_t choices, int64_t* bytes) try {
  if (!bytes) return GSPMD_ERR_NULL;
  Route r;
  const int32_t st = analyse(mesh, logits_sh, choices, &r);
  if (st != GSPMD_OK) return st;
  *bytes = r.workspace();
  return GSPMD_OK;
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

int32_t gspmd_route(const gspmd_mesh* mesh, const gspmd_shard_buf* logits_shards, const gspmd_sharding* logits_sh, int32_t choices, int32_t normalise, const gspmd_route_buf* route,
                    void* workspace, int64_t workspace_bytes, void* hip_stream) try {
  if (!logits_shards) return GSPMD_ERR_NULL;
  Route r;
  int32_t st = analyse(mesh, logits_sh, choices, &r);
  if (st != GSPMD_OK) return st;
  const int32_t dtype = logits_shards[0].dtype;
  if (dtype != GSPMD_F32 && dtype != GSPMD_BF16) return GSPMD_ERR_UNSUPPORTED;
  if ((st = check_route(route, kExperts | kWeights | kSlots | kOrder | kSizes, r.T > 0)) != GSPMD_OK) return st;
  Replicas logits(r.na);
  int64_t ld = -1;
  if ((st = collect(mesh, r, logits_shards, dtype, &ld, &logits)) != GSPMD_OK) return st;
  const int64_t bytes = r.workspace();
  if (bytes > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & (kWsAlign - 1)) || workspace_bytes < bytes)) return GSPMD_ERR_WORKSPACE;
  if (launches_are_dry()) return GSPMD_OK;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const RouteArgs a = arguments(r, logits, ld, *route, normalise);
  int bits = 1;
  while ((int64_t(1) << bits) <= r.E) ++bits;               // of the numbers 0 .. E
  if (r.few()) {
    return launch_route(r.E, a, [&](auto each, const auto& b) {
      constexpr int R = decltype(each)::value;
      typedef std::decay_t<decltype(b)> A;
      if (dtype == GSPMD_BF16) hipLaunchKernelGGL((route_few_kernel<bf16_bits, R, A>), dim3(1), dim3(kOrderThreads), 0, stream, b, bits, route->slots, route->order, route->sizes);
      else hipLaunchKernelGGL((route_few_kernel<float, R, A>), dim3(1), dim3(kOrderThreads), 0, stream, b, bits, route->slots, route->order, route->sizes);
    });
  }
  int32_t* const counts = static_cast<int32_t*>(workspace);
  const unsigned tiles = static_cast<unsigned>(r.tiles());
  st = launch_route(r.E, a, [&](auto each, const auto& b) {
    constexpr int R = decltype(each)::value;
    typedef std::decay_t<decltype(b)> A;
    if (dtype == GSPMD_BF16) hipLaunchKernelGGL((route_kernel<bf16_bits, R, A>), dim3(tiles), dim3(kOrderThreads), 0, stream, b, counts);
    else hipLaunchKernelGGL((route_kernel<float, R, A>), dim3(tiles), dim3(kOrderThreads), 0, stream, b, counts);
  });
  if (st != GSPMD_OK) return st;
  int32_t* totals = nullptr;
  if (tiles > kTilesSummed) {
    totals = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + r.counts_bytes());
    hipLaunchKernelGGL(route_sums_kernel, dim3(static_cast<unsigned>(r.E)), dim3(kOrderThreads), 0, stream, counts, static_cast<int>(tiles), a.E, totals);
    if ((st = launched()) != GSPMD_OK) return st;
  }
  hipLaunchKernelGGL(route_places_kernel, dim3(tiles), dim3(kOrderThreads), 0, stream, route->experts, counts, totals, a.T * a.k, kTileTokens * a.k, a.E, static_cast<int>(tiles), bits, route->slots,
                     route->order, route->sizes);
  return launched();
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

int32_t gspmd_route_grad(const gspmd_mesh* mesh, const gspmd_shard_buf* logits_shards, const gspmd_sharding* logits_sh, int32_t choices, int32_t normalise, const gspmd_route_buf* route,
                         const float* dweights, const gspmd_shard_buf* dlogits_shards, void* hip_stream) try {
  if (!logits_shards || !dlogits_shards) return GSPMD_ERR_NULL;
  Route r;
  int32_t st = analyse(mesh, logits_sh, choices, &r);
  if (st != GSPMD_OK) return st;
  const int32_t dtype = logits_shards[0].dtype;
  if (dtype != GSPMD_F32 && dtype != GSPMD_BF16) return GSPMD_ERR_UNSUPPORTED;
  if ((st = check_route(route, kExperts | kWeights, r.T > 0)) != GSPMD_OK) return st;
  if (!dweights && r.T > 0) return GSPMD_ERR_NULL;
  if (loose(dweights)) return GSPMD_ERR_BAD_BUFFER;
  Replicas logits(r.na), dlogits(r.na);
  int64_t ld = -1, ld_d = -1;
  if ((st = collect(mesh, r, logits_shards, dtype, &ld, &logits)) != GSPMD_OK || (st = collect(mesh, r, dlogits_shards, dtype, &ld_d, &dlogits)) != GSPMD_OK) return st;
  if (r.T == 0 || launches_are_dry()) return GSPMD_OK;
  RouteArgs a = arguments(r, logits, ld, *route, normalise);
  a.ld_d = static_cast<int32_t>(ld_d);
  a.dweights = dweights;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  for (const auto& level : dlogits.which) {
    for (int64_t i = 0; i < r.na; ++i) a.shard[i].dlogits = level[static_cast<size_t>(i)];
    st = launch_route(r.E, a, [&](auto each, const auto& b) {
      constexpr int R = decltype(each)::value;
      typedef std::decay_t<decltype(b)> A;
      if (dtype == GSPMD_BF16) hipLaunchKernelGGL((route_grad_kernel<bf16_bits, R, A>), token_grid(r.ts * r.na), dim3(256), 0, stream, b);
      else hipLaunchKernelGGL((route_grad_kernel<float, R, A>), token_grid(r.ts * r.na), dim3(256), 0, stream, b);
    });
    if (st != GSPMD_OK) return st;
  }
  return GSPMD_OK;
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

int32_t gspmd_dispatch(const gspmd_mesh* mesh, const gspmd_shard_buf* x_shards, const gspmd_sharding* x_sh, int32_t choices, const gspmd_route_buf* route, const gspmd_shard_buf* rows_shards,
                       const gspmd_sharding* rows_sh, void* hip_stream) try {
  if (!x_shards || !rows_shards) return GSPMD_ERR_NULL;
  Exchange g;
  int32_t st = analyse_exchange(mesh, x_sh, rows_sh, choices, &g);
  if (st != GSPMD_OK) return st;
  if ((st = check_route(route, kExperts | kSlots, g.T > 0)) != GSPMD_OK) return st;
  Replicas x(g.na), rows(g.nb);
  int64_t ld_x = -1, ld_rows = -1;
  const int32_t dtype = x_shards[0].dtype;
  if ((st = collect(mesh, g, x_shards, dtype, true, &ld_x, &x)) != GSPMD_OK || (st = collect(mesh, g, rows_shards, dtype, false, &ld_rows, &rows)) != GSPMD_OK) return st;
  if (g.T == 0 || g.M == 0 || launches_are_dry()) return GSPMD_OK;
  ExchangeArgs a = arguments(g, *route);
  a.ld_tokens = ld_x;
  a.ld_rows = ld_rows;
  set(a.tokens, x.which[0]);
  for (const auto& level : rows.which) {
    set(a.rows, level);
    if ((st = run_exchange(kDispatch, dtype, a, hip_stream)) != GSPMD_OK) return st;
  }
  return GSPMD_OK;
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

int32_t gspmd_combine(const gspmd_mesh* mesh, const gspmd_shard_buf* rows_shards, const gspmd_sharding* rows_sh, int32_t choices, const gspmd_route_buf* route, int32_t weighted,
                      const gspmd_shard_buf* y_shards, const gspmd_sharding* y_sh, void* hip_stream) try {
  if (!y_shards || !rows_shards) return GSPMD_ERR_NULL;
  Exchange g;
  int32_t st = analyse_exchange(mesh, y_sh, rows_sh, choices, &g);
  if (st != GSPMD_OK) return st;
  if ((st = check_route(route, kExperts | kSlots | (weighted ? kWeights : 0), g.T > 0)) != GSPMD_OK) return st;
  Replicas y(g.na), rows(g.nb);
  int64_t ld_y = -1, ld_rows = -1;
  const int32_t dtype = rows_shards[0].dtype;
  if ((st = collect(mesh, g, y_shards, dtype, true, &ld_y, &y)) != GSPMD_OK || (st = collect(mesh, g, rows_shards, dtype, false, &ld_rows, &rows)) != GSPMD_OK) return st;
  if (g.T == 0 || g.M == 0 || launches_are_dry()) return GSPMD_OK;
  ExchangeArgs a = arguments(g, *route);
  a.ld_tokens = ld_y;
  a.ld_rows = ld_rows;
  a.weights = weighted ? route->weights : nullptr;
  set(a.rows, rows.which[0]);
  for (const auto& level : y.which) {
    set(a.tokens, level);
    if ((st = run_exchange(kCombine, dtype, a, hip_stream)) != GSPMD_OK) return st;
  }
  return GSPMD_OK;
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

int32_t gspmd_combine_grad(const gspmd_mesh* mesh, const gspmd_shard_buf* dy_shards, const gspmd_sharding* dy_sh, const gspmd_shard_buf* rows_shards, const gspmd_sharding* rows_sh, int32_t choices,
                           const gspmd_route_buf* route, const gspmd_shard_buf* drows_shards, float* dweights, void* hip_stream) try {
  if (!dy_shards || !rows_shards || !drows_shards) return GSPMD_ERR_NULL;
  Exchange g;
  int32_t st = analyse_exchange(mesh, dy_sh, rows_sh, choices, &g);
  if (st != GSPMD_OK) return st;
  if ((st = check_route(route, kExperts | kSlots | kWeights, g.T > 0)) != GSPMD_OK) return st;
  if (!dweights && g.T > 0) return GSPMD_ERR_NULL;
  if (loose(dweights)) return GSPMD_ERR_BAD_BUFFER;
  Replicas dy(g.na), rows(g.nb), drows(g.nb);
  int64_t ld_dy = -1, ld_rows = -1, ld_drows = -1;
  const int32_t dtype = rows_shards[0].dtype;
  if ((st = collect(mesh, g, dy_shards, dtype, true, &ld_dy, &dy)) != GSPMD_OK || (st = collect(mesh, g, rows_shards, dtype, false, &ld_rows, &rows)) != GSPMD_OK ||
      (st = collect(mesh, g, drows_shards, dtype, false, &ld_drows, &drows)) != GSPMD_OK)
    return st;
  if (g.T == 0 || launches_are_dry()) return GSPMD_OK;
  ExchangeArgs a = arguments(g, *route);
  a.ld_tokens = ld_dy;
  a.ld_rows = ld_rows;
  a.ld_drows = ld_drows;
  a.weights = route->weights;
  a.dweights = dweights;
  set(a.tokens, dy.which[0]);
  set(a.rows, rows.which[0]);
  for (const auto& level : drows.which) {
    set(a.drows, level);
    if ((st = run_exchange(kCombineGrad, dtype, a, hip_stream)) != GSPMD_OK) return st;
  }
  return GSPMD_OK;
} catch (...) { return GSPMD_ERR_HOST_MEMORY; }

}  // extern "C"
