// Losses over a split vocabulary (include/gspmd.h: gspmd_softmax_xent, gspmd_softmax_distill).
//
// Tokens are taken in pieces, in the order of all shards together.  A piece's logits go to the workspace as float32; softmax_rows_kernel makes of each row the token's loss
// and, in place, D, the gradient with respect to the logits; two more products make of D the piece's rows of dx and its share of dw.  Losses alone do not keep the logits where their product goes to large
// tiles (kernels_stats.h); a handful of tokens and a small vocabulary matrix have kernels of their own (kernels_few.h, kernels_small.h).
// dx is a sum over the vocabulary.  Where the tokens give it too few output tiles to fill the chip, or the vocabulary's shards lie apart, its ranges are products of their own, float32 partials
// that add_up_kernel adds in ascending order.  dw is a sum over the tokens: x from several shards is put together first (it is small beside w), and pieces add up in float32.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <map>
#include <vector>

#include "../../include/gspmd.h"
#include "dots.h"
#include "kernels_few.h"
#include "kernels_small.h"
#include "kernels_softmax.h"
#include "kernels_stats.h"
#include "plan.h"

namespace gspmd {
namespace {

// Logits of a piece, at most (float32; at least one token's): what the workspace query provides for.  Large, so that the products keep whole rounds of tiles and dw is summed once: pieces small enough
// for the 256 MB cache saved no time (the logits' tiles are stored past it).
constexpr int64_t kPieceBytes = int64_t(1) << 31;
constexpr int64_t kColumnAlign = 64;           // and 8 in narrow shards (Loss::per_cols): the kernels take four logits, or 16 bytes of an operand, of one shard at a time
// Up to so many tokens what D's rounding to bfloat16 loses takes part in the products, as rows of its own: gradients are then off by their own rounding alone (0.0017 of their size, else 0.0024).
// These products are bound by w and dw: 2048 x 32000, 64 tokens 125 us, without 108; 128 tokens 149, 129.
constexpr int64_t kFewTokens = 128;
// Shards of fewer tokens (than a row of tiles) are put together, or each reads the vocabulary matrix for itself (losses of 200 tokens in 4 shards, 2048 x 16000: 30 us, else 40).
constexpr int64_t kFewRows = 256;
// Elements of a partial of dx that are hardly noticed: ranges of 512 entries, else of 2048 (200 tokens, 1001 x 16001: 73 us, by 2048 78; 1024 tokens, 2048 x 8000: 126, by 512 137).
constexpr int64_t kSmallSum = int64_t(1) << 20;
// Shards of the vocabulary of less than a tile, in products that are worth a copy of w and a launch for dw's places (losses of 4000 tokens, 2048 x 800 in 8 shards: 31 us, each for itself 34; gradients of
// 16000 tokens, 8000 x 110 in 8 shards float32 1153, each for itself 3147; 1000 tokens, 1024 x 400, 0.4e9: 60.5, together 63).
constexpr int64_t kNarrow = 128;
constexpr double kNarrowWork = 2e9;
// Logits that caches do not hold: not kept, even by the kernel that is slower at their product (losses alone, us kept / not kept: 2048 x 128 x 16000, 131 MB, 54 / 37; 4096 x 64 x 32000 232 / 103;
// 7884 x 404 x 55589 1032 / 634; 9670 x 96 x 2251, 87 MB, 61 / 65).
constexpr int64_t kLongLogits = int64_t(96) << 20;
// One launch for everything (kernels_small.h) against four to six, us a step with gradients, M x V: bfloat16 100 x 160, 4 tokens 18 / 31, 500 22 / 29, 4000 26 / 34; 256 x 256 (128 KB) 21 / 25, 27 / 28,
// 31 / 34; 256 x 500 25 / 25, 33 / 31, 40 / 37; 512 x 512 33 / 26, 42 / 31, 57 / 39; float32 100 x 160 (64 KB) 19 / 26, 28 / 32, 34 / 39; 256 x 256 27 / 25, 40 / 35, 44 / 41.  Losses alone
// (against two launches): 100 x 160 12 / 15.5; 256 x 256 bfloat16 12 / 15.5, float32 15 / 15, 500 tokens 18 / 15.
constexpr int64_t kSmallMost = 4096, kSmallWeights = int64_t(128) << 10;
// A handful of tokens (kernels_few.h): w that the caches hold, and workgroups of their kernels.
constexpr int64_t kFewWeights = int64_t(32) << 20;
constexpr int64_t kFewWorkgroups = 12 * 256;

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
  int64_t valid_v(int64_t j) const { return std::max<int64_t>(0, std::min(vs, V - j * vs)); }
  // a row of logits: the vocabulary shards that hold any entry, one after the other
  int64_t windows() const { return (V + vs - 1) / vs; }
  // Shards start on whole lines, unless that would make rows much longer (110 entries in 8 shards: 512 columns, not 112), and on 64 columns where their products may end in statistics.
  int64_t per_cols() const { return round_up(vs, windows() == 1 || vs >= 1024 || (vs >= kNarrow && !dx && !dw && dtype == GSPMD_BF16) ? kColumnAlign : 8); }
  int64_t cols() const { return (windows() - 1) * per_cols() + valid_v(windows() - 1); }
  int64_t ldz() const { return round_up(windows() * per_cols(), kColumnAlign); }
  int64_t w_rows() const { return vocab_dim == 0 ? vs : M; }
  int64_t w_cols() const { return vocab_dim == 0 ? M : vs; }
  // both parts of D
  bool with_lost() const { return (dx || dw) && dtype == GSPMD_BF16 && T <= kFewTokens; }
  int64_t parts() const { return with_lost() ? 2 : 1; }
  int64_t ldx() const { return round_up(std::max<int64_t>(M, 1), kColumnAlign); }        // of x put together
  int64_t ld_sum() const { return round_up(std::max<int64_t>(M, 1), 4); }                // of dx's partials
  // Ranges of the vocabulary whose products make dx, for pieces of `rows` tokens: of all of it where it lies in one matrix, and of one of its shards.
  int64_t ranges(int64_t rows) const {
    if (!dx || rows == 0) return 1;
    const bool few = rows * parts() <= 128, small = dtype == GSPMD_F32 || few;
    const int64_t edge = small ? 64 : 256, tiles = ((rows * parts() + edge - 1) / edge) * ((M + edge - 1) / edge);
    const int64_t want = dtype == GSPMD_F32 ? 1024 : few ? 512 : 256;         // workgroups: a round of those kernels' on 256 compute units (not searched: nor is the cap of 16)
    // entries of a range (float32, 100 tokens, 300 x 3000 by 256 37.5 us, by 512 41; 512 tokens, 512 x 3000 73 and 69)
    const int64_t least = dtype == GSPMD_F32 && rows <= 256 ? 256 : small || rows * M <= kSmallSum ? 512 : 2048;
    return std::max<int64_t>(1, std::min({want / std::max<int64_t>(tiles, 1), V / least, int64_t(16)}));
  }
  int64_t ranges_of_shard(int64_t rows) const { return std::max<int64_t>(1, std::min(ranges(rows), int64_t(32)) / windows()); }
  int64_t most_ranges(int64_t rows) const { return std::max(ranges(rows), windows() * ranges_of_shard(rows)); }
  bool adds_up(int64_t rows) const { return dx && (most_ranges(rows) > 1 || with_lost()); }
  // Ranges of the tokens whose products make dw together, in one matrix of all shards, where its tiles are few (bfloat16, 4000 tokens, 512 x 2000 68 us, in one range 81; float32, 2000 tokens, 512 x 800
  // 73 and 79; 12480 tokens, 135 x 707 153 and 285) ..
  int64_t dw_ranges() const {
    if (!dw || T == 0) return 1;
    const int64_t edge = dtype == GSPMD_F32 ? 64 : 256, tiles = ((cols() + edge - 1) / edge) * ((M + edge - 1) / edge);
    const int64_t want = dtype == GSPMD_F32 ? 1024 : 256, least = dtype == GSPMD_F32 ? 512 : 1024;
    return std::max<int64_t>(1, std::min({want / std::max<int64_t>(tiles, 1), T / least, int64_t(16)}));
  }
  double work() const { return static_cast<double>(T) * static_cast<double>(M) * static_cast<double>(V); }
  bool narrow() const { return nb > 1 && vs < kNarrow && work() >= kNarrowWork; }
  // .. of each shard of tokens by itself, where the partials are less than x put together: no copy of x then (12856 tokens in 3 shards, 2203 x 284: a copy is 27 of 165 us).
  bool ranges_by_shard() const { return dw && na > 1 && !with_lost() && ts >= kFewRows && na * V * 4 <= T * esize(); }
  int64_t dw_parts() const { return ranges_by_shard() ? na * std::max<int64_t>(1, dw_ranges() / na) : dw_ranges(); }
  bool joins_dw() const { return dw && M > 0 && (dw_parts() > 1 || narrow()); }
  int64_t ld_dw() const { return vocab_dim == 0 ? ld_sum() : ldz(); }
  int64_t dw_part() const { return (vocab_dim == 0 ? ldz() : M) * ld_dw(); }
  int64_t joined_dw_bytes() const { return joins_dw() ? round_up(dw_parts() * dw_part() * 4, kWsAlign) : 0; }
  int64_t most_rows() const { return std::min(T, std::max<int64_t>(1, kPieceBytes / (ldz() * 4))); }
  // A padded copy of operands whose rows are not padded to 16 bytes, which the products read several times slower than they are copied once (1001 x 16001: 600 tokens 131 us, without 153; losses
  // alone, 600 tokens 49 and 54, 2000 tokens 87 and 133; 200 tokens 78 and 73; losses of 512 tokens, 515 x 8001 26 and 21) ..
  bool packing_pays() const {
    return dtype == GSPMD_BF16 && (T >= 1024 || (T >= (dx || dw ? 342 : 512) && work() >= 4e9));
  }
  // .. and of a vocabulary in many shards, where dx's partials, one for each, would be more than that copy (bfloat16, 3000 tokens, 1024 x 16000 in 8 shards, 2 T windows / V = 3, 329 us, apart 359; 4096 tokens,
  // 2048 x 32000 in 4, 1.0, 1386, apart 1347; nothing was measured between the two, the limit is the upper one), or whose shards are narrow.
  bool joining_pays() const { return windows() > 1 && ((dx && 2 * T * windows() >= 3 * V) || narrow()); }
  int64_t packed_w_bytes() const { return round_up((vocab_dim == 0 ? ldz() * ldx() : std::max<int64_t>(M, 1) * ldz()) * esize(), kWsAlign); }
  // ---- the workspace, for pieces of `rows` tokens
  int64_t table_bytes() const { return round_up((na * nb + 32 + nb) * kTableBytesPerProblem, kWsAlign); }
  int64_t x_bytes(int64_t rows) const { return round_up(rows * parts() * ldx() * esize(), kWsAlign); }
  int64_t z_bytes(int64_t rows) const { return round_up(rows * parts() * ldz() * 4, kWsAlign); }
  int64_t sum_bytes(int64_t rows) const { return adds_up(rows) ? round_up(most_ranges(rows) * parts() * rows * ld_sum() * 4, kWsAlign) : 0; }
  int64_t dw_size() const { return round_up(w_rows() * round_up(w_cols(), 4) * 4, kWsAlign) / 4; }                 // float32 elements of a shard's partial
  int64_t dw_bytes(int64_t rows) const { return dw && rows < T ? 2 * nb * dw_size() * 4 : 0; }
  // ---- a handful of tokens (kernels_few.h): as many as were measured faster there, all sizes of w from 0.6 to 262 MB together (us, a step with gradients, these kernels / the others;
  // M x V): float32, [V, M], 1 token 640 x 10368 32 / 51, 2048 x 32000 182 / 225; 8 tokens 37 / 52, 185 / 237; 16 tokens 55 / 53, 242 / 239; [M, V], 4 tokens 40 / 52, 183 / 225;
  // 8 tokens 50 / 53, 131 / 123 (2048 x 16000).  bfloat16, [V, M], 1 token 128 x 2304 27 / 34, 1024 x 16000 34 / 42, 2048 x 16000 55 / 57, 2048 x 32000 106 / 101; 3 tokens 24 / 32, 39 / 41,
  // 63 / 58, 115 / 102; 8 tokens 640 x 10368 43 / 35; losses alone, 1 token 640 x 10368 14 / 15.5, 1024 x 16000 15 / 17, 4 tokens
  // 16 / 16.5; [M, V], 3 tokens 640 x 10368 36 / 35, 2048 x 16000 84 / 59.
  // bfloat16 beyond 32 MB of w: only where its rows are not whole lines, which the others read slowly (3001 x 20001 in 4 shards, 1 token 98 / 137, 4 tokens 111 / 140; 904 x 50000, 2 tokens 85 / 99,
  // 4 tokens 90 / 100; 1900 x 20000 76 / 90; 6390 x 116189 in 8 shards, rows of 6392, 1026 / 1018; losses alone, 3001 x 20001, 1 token 35 / 58, 4 tokens 44 / 60;
  // whole lines: 3904 x 123392, 1 token 600 / 540, 4 tokens 612 / 548; losses alone, 1 token 2048 x 32000 38.7 / 36.5, 4096 x 32000 67 / 64), and losses of one or two tokens over many short rows (1024 x 50000 31 / 35, 1536 x 80000 55 / 69, 2048 x 128000 110 / 144, 512 x 128000 41 / 41).
  bool few() const {
    const int64_t most = dtype == GSPMD_F32 ? (vocab_dim == 0 || V * M * 4 <= kFewWeights ? 8 : 4) : vocab_dim == 0 ? 4 : 0;
    return T > 0 && T <= most && M > 0 && nb <= kFewWindows && na <= kInlineTokenShards;
  }
  bool few_takes(bool w_lines) const { return few() && (dtype == GSPMD_F32 || !w_lines || V * M * 2 <= kFewWeights || (!dx && !dw && T <= 2 && V >= 48000 && M <= 2048)); }
  int64_t few_lanes() const {                // [V, M]: of a row
    int64_t lanes = 1;
    while (lanes < 64 && lanes * 16 / esize() < M) lanes *= 2;
    return lanes;
  }
  // Ranges of the vocabulary that dx has partials of: enough workgroups, as long as the partials are little beside w.
  int64_t few_ranges(int64_t* each, int64_t* blocks) const {
    if (vocab_dim == 1) {
      *blocks = (vs + 1024 / esize() - 1) / (1024 / esize());
      const int64_t y = std::max<int64_t>(1, std::min<int64_t>(kFewWorkgroups / std::max<int64_t>(nb * *blocks, 1), M / 32));
      *each = round_up((M + y - 1) / y, 32);
      return nb * *blocks;
    }
    const int64_t across = few_across(), sides = 4 * (64 / few_lanes());
    const int64_t ranges = std::max<int64_t>(1, std::min({kFewWorkgroups / across, V * esize() / (32 * T), int64_t(512)}) / nb);
    *each = round_up((vs + ranges - 1) / ranges, sides);
    *blocks = (vs + *each - 1) / *each;
    return nb * *blocks;
  }
  int64_t few_across() const { return (M + few_lanes() * 16 / esize() - 1) / (few_lanes() * 16 / esize()); }
  int64_t few_bytes() const {
    int64_t each, blocks;
    return round_up(T * ldz() * 4, kWsAlign) + (dx ? few_ranges(&each, &blocks) * T * ld_sum() * 4 : 0);
  }
  // All in one workgroup for 16 tokens (kernels_small.h).
  bool small() const { return T > 0 && T <= kSmallMost && M >= 8 && (vocab_dim == 0 || vs >= 8) && V * M * esize() <= kSmallWeights && ldz() <= kSmallColumns && na <= kSmallShards && nb <= kSmallShards; }
  // Workgroups for the same tokens: as many as have a part of dx's columns or of dw's tiles to make (bfloat16, 16 tokens, 256 x 256 22 us, by one 25; 40 tokens, 600 x 100 24 and 27; 4 tokens, 100 x 160
  // 17.7 and 17).
  int64_t small_slices() const {
    const int64_t across = (M + 63) / 64, blocks = (na * ts + kSmallTokens - 1) / kSmallTokens;
    int64_t want = 1;
    if (dx) want = std::min<int64_t>(across, (across * ldz() + 1023) / 1024);
    if (dw && T <= kSmallTokens) want = std::max(want, std::min<int64_t>(64, across * ldz() / 512));
    return std::max<int64_t>(1, std::min(want, 256 / blocks));
  }
  int64_t bytes(int64_t rows) const { return table_bytes() + x_bytes(rows) + z_bytes(rows) + sum_bytes(rows) + dw_bytes(rows); }
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
  if (l->T > kMost || l->M > kMost || l->V > kMost || l->ldz() > kMost || l->na * l->nb > kMaxProblems / 2) return GSPMD_ERR_UNSUPPORTED;
  return GSPMD_OK;
}

struct Buffers {                             // the distinct ones of one position, the first of which is computed into
  gspmd_shard_buf first;
  std::vector<gspmd_shard_buf> others;
};

void add_buffer(std::vector<Buffers>& at, int64_t pos, bool seen, const gspmd_shard_buf& b) {
  Buffers& here = at[static_cast<size_t>(pos)];
  if (!seen) {
    here.first = b;
    return;
  }
  if (b.data == here.first.data) return;
  for (const auto& o : here.others) if (o.data == b.data) return;
  here.others.push_back(b);
}

// A shard's row stride in elements, or -1.
int64_t stride_of(const gspmd_shard_buf& b, int64_t cols) {
  const int64_t ld = b.row_stride > 0 ? b.row_stride : cols;
  return ld < cols || ld > INT32_MAX ? -1 : std::max<int64_t>(ld, 1);
}

bool padded(const gspmd_shard_buf& b, int64_t ld) { return !(reinterpret_cast<uintptr_t>(b.data) & 15) && !(ld & 7); }

template <typename T, bool GRAD, bool LOST>
void launch_rows_as(const SoftmaxRows& a, unsigned rows, hipStream_t stream) {
  const size_t lds = static_cast<size_t>((a.targets + 3) & ~3) * 12;
  if (a.cols <= 64 * 4 * 4) hipLaunchKernelGGL((softmax_rows_kernel<T, 64, 4, false, GRAD, LOST>), dim3(rows), dim3(64), lds, stream, a);
  else if (a.cols <= 256 * 4 * 8) hipLaunchKernelGGL((softmax_rows_kernel<T, 256, 8, false, GRAD, LOST>), dim3(rows), dim3(256), lds, stream, a);
  else if (a.cols <= 512 * 4 * 8) hipLaunchKernelGGL((softmax_rows_kernel<T, 512, 8, false, GRAD, LOST>), dim3(rows), dim3(512), lds, stream, a);
  else if (a.cols <= 1024 * 4 * 8) hipLaunchKernelGGL((softmax_rows_kernel<T, 1024, 8, false, GRAD, LOST>), dim3(rows), dim3(1024), lds, stream, a);
  else if (a.cols <= 1024 * 4 * 16) hipLaunchKernelGGL((softmax_rows_kernel<T, 1024, 16, false, GRAD, LOST>), dim3(rows), dim3(1024), lds, stream, a);
  else hipLaunchKernelGGL((softmax_rows_kernel<T, 1024, 8, true, GRAD, LOST>), dim3(rows), dim3(1024), lds, stream, a);
}

int32_t launched() { return hipGetLastError() == hipSuccess ? GSPMD_OK : GSPMD_ERR_DEVICE; }

int32_t launch_rows(const SoftmaxRows& a, const Loss& l, int64_t rows, hipStream_t stream) {
  const unsigned n = static_cast<unsigned>(rows);
  if (!l.dx && !l.dw) launch_rows_as<float, false, false>(a, n, stream);
  else if (l.dtype == GSPMD_F32) launch_rows_as<float, true, false>(a, n, stream);
  else if (l.with_lost()) launch_rows_as<bf16_bits, true, true>(a, n, stream);
  else launch_rows_as<bf16_bits, true, false>(a, n, stream);
  return launched();
}

dim3 rows_grid(int64_t vectors, int64_t rows) {
  return dim3(static_cast<unsigned>((vectors + 255) / 256), static_cast<unsigned>(std::min<int64_t>(rows, 32768)));
}

// Copies that nothing has needed yet, launched two at a time (x and w one after the other: 4 us more).
struct Packs {
  PackTwo args;
  int n = 0;
  int32_t dtype;
  hipStream_t stream;
  int32_t flush() {
    if (n == 0) return GSPMD_OK;
    int64_t blocks = 0;
    for (int k = 0; k < 2; ++k) {
      args.across[k] = k < n ? (args.two[k].chunks + 255) / 256 : 0;
      args.down[k] = k < n ? std::min(args.two[k].rows, 32768) : 0;
      blocks += static_cast<int64_t>(args.across[k]) * args.down[k];
    }
    const dim3 grid(static_cast<unsigned>(blocks));
    if (dtype == GSPMD_BF16) hipLaunchKernelGGL((pack_rows_kernel<uint16_t>), grid, dim3(256), 0, stream, args);
    else hipLaunchKernelGGL((pack_rows_kernel<uint32_t>), grid, dim3(256), 0, stream, args);
    n = 0;
    return launched();
  }
  int32_t add(const PackRows& a) {
    if (a.rows <= 0 || a.chunks <= 0) return GSPMD_OK;       // (a table of shards beyond the last token)
    args.two[n++] = a;
    return n == 2 ? flush() : static_cast<int32_t>(GSPMD_OK);
  }
};

int32_t launch_add_up(const AddUp& a, int32_t dtype, hipStream_t stream) {
  const dim3 grid = rows_grid((a.cols + 3) / 4, a.rows);
  if (dtype == GSPMD_BF16) hipLaunchKernelGGL((add_up_kernel<bf16_bits>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((add_up_kernel<float>), grid, dim3(256), 0, stream, a);
  return launched();
}

int32_t copy_rows(const gspmd_shard_buf& from, const gspmd_shard_buf& to, int64_t rows, int64_t cols, int64_t ld_from, int64_t ld_to, hipStream_t stream) {
  if (rows == 0 || cols == 0) return GSPMD_OK;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((cols + 255) / 256, 64)), static_cast<unsigned>(std::min<int64_t>(rows, 4096)));
  if (from.dtype == GSPMD_BF16) hipLaunchKernelGGL((copy_rows_kernel<uint16_t>), grid, dim3(256), 0, stream, static_cast<const uint16_t*>(from.data), static_cast<uint16_t*>(to.data), rows, cols, ld_from, ld_to);
  else hipLaunchKernelGGL((copy_rows_kernel<uint32_t>), grid, dim3(256), 0, stream, static_cast<const uint32_t*>(from.data), static_cast<uint32_t*>(to.data), rows, cols, ld_from, ld_to);
  return launched();
}

int32_t check_shard(const gspmd_shard_buf& b, int32_t dtype, int64_t rows, int64_t cols) {
  if (b.dtype != dtype) return GSPMD_ERR_UNSUPPORTED;
  if (b.row_stride < 0 || stride_of(b, cols) < 0) return GSPMD_ERR_BAD_BUFFER;
  if (!b.data && rows > 0 && cols > 0) return GSPMD_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(b.data) & (dtype == GSPMD_BF16 ? 1 : 3)) return GSPMD_ERR_BAD_BUFFER;
  return GSPMD_OK;
}

// Every array of a token at its elements' alignment: weights and losses are reached by scalar instructions too, which take an address's last two bits for zeros.
bool aligned(const gspmd_token_buf& tb, bool teacher) {
  const uintptr_t words = reinterpret_cast<uintptr_t>(tb.ids) | reinterpret_cast<uintptr_t>(tb.weights) | reinterpret_cast<uintptr_t>(tb.loss) | reinterpret_cast<uintptr_t>(tb.lse);
  return !(words & 3) && !(teacher && (reinterpret_cast<uintptr_t>(tb.logits) & (tb.logits_dtype == GSPMD_BF16 ? 1 : 3)));
}

Problem product(const void* a, int64_t lda, const void* b, int64_t ldb, void* c, int64_t ldc, int64_t m, int64_t n, int64_t k, int64_t m_static, int64_t n_static) {
  Problem p;
  std::memset(&p, 0, sizeof(p));
  p.A = a;
  p.B = b;
  p.C = c;
  p.lda = static_cast<int32_t>(lda);
  p.ldb = static_cast<int32_t>(ldb);
  p.ldc = static_cast<int32_t>(ldc);
  p.Ms = static_cast<int32_t>(m_static);
  p.Ns = static_cast<int32_t>(n_static);
  if (m > 0 && n > 0 && k > 0) {               // all or none: without a term to sum the output is its zero fill
    p.Mv = static_cast<int32_t>(m);
    p.Nv = static_cast<int32_t>(n);
    p.Kv = static_cast<int32_t>(k);
  }
  return p;
}

// The calls' kernels for a handful of tokens: `a` and `rows` hold the arguments of both products and of the row kernel.
template <typename T, int NT>
int32_t launch_few_logits(const FewTokens& a, const Loss& l, hipStream_t stream) {
  FewTokens b = a;
  if (l.vocab_dim == 0) {
    constexpr int kRows = NT >= 4 ? 4 : 8;
    const int64_t per_block = 4 * (64 / a.lanes) * kRows;
    b.blocks = static_cast<int32_t>((l.vs + per_block - 1) / per_block);
    hipLaunchKernelGGL((few_logits_kernel<T, NT, kRows>), dim3(static_cast<unsigned>(l.windows() * b.blocks)), dim3(256), 0, stream, b);
  } else if constexpr (sizeof(T) == 4) {
    auto go = [&](auto side) {               // narrower where wide ones would leave compute units without one
      constexpr int kSide = decltype(side)::value, kCols = kSide * few_vec<T>(), lds = std::max(512 * NT, (kFewAcross / 64) * NT * kCols) * 4;
      b.blocks = static_cast<int32_t>((l.vs + kCols - 1) / kCols);
      hipLaunchKernelGGL((few_logits_across_kernel<T, NT, kSide>), dim3(static_cast<unsigned>(l.windows() * b.blocks)), dim3(kFewAcross), lds, stream, b);
    };
    if (l.V >= 64 * 16 * few_vec<T>()) go(std::integral_constant<int, 16>{}); else go(std::integral_constant<int, 4>{});
  }
  return launched();
}

template <typename T, int NT>
int32_t launch_few_gradients(const FewTokens& a, const Loss& l, int64_t ranges, hipStream_t stream) {
  if (l.vocab_dim == 0)
    hipLaunchKernelGGL((few_gradients_kernel<T, NT>), dim3(static_cast<unsigned>(l.few_across()), static_cast<unsigned>(ranges)), dim3(256), (few_gradients_lds<T, NT>(a.lanes)), stream, a);
  else if constexpr (sizeof(T) == 4)
    hipLaunchKernelGGL((few_gradients_across_kernel<T, NT>), dim3(static_cast<unsigned>(ranges), static_cast<unsigned>((l.M + a.each - 1) / a.each)), dim3(256), 256 * NT * 4, stream, a);
  return launched();
}

template <typename T, typename Go>
int32_t few_by_tokens(int64_t tokens, Go go) {
  if (tokens <= 1) return go(std::integral_constant<int, 1>{});
  if (tokens <= 2) return go(std::integral_constant<int, 2>{});
  if constexpr (sizeof(T) == 4) if (tokens > 4) return go(std::integral_constant<int, 8>{});
  return go(std::integral_constant<int, 4>{});
}

template <typename T>
int32_t run_few(const Loss& l, FewTokens& a, const SoftmaxRows& rows, AddUp& sums, hipStream_t stream) {
  int32_t st = few_by_tokens<T>(l.T, [&](auto nt) { return launch_few_logits<T, decltype(nt)::value>(a, l, stream); });
  if (st != GSPMD_OK) return st;
  const unsigned tokens = static_cast<unsigned>(l.na * l.ts);
  if (l.dx || l.dw) launch_rows_as<float, true, false>(rows, tokens, stream); else launch_rows_as<float, false, false>(rows, tokens, stream);
  if ((st = launched()) != GSPMD_OK || !(l.dx || l.dw)) return st;
  int64_t each, blocks;
  const int64_t ranges = l.few_ranges(&each, &blocks);
  a.each = static_cast<int32_t>(each);
  a.blocks = static_cast<int32_t>(blocks);
  st = few_by_tokens<T>(l.T, [&](auto nt) { return launch_few_gradients<T, decltype(nt)::value>(a, l, ranges, stream); });
  if (st != GSPMD_OK || !l.dx) return st;
  sums.partials = a.sums;
  sums.stride = l.T * l.ld_sum();
  sums.ld_in = l.ld_sum();
  sums.count = static_cast<int32_t>(ranges);
  hipLaunchKernelGGL((add_up_few_kernel<T>), dim3(static_cast<unsigned>((l.M + 63) / 64), static_cast<unsigned>(sums.rows)), dim3(256), 0, stream, sums);
  return launched();
}

template <typename T>
int32_t launch_small(const SmallLoss& a, const Loss& l, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((l.na * l.ts + kSmallTokens - 1) / kSmallTokens), static_cast<unsigned>(l.small_slices()));
  auto go = [&](auto dw) {
    constexpr bool kDw = decltype(dw)::value;
    if (l.vocab_dim == 0) hipLaunchKernelGGL((small_loss_kernel<T, 0, kDw>), grid, dim3(kSmallThreads), 0, stream, a);
    else hipLaunchKernelGGL((small_loss_kernel<T, 1, kDw>), grid, dim3(kSmallThreads), 0, stream, a);
  };
  if (a.dw[0] != nullptr) go(std::true_type{}); else go(std::false_type{});
  return launched();
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
  const int64_t w_rows = l.w_rows(), w_cols = l.w_cols();
  for (int64_t at = 0; at < l.P; ++at) {
    const int64_t p = mesh->device_ids[at];
    int64_t coords[kMaxRank], rest = at;
    for (int a = mesh->rank - 1; a >= 0; --a) {
      coords[a] = rest % mesh->shape[a];
      rest /= mesh->shape[a];
    }
    const int64_t i = l.axis_t >= 0 ? coords[l.axis_t] : 0, j = l.axis_v >= 0 ? coords[l.axis_v] : 0;
    if ((st = check_shard(x_shards[p], l.dtype, l.ts, l.M)) != GSPMD_OK || (st = check_shard(w_shards[p], l.dtype, w_rows, w_cols)) != GSPMD_OK) return st;
    if (l.dx && (st = check_shard(dx_shards[p], l.dtype, l.ts, l.M)) != GSPMD_OK) return st;
    if (l.dw && (st = check_shard(dw_shards[p], l.dtype, w_rows, w_cols)) != GSPMD_OK) return st;
    auto other_stride = [&](const gspmd_shard_buf* shards, int64_t cols) { return shards && stride_of(shards[p], cols) != stride_of(shards[0], cols); };      // (0 is that of a dense shard)
    if (other_stride(x_shards, l.M) || other_stride(w_shards, w_cols) || other_stride(dx_shards, l.M) || other_stride(dw_shards, w_cols)) return GSPMD_ERR_BAD_BUFFER;
    const gspmd_token_buf& tb = tokens[p];
    if (l.ts > 0 && (!tb.ids || !tb.loss || (teacher && !tb.logits))) return GSPMD_ERR_NULL;
    if (teacher && tb.logits_dtype != GSPMD_F32 && tb.logits_dtype != GSPMD_BF16) return GSPMD_ERR_UNSUPPORTED;
    if (teacher && tb.logits_dtype != tokens[0].logits_dtype) return GSPMD_ERR_UNSUPPORTED;
    if (l.ts > 0 && !aligned(tb, teacher)) return GSPMD_ERR_BAD_BUFFER;
    const bool ts = seen_t[static_cast<size_t>(i)], vs = seen_v[static_cast<size_t>(j)];
    if (!ts) x[static_cast<size_t>(i)].first = x_shards[p];
    if (!vs) w[static_cast<size_t>(j)].first = w_shards[p];
    if (l.dx) add_buffer(dx, i, ts, dx_shards[p]);
    if (l.dw) add_buffer(dw, j, vs, dw_shards[p]);
    auto& mine = token[static_cast<size_t>(i)];
    const bool known = std::any_of(mine.begin(), mine.end(), [&](const gspmd_token_buf& o) { return o.loss == tb.loss && o.lse == tb.lse; });
    if (!known) mine.push_back(tb);
    seen_t[static_cast<size_t>(i)] = seen_v[static_cast<size_t>(j)] = 1;
  }
  // (the first of a shard's is what the kernel writes: one with an lse, if any has)
  for (auto& list : token) std::stable_partition(list.begin(), list.end(), [](const gspmd_token_buf& tb) { return tb.lse != nullptr; });

  // partitions that hold the same results in buffers of their own
  const bool dry = launches_are_dry();
  const int64_t ldx_in = stride_of(x_shards[0], l.M), ldw = stride_of(w_shards[0], w_cols);
  const int64_t lddx = l.dx ? stride_of(dx_shards[0], l.M) : 0, lddw = l.dw ? stride_of(dw_shards[0], w_cols) : 0;
  auto spread_results = [&]() -> int32_t {
    if (dry) return GSPMD_OK;
    auto spread = [&](const std::vector<Buffers>& at, int64_t r, int64_t c, int64_t ld) {
      for (const auto& b : at)
        for (const auto& o : b.others)
          if ((st = copy_rows(b.first, o, r, c, ld, ld, stream)) != GSPMD_OK) return st;
      return static_cast<int32_t>(GSPMD_OK);
    };
    if (l.dx && (st = spread(dx, l.ts, l.M, lddx)) != GSPMD_OK) return st;
    if (l.dw && (st = spread(dw, w_rows, w_cols, lddw)) != GSPMD_OK) return st;
    for (const auto& list : token)
      for (size_t k = 1; k < list.size(); ++k) {
        auto one = [&](float* from, float* to) {
          if (!from || !to || from == to) return static_cast<int32_t>(GSPMD_OK);
          return copy_rows(gspmd_shard_buf{from, GSPMD_F32, 0}, gspmd_shard_buf{to, GSPMD_F32, 0}, 1, l.ts, l.ts, l.ts, stream);
        };
        if ((st = one(list[0].loss, list[k].loss)) != GSPMD_OK || (st = one(list[0].lse, list[k].lse)) != GSPMD_OK) return st;
      }
    return GSPMD_OK;
  };

  auto rows_args = [&](SoftmaxRows* a, float* z, int64_t at, int64_t i0, int64_t shards) {      // for rows of tokens `at` .. of all, the first of them in shard i0
    std::memset(a, 0, sizeof(*a));
    for (int64_t i = 0; i < shards; ++i) {
      const gspmd_token_buf& tb = token[static_cast<size_t>(i0 + i)][0];
      a->shard[i] = TokenShard{tb.ids, teacher ? tb.logits : nullptr, tb.weights, tb.loss, tb.lse};
    }
    a->z = z;
    a->ldz = l.ldz();
    a->first = static_cast<int32_t>(at);
    a->tokens = static_cast<int32_t>(l.T);
    a->per_shard = static_cast<int32_t>(l.ts);
    a->first_shard = static_cast<int32_t>(i0);
    a->cols = static_cast<int32_t>(l.cols());
    a->vocab = static_cast<int32_t>(l.V);
    a->per = static_cast<int32_t>(l.vs);
    a->per_cols = static_cast<int32_t>(l.per_cols());
    a->by_cols = fast_div(static_cast<uint32_t>(l.per_cols()));
    a->targets = targets;
    a->inv_tau = 1.f / tau;
    a->logits_bf16 = teacher && tokens[0].logits_dtype == GSPMD_BF16;
  };

  // ---- a handful of tokens: kernels of their own, all tokens at once
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & (kWsAlign - 1))) return GSPMD_ERR_WORKSPACE;
  bool w_padded = true;
  for (int64_t j = 0; j < l.windows(); ++j) w_padded = w_padded && padded(w[static_cast<size_t>(j)].first, ldw);
  const bool may_be_small = l.small() && targets <= kSmallTargets && !a_product_is_pinned();
  if (!(may_be_small && workspace_bytes >= l.bytes(l.T)) && l.few_takes(w_padded && ldw * l.esize() % 128 == 0) && workspace_bytes >= l.few_bytes()) {
    if (dry) return GSPMD_OK;
    FewTokens a;
    std::memset(&a, 0, sizeof(a));
    AddUp sums;
    std::memset(&sums, 0, sizeof(sums));
    SoftmaxRows rows;
    a.z = static_cast<float*>(workspace);
    rows_args(&rows, a.z, 0, 0, l.na);
    for (int64_t j = 0; j < l.nb; ++j) {
      a.w[j] = w[static_cast<size_t>(j)].first.data;
      a.dw[j] = l.dw ? dw[static_cast<size_t>(j)].first.data : nullptr;
    }
    for (int64_t n = 0; n < kFewMost; ++n) {
      const int64_t t = std::min(n, l.T - 1);
      a.x[n] = static_cast<const char*>(x[static_cast<size_t>(t / l.ts)].first.data) + t % l.ts * ldx_in * l.esize();
    }
    a.sums = l.dx ? a.z + round_up(l.T * l.ldz() * 4, kWsAlign) / 4 : nullptr;
    a.ldz = l.ldz();
    a.ldw = ldw;
    a.lddw = lddw;
    a.ld_sum = l.ld_sum();
    a.tokens = static_cast<int32_t>(l.T);
    a.M = static_cast<int32_t>(l.M);
    a.vocab = static_cast<int32_t>(l.V);
    a.per = static_cast<int32_t>(l.vs);
    a.per_cols = static_cast<int32_t>(l.per_cols());
    a.shards = static_cast<int32_t>(l.nb);
    a.lanes = static_cast<int32_t>(l.few_lanes());
    for (int64_t i = 0; l.dx && i < l.na; ++i) sums.to[i] = dx[static_cast<size_t>(i)].first.data;
    sums.ld_out = lddx;
    sums.rows = static_cast<int32_t>(l.na * l.ts);
    sums.cols = a.M;
    sums.tokens = a.tokens;
    sums.per_row = static_cast<int32_t>(l.ts);
    st = l.dtype == GSPMD_BF16 ? run_few<bf16_bits>(l, a, rows, sums, stream) : run_few<float>(l, a, rows, sums, stream);
    return st != GSPMD_OK ? st : spread_results();
  }

  // ---- pieces: as many tokens as the workspace holds (more than the query asks for is not used)
  int64_t rows = l.most_rows();
  if (l.bytes(rows) > workspace_bytes) {
    int64_t fit = 0;                            // the most that fit (bytes() does not grow evenly: ranges fall as rows grow, so every size is looked at by halves)
    for (int64_t step = rows; step > 0; step /= 2)
      while (fit + step < rows && l.bytes(fit + step) <= workspace_bytes) fit += step;
    if (fit == 0 && l.T > 0) return GSPMD_ERR_WORKSPACE;
    rows = fit;
  }
  int64_t pieces = rows > 0 ? (l.T + rows - 1) / rows : 1;
  if (pieces > 1) {                             // even ones, in whole tiles where that makes no more of them
    const int64_t even = (l.T + pieces - 1) / pieces, up = round_up(even, 256), next = up < rows ? up : even;
    if (l.bytes(next) <= workspace_bytes) rows = next;
    pieces = (l.T + rows - 1) / rows;
  }
  char* ws = static_cast<char*>(workspace);
  auto take = [&](int64_t bytes) {
    char* at = ws;
    ws += bytes;
    return at;
  };
  void* const tables = take(l.table_bytes());
  char* const x_all = take(l.x_bytes(rows));
  float* const z = reinterpret_cast<float*>(take(l.z_bytes(rows)));
  float* const sums = reinterpret_cast<float*>(take(l.sum_bytes(rows)));
  float* const dw_sums = reinterpret_cast<float*>(take(l.dw_bytes(rows)));
  int64_t room = workspace_bytes - (ws - static_cast<char*>(workspace));
  const bool join_dw = pieces == 1 && l.joins_dw() && room >= l.joined_dw_bytes();
  float* const dw_parts = reinterpret_cast<float*>(take(join_dw ? l.joined_dw_bytes() : 0));
  room -= join_dw ? l.joined_dw_bytes() : 0;
  char* const w_all = ws;
  const int64_t e = l.esize(), ldz = l.ldz(), ldd = ldz * 4 / e, per_cols = l.per_cols(), nw = l.windows(), vec = 16 / e;
  const bool lost = l.with_lost(), small = may_be_small && pieces == 1;

  Packs packs;
  packs.dtype = l.dtype;
  packs.stream = stream;
  // ---- the vocabulary matrix: shard by shard, or in one padded copy of all of them (zeros between)
  struct Window { const char* data; int64_t ld, col, entries; };
  std::vector<Window> windows;
  bool x_padded = true;
  for (int64_t i = 0; i < l.na; ++i) x_padded = x_padded && padded(x[static_cast<size_t>(i)].first, ldx_in);
  if (!small && ((!w_padded && l.packing_pays()) || l.joining_pays()) && room >= l.packed_w_bytes() && l.M > 0) {
    const int64_t ld = vocab_dim == 0 ? l.ldx() : ldz, chunks = ld / vec;
    for (int64_t from = 0; from < nw && !dry; from += kInlineTokenShards) {
      const int64_t n = std::min<int64_t>(kInlineTokenShards, nw - from);
      PackRows a;
      std::memset(&a, 0, sizeof(a));
      for (int64_t j = 0; j < n; ++j) a.from[j] = w[static_cast<size_t>(from + j)].first.data;
      a.ld = ld;
      a.ld_from = ldw;
      a.copies = 1;
      a.per_cols = static_cast<int32_t>(per_cols);
      a.per = static_cast<int32_t>(l.vs);
      if (vocab_dim == 0) {                     // a shard's rows are per_cols apart
        a.to = w_all + from * per_cols * ld * e;
        a.rows = static_cast<int32_t>(n * per_cols);
        a.chunks = static_cast<int32_t>(chunks);
        a.total = static_cast<int32_t>(l.V - from * l.vs);
        a.per_row = static_cast<int32_t>(per_cols);
        a.cols = static_cast<int32_t>(l.M);
      } else {
        a.to = w_all + from * per_cols * e;
        a.rows = static_cast<int32_t>(l.M);
        a.chunks = static_cast<int32_t>(n * per_cols / vec);
        a.by_columns = 1;
        a.cols = static_cast<int32_t>(l.V - from * l.vs);
      }
      if ((st = packs.add(a)) != GSPMD_OK) return st;
    }
    windows.push_back(Window{w_all, ld, 0, l.cols()});
  } else {
    for (int64_t j = 0; j < nw; ++j) windows.push_back(Window{static_cast<const char*>(w[static_cast<size_t>(j)].first.data), ldw, j * per_cols, l.valid_v(j)});
  }
  auto w_from = [&](const Window& v, int64_t entry) { return v.data + (vocab_dim == 0 ? entry * v.ld : entry) * e; };
  // x put together: where dw sums over tokens of several shards, or over both parts of D, where shards have so few tokens that each would read the vocabulary matrix for
  // itself (15 tokens in two shards, 8099 x 124058: 690 us so), and where rows are not padded
  const bool copied_x = lost && l.dw && l.na == 1;           // by the row kernel, beside D: only dw needs it
  const bool pack_x = l.M > 0 && !copied_x && ((l.dw && l.na > 1 && !(join_dw && l.ranges_by_shard())) || (l.na > 1 && l.ts < kFewRows) || (!x_padded && l.packing_pays()));

  // dw of a piece: straight into its shards, over several pieces in float32, or over ranges of the tokens in float32 for all shards together
  auto make_dw = [&](int64_t piece, int64_t first, int64_t n, bool put_together) -> int32_t {
    const bool last = piece == pieces - 1;
    const char* const d = reinterpret_cast<const char*>(z);
    std::vector<Problem> ps;
    if (join_dw) {
      const int64_t ldx = put_together ? l.ldx() : ldx_in, k = n * l.parts(), entries = l.cols();
      const int64_t span = l.ranges_by_shard() ? l.ts : std::max<int64_t>(k, 1), parts = l.ranges_by_shard() ? l.dw_parts() / l.na : l.dw_parts(), each = round_up((span + parts - 1) / parts, 64);
      ps.clear();
      for (int64_t at = 0; at < k;) {
        const int64_t i = at / span, here = std::min({each, k - at, (i + 1) * span - at});
        const char *const dr = d + at * ldd * e, *const xr = put_together ? x_all + at * ldx * e : static_cast<const char*>(x[static_cast<size_t>(i)].first.data) + (at - i * span) * ldx * e;
        float* const c = dw_parts + static_cast<int64_t>(ps.size()) * l.dw_part();
        at += here;
        ps.push_back(vocab_dim == 0 ? product(dr, ldd, xr, ldx, c, l.ld_dw(), entries, l.M, here, entries, l.M) : product(xr, ldx, dr, ldd, c, l.ld_dw(), l.M, entries, here, l.M, entries));
      }
      const int32_t count_all = static_cast<int32_t>(ps.size());
      if ((st = run_dots(ps, GSPMD_LAYOUT_LHS_K_MAJOR, l.dtype, GSPMD_F32, tables, l.table_bytes(), stream)) != GSPMD_OK) return st;
      for (int64_t from_shard = 0; from_shard < l.nb && !dry; from_shard += kInlineTokenShards) {
        const int64_t shards = std::min<int64_t>(kInlineTokenShards, l.nb - from_shard), before = from_shard * per_cols;
        AddUp a;
        std::memset(&a, 0, sizeof(a));
        for (int64_t j = 0; j < shards; ++j) a.to[j] = dw[static_cast<size_t>(from_shard + j)].first.data;
        a.partials = dw_parts + (vocab_dim == 0 ? before * l.ld_dw() : before);
        a.stride = l.dw_part();
        a.ld_in = l.ld_dw();
        a.ld_out = lddw;
        a.count = count_all;
        a.apart = static_cast<int32_t>(per_cols);
        a.per_row = static_cast<int32_t>(l.vs);
        a.first = static_cast<int32_t>(from_shard * l.vs);
        a.first_shard = static_cast<int32_t>(from_shard);
        a.tokens = static_cast<int32_t>(l.V);
        a.by_columns = vocab_dim;
        a.rows = static_cast<int32_t>(vocab_dim == 0 ? shards * l.vs : l.M);
        a.cols = static_cast<int32_t>(vocab_dim == 0 ? l.M : shards * per_cols);
        if ((st = launch_add_up(a, l.dtype, stream)) != GSPMD_OK) return st;
      }
    } else if (l.dw) {
      const char* const from = put_together ? x_all : static_cast<const char*>(x[0].first.data) + first * ldx_in * e;
      const int64_t ldx = put_together ? l.ldx() : ldx_in, k = n * l.parts(), ld_part = round_up(w_cols, 4);
      ps.clear();
      for (int64_t j = 0; j < l.nb; ++j) {
        const gspmd_shard_buf& o = dw[static_cast<size_t>(j)].first;
        void* const c = pieces == 1 ? o.data : dw_sums + (j * 2 + (piece > 0 ? 1 : 0)) * l.dw_size();
        const int64_t ldc = pieces == 1 ? lddw : ld_part, entries = l.valid_v(j);
        const char* const dj = d + j * per_cols * e;
        ps.push_back(vocab_dim == 0 ? product(dj, ldd, from, ldx, c, ldc, entries, l.M, k, w_rows, w_cols) : product(from, ldx, dj, ldd, c, ldc, l.M, entries, k, w_rows, w_cols));
      }
      if ((st = run_dots(ps, GSPMD_LAYOUT_LHS_K_MAJOR, l.dtype, pieces == 1 ? l.dtype : static_cast<int32_t>(GSPMD_F32), tables, l.table_bytes(), stream)) != GSPMD_OK) return st;
      for (int64_t j = 0; piece > 0 && j < l.nb; ++j) {
        const gspmd_shard_buf& o = dw[static_cast<size_t>(j)].first;
        float* const sum = dw_sums + j * 2 * l.dw_size();
        if ((st = run_sum({sum, sum + l.dw_size()}, w_rows, w_cols, ld_part, last ? o.data : sum, last ? lddw : ld_part, last ? l.dtype : static_cast<int32_t>(GSPMD_F32),
                          stream)) != GSPMD_OK) return st;
      }
    }
    return GSPMD_OK;
  };
  // ---- all in one launch, but for dw's sum over more tokens than a workgroup's
  if (small) {
    const bool in_one = l.T <= kSmallTokens, dw_after = l.dw && !in_one;
    const bool copies = dw_after && (lost || (l.na > 1 && !(join_dw && l.ranges_by_shard())) || (!x_padded && l.packing_pays()));
    SmallLoss a;
    std::memset(&a, 0, sizeof(a));
    rows_args(&a.rows, dw_after ? z : nullptr, 0, 0, l.na);
    a.rows.lost = l.T;
    a.rows.ldx = ldx_in;
    a.rows.x_copies = copies ? reinterpret_cast<bf16_bits*>(x_all) : nullptr;
    a.rows.ld_copy = l.ldx();
    for (int64_t j = 0; j < l.nb; ++j) {
      a.w[j] = w[static_cast<size_t>(j)].first.data;
      a.dw[j] = l.dw && in_one ? dw[static_cast<size_t>(j)].first.data : nullptr;
    }
    for (int64_t i = 0; i < l.na; ++i) {
      a.x[i] = x[static_cast<size_t>(i)].first.data;
      a.dx[i] = l.dx ? dx[static_cast<size_t>(i)].first.data : nullptr;
    }
    a.ldw = ldw;
    a.lddw = lddw;
    a.lddx = lddx;
    a.M = static_cast<int32_t>(l.M);
    a.shards = static_cast<int32_t>(l.nb);
    a.token_shards = static_cast<int32_t>(l.na);
    a.lost = lost;
    if (!dry && (st = l.dtype == GSPMD_BF16 ? launch_small<bf16_bits>(a, l, stream) : launch_small<float>(a, l, stream)) != GSPMD_OK) return st;
    if (dw_after && (st = make_dw(0, 0, l.T, copies)) != GSPMD_OK) return st;
    return spread_results();
  }

  for (int64_t piece = 0; piece < pieces; ++piece) {
    const int64_t first = piece * rows, n = std::min(rows, l.T - first);       // tokens
    const bool last = piece == pieces - 1;
    const int64_t end = last ? l.na * l.ts : first + n;                        // .. and with the last ones the padding of all shards
    // the token shards that rows first .. end of all of them lie in: (shard, first row in it, rows)
    auto each_shard = [&](auto&& go) {
      for (int64_t at = first; at < end;) {
        const int64_t i = at / l.ts, stop = std::min(end, (i + 1) * l.ts);
        if (const int32_t s = go(i, at - i * l.ts, stop - at, at - first); s != GSPMD_OK) return s;
        at = stop;
      }
      return static_cast<int32_t>(GSPMD_OK);
    };
    // launches whose tables hold so many shards: (first row of all, rows, first shard, shards)
    auto by_tables = [&](auto&& go) {
      for (int64_t at = first; at < end && !dry;) {
        const int64_t i = at / l.ts, shards = std::min<int64_t>(kInlineTokenShards, l.na - i), stop = std::min(end, (i + shards) * l.ts);
        if (const int32_t s = go(at, stop - at, i, shards); s != GSPMD_OK) return s;
        at = stop;
      }
      return static_cast<int32_t>(GSPMD_OK);
    };
    if (pack_x)
      st = by_tables([&](int64_t at, int64_t count, int64_t i0, int64_t shards) -> int32_t {
        PackRows a;
        std::memset(&a, 0, sizeof(a));
        for (int64_t i = 0; i < shards; ++i) a.from[i] = x[static_cast<size_t>(i0 + i)].first.data;
        a.ld_from = ldx_in;
        a.to = x_all + (at - first) * l.ldx() * e;
        a.ld = l.ldx();
        a.rows = static_cast<int32_t>(std::min(count, first + n - at));
        a.chunks = static_cast<int32_t>(l.ldx() / vec);
        a.first = static_cast<int32_t>(at);
        a.total = static_cast<int32_t>(l.T);
        a.per_row = a.per = static_cast<int32_t>(l.ts);
        a.first_shard = static_cast<int32_t>(i0);
        a.cols = static_cast<int32_t>(l.M);
        a.copies = lost && l.dw ? 2 : 1;
        a.apart = static_cast<int32_t>(n);
        return packs.add(a);
      });
    if (st != GSPMD_OK || (st = packs.flush()) != GSPMD_OK) return st;
    // ---- logits.  Where they need not be kept (without gradients) their tiles end in what the losses need of them.
    const int64_t groups = (l.cols() + 63) / 64, pair_bytes = round_up(groups * n * 8, kWsAlign), target_bytes = round_up(n * targets * 4, kWsAlign);
    bool stats = !l.dx && !l.dw && l.dtype == GSPMD_BF16 && l.M > 0 && n > 0 && per_cols % 64 == 0 && targets <= kStatsTargets && pair_bytes + 2 * target_bytes <= l.z_bytes(rows);
    const int32_t logits_layout = vocab_dim == 0 ? GSPMD_LAYOUT_RHS_K_CONTIGUOUS : 0;
    std::vector<Problem> ps;
    auto logits = [&](const char* from, int64_t ld, int64_t row, int64_t count) {
      const bool one = windows.size() == 1;                  // one copy of all shards, zeros between: one product; but what lies between is no entry of the vocabulary
      for (int64_t j = 0; j < (one && !stats ? 1 : nw); ++j) {
        const Window& v = windows[one ? 0 : static_cast<size_t>(j)];
        const int64_t entries = one && !stats ? v.entries : l.valid_v(j);
        ps.push_back(product(from, ld, w_from(v, one ? j * per_cols : 0), v.ld, z + row * ldz + j * per_cols, ldz, count, entries, l.M, count, entries));
      }
    };
    auto all_logits = [&] {
      ps.clear();
      if (pack_x) {
        logits(x_all, l.ldx(), 0, n);
        return;
      }
      each_shard([&](int64_t i, int64_t at, int64_t count, int64_t row) -> int32_t {
        const int64_t valid = std::min(count, n - row);
        if (valid > 0) logits(static_cast<const char*>(x[static_cast<size_t>(i)].first.data) + at * ldx_in * e, ldx_in, row, valid);
        return GSPMD_OK;
      });
    };
    all_logits();
    if (stats && !takes_stats(ps, logits_layout, n * ldz * 4 >= kLongLogits)) {
      stats = false;
      all_logits();
    }
    if (stats) {
      char* const base = reinterpret_cast<char*>(z);
      const bool own_ids = l.na == 1 && nw == 1;             // they are the columns
      int32_t* const columns = own_ids ? const_cast<int32_t*>(token[0][0].ids) + first * targets : reinterpret_cast<int32_t*>(base + pair_bytes);
      float* const of_targets = reinterpret_cast<float*>(base + pair_bytes + target_bytes);
      for (Problem& p : ps) {
        const int64_t at = static_cast<float*>(p.C) - z;
        p.join_first = static_cast<int32_t>(at / ldz);
        p.join_slot = static_cast<int32_t>(at % ldz);
        p.C = z;
        p.ldc = static_cast<int32_t>(n);
      }
      auto merge_args = [&](SoftmaxMerge* m, int64_t at, int64_t i0, int64_t shards) {
        rows_args(&m->rows, z + (at - first) * 2, at, i0, shards);
        m->rows.ldz = n;
        m->rows.cols = static_cast<int32_t>(groups);
        m->columns = columns + (at - first) * targets;
        m->end = static_cast<int32_t>(l.cols());
        m->logits = of_targets + (at - first) * targets;
      };
      if (!own_ids) st = by_tables([&](int64_t at, int64_t count, int64_t i0, int64_t shards) -> int32_t {
        SoftmaxMerge m;
        merge_args(&m, at, i0, shards);
        m.count = static_cast<int32_t>(std::max<int64_t>(0, std::min(count, first + n - at)));
        const int64_t total = m.count * static_cast<int64_t>(targets);
        if (total == 0) return GSPMD_OK;
        hipLaunchKernelGGL(target_columns_kernel, dim3(static_cast<unsigned>(std::min<int64_t>((total + 255) / 256, 4096))), dim3(256), 0, stream, m);
        return launched();
      });
      if (st != GSPMD_OK) return st;
      const SoftmaxFinish finish{columns, of_targets, targets, kLog2e / tau};
      if ((st = run_stats(ps, logits_layout, finish, tables, l.table_bytes(), stream)) != GSPMD_OK) return st;
      st = by_tables([&](int64_t at, int64_t count, int64_t i0, int64_t shards) -> int32_t {
        SoftmaxMerge m;
        merge_args(&m, at, i0, shards);
        m.count = static_cast<int32_t>(count);
        if (count >= 4096) hipLaunchKernelGGL((softmax_merge_kernel<16>), dim3(static_cast<unsigned>((count + 15) / 16)), dim3(kMergeThreads), 0, stream, m);
        else hipLaunchKernelGGL((softmax_merge_kernel<4>), dim3(static_cast<unsigned>((count + 3) / 4)), dim3(kMergeThreads), 0, stream, m);
        return launched();
      });
      if (st != GSPMD_OK) return st;
      continue;
    }
    if ((st = run_dots(ps, logits_layout, l.dtype, GSPMD_F32, tables, l.table_bytes(), stream)) != GSPMD_OK) return st;
    // ---- rows
    st = by_tables([&](int64_t at, int64_t count, int64_t i0, int64_t shards) {
      SoftmaxRows a;
      rows_args(&a, z + (at - first) * ldz, at, i0, shards);
      a.lost = n;
      if (copied_x) {
        a.x = static_cast<const bf16_bits*>(x[0].first.data);
        a.x_copies = reinterpret_cast<bf16_bits*>(x_all);
        a.ldx = ldx_in;
        a.ld_copy = l.ldx();
        a.x_cols = static_cast<int32_t>(l.M);
      }
      return launch_rows(a, l, count, stream);
    });
    if (st != GSPMD_OK) return st;
    const char* const d = reinterpret_cast<const char*>(z);
    // ---- dx: the piece's rows
    const int32_t dx_layout = vocab_dim == 0 ? 0 : GSPMD_LAYOUT_RHS_K_CONTIGUOUS;
    const int64_t ranges = windows.size() == 1 ? l.ranges(rows) : l.ranges_of_shard(rows);
    if (l.dx && !lost && windows.size() == 1 && ranges == 1) {
      ps.clear();
      const Window& v = windows[0];
      each_shard([&](int64_t i, int64_t at, int64_t count, int64_t row) -> int32_t {
        const gspmd_shard_buf& o = dx[static_cast<size_t>(i)].first;
        ps.push_back(product(d + row * ldz * 4, ldd, v.data, v.ld, static_cast<char*>(o.data) + at * lddx * e, lddx, std::min(count, n - row), l.M, v.entries, count, l.M));
        return GSPMD_OK;
      });
      if ((st = run_dots(ps, dx_layout, l.dtype, l.dtype, tables, l.table_bytes(), stream)) != GSPMD_OK) return st;
    } else if (l.dx && l.M > 0) {
      ps.clear();
      const int64_t both = n * l.parts(), size = both * l.ld_sum();
      for (const Window& v : windows) {
        const int64_t each = round_up((v.entries + ranges - 1) / ranges, 256);
        for (int64_t from = 0; from < v.entries; from += each)
          ps.push_back(product(d + (v.col + from) * e, ldd, w_from(v, from), v.ld, sums + static_cast<int64_t>(ps.size()) * size, l.ld_sum(), both, l.M,
                               std::min(each, v.entries - from), both, l.M));
      }
      const int64_t count_all = static_cast<int64_t>(ps.size()) * l.parts();
      if (n > 0 && (st = run_dots(ps, dx_layout, l.dtype, GSPMD_F32, tables, l.table_bytes(), stream)) != GSPMD_OK) return st;
      st = by_tables([&](int64_t at, int64_t count, int64_t i0, int64_t shards) {
        AddUp a;
        std::memset(&a, 0, sizeof(a));
        for (int64_t i = 0; i < shards; ++i) a.to[i] = dx[static_cast<size_t>(i0 + i)].first.data;
        a.partials = sums + (at - first) * l.ld_sum();
        a.stride = n * l.ld_sum();
        a.ld_in = l.ld_sum();
        a.ld_out = lddx;
        a.count = static_cast<int32_t>(count_all);
        a.rows = static_cast<int32_t>(count);
        a.cols = static_cast<int32_t>(l.M);
        a.first = static_cast<int32_t>(at);
        a.tokens = static_cast<int32_t>(l.T);
        a.per_row = a.apart = static_cast<int32_t>(l.ts);
        a.first_shard = static_cast<int32_t>(i0);
        return launch_add_up(a, l.dtype, stream);
      });
      if (st != GSPMD_OK) return st;
    }
    if ((st = make_dw(piece, first, n, pack_x || copied_x)) != GSPMD_OK) return st;
  }
  return spread_results();
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
  const int64_t rows = l.most_rows();
  *bytes = l.bytes(rows) + (l.packing_pays() || l.joining_pays() ? l.packed_w_bytes() : 0) + (rows == l.T ? l.joined_dw_bytes() : 0);
  if (l.few()) *bytes = std::max(*bytes, l.few_bytes());
  if (least) *least = std::min(*bytes, l.bytes(std::min<int64_t>(l.T, 1)));
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
