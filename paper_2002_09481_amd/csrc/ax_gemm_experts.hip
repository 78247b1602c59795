// Matrix products of rows grouped by expert: the tiles of ax_gemm_tile.h, each of which looks up whose rows it has.
//
// Bound: few experts with many rows as ax_gemm.hip's tiles.  Many with few: sums by the stores of the weights' gradients, rows by what the
// compute units fetch, and by tiles that the experts' ends leave partly empty.  Measured (us, bf16, experts / rows / inputs / outputs, sizes
// that differ up to 20 times): rows 8/16384/2048/4096 266 (1030 TF), 32/8192/1024/1408 39 (600 TF); sums 8/16384/2048/4096 245 (1120 TF),
// 32/8192/1024/1408 47 (92 MB of results; 3 workgroups a compute unit, with tiles of 256 x 256 54, two workgroups of 128 x 128 56),
// 32/32768/1024/1408 110 (in the order of the experts, larger or not, 160: the launch ends with the tiles of a large one; whole experts an
// XCD, by size in turn, 3 to 8 % faster with 32 or 64 of them and 25 % slower with eight).
//
// Rows by rows (kRows): a tile never spans two experts, so one of 256 rows wastes half of itself at an expert's end on the
// average; the tile's height goes by the rows that an expert can expect.  Sums over rows (kSums, the weights' gradients): one
// product for each expert, with its rows for the contraction; an expert without rows writes zeros.  Nothing is cut along the
// contraction: experts are many, and their sizes are not known where the launch is planned.
#include <algorithm>

#include "ax_gemm_tile.h"

namespace ax {
namespace {

// Configurations of their own.  Tiles of which three fit a compute unit; rows by rows: between the others where one more round of
// two would be needed.  Sums: contractions are short, a workgroup mostly waits for its first stage and for its stores.  And a height between 64
// and 128 rows, where it saves a compute unit its third or fourth tile: 184 products and gradients of 128 to 16384 rows, 1 to 64 experts, 256 to 8192
// inputs and outputs, drawn among those that it is chosen for, take 0.97 of the time without it on the average (101 of them less by more than
// 2 %, 38 more; 0.73 to 1.38, the worst a few hundred rows with weights read in place at a pitch of 8 KB).
constexpr TileShape kThreeRows = {64, 128, 128, 3, 2.5, 0.60, 0.93};
constexpr TileShape kThreeSums = {128, 128, 64, 3, 3.0, 0.90, 1.40};
constexpr TileShape kMiddleRows = {96, 128, 128, 2, 3.0, 0.55, 0.80};
constexpr int kThree = 4, kMiddle = 5;

template <int LA, int LB, int NB, Grouping GR>
void launch_bf16(const Args& a, int tile, int grid, hipStream_t s) {
  constexpr int OT = AX_BF16;
  switch (tile) {
    case 0: gemm_kernel<false, 1, LA, LB, NB, 256, 256, 2, 4, 128, 2, 2, OT, GR><<<grid, 512, 0, s>>>(a); break;
    case 1: gemm_kernel<false, 1, LA, LB, NB, 128, 128, 2, 2, 128, 2, 2, OT, GR><<<grid, 256, 0, s>>>(a); break;
    case 2: gemm_kernel<false, 1, LA, LB, NB, 64, 128, 1, 4, 128, 3, 2, OT, GR><<<grid, 256, 0, s>>>(a); break;
    case kThree:
      if constexpr (GR != kSums) gemm_kernel<false, 1, LA, LB, NB, 64, 128, 1, 4, 128, 2, 3, OT, GR><<<grid, 256, 0, s>>>(a);
      else gemm_kernel<false, 1, LA, LB, NB, 128, 128, 2, 2, 64, 3, 3, OT, GR><<<grid, 256, 0, s>>>(a);
      break;
    case kMiddle:
      if constexpr (GR != kSums) gemm_kernel<false, 1, LA, LB, NB, 96, 128, 1, 4, 128, 2, 2, OT, GR><<<grid, 256, 0, s>>>(a);
      break;
    default:
      if constexpr (LA == 0) gemm_kernel<false, 1, LA, LB, NB, 32, 128, 1, 4, 128, 3, 2, OT, GR><<<grid, 256, 0, s>>>(a);
      break;
  }
}
template <int LA, int LB, int NB, Grouping GR>
void launch_f32(const Args& a, int tile, int grid, hipStream_t s) {
  constexpr int OT = AX_F32;
  if constexpr (LA == 0 && LB == 0 && NB == 1) {
    if (tile == 0) {
      gemm_kernel<false, 3, LA, LB, NB, 128, 128, 2, 4, 64, 3, 2, OT, GR><<<grid, 512, 0, s>>>(a);
      return;
    }
  }
  gemm_kernel<false, 3, LA, LB, NB, 64, 128, 2, 2, 64, 2, 2, OT, GR><<<grid, 256, 0, s>>>(a);
}
template <int LA, int LB, int NB, Grouping GR>
void launch_tiles(const Args& a, int tile, int grid, hipStream_t s) {
  if constexpr (GR == kRows) {
    if (a.index) return launch_bf16<LA, LB, NB, kFound>(a, tile, grid, s);
  }
  if (a.g.pieces == 3) launch_f32<LA, LB, NB, GR>(a, tile, grid, s);
  else launch_bf16<LA, LB, NB, GR>(a, tile, grid, s);
}

const TileShape& shape_of(const GemmArgs& g, bool sums, int tile) {
  if (g.pieces == 3) return kTiles3[tile];
  return tile < kThree ? kTiles[tile] : sums ? kThreeSums : tile == kThree ? kThreeRows : kMiddleRows;
}
long long tiles_across(const GemmArgs& g, const TileShape& T) {
  const int bns = T.bn / (g.gated ? 2 : 1);
  return (long long)((g.N + bns - 1) / bns) * (g.dual ? 2 : 1);
}

// Most tiles that there can be: every expert with rows begins one that it may not fill.
long long grid_of(const GemmArgs& g, const Groups& e, bool sums, const TileShape& T) {
  if (sums) return (long long)e.experts * ((g.M + T.bm - 1) / T.bm) * tiles_across(g, T);
  const long long m = e.offsets ? e.rows / T.bm + std::min<long long>(e.experts, e.rows) : (e.rows + T.bm - 1) / T.bm;
  return m * tiles_across(g, T);
}

}  // namespace

// The tiles with the least estimated time, as plan_gemm, for experts of equal sizes with half a tile's height wasted in each.
int plan_experts(const GemmArgs& g, const Groups& e, bool sums) {
  const bool three = g.pieces == 3;
  const double rows = (double)e.rows, experts = (double)std::max<long long>(1, std::min<long long>(e.experts, e.rows));
  const double kbytes = 2.0 * (sums ? rows / experts : (double)g.K);
  int best = three ? 1 : 0;
  double least = 1e300;
  for (int t = 0; t < (three ? kNumTiles3 : sums ? kThree + 1 : kMiddle + 1); ++t) {
    const TileShape& T = shape_of(g, sums, t);
    if (T.bm == 32 && g.la != 0) continue;
    if (three && t == 0 && (g.la != 0 || g.lb != 0 || g.gated)) continue;
    if (t > 0 && grid_of(g, e, sums, T) > kMaxGrid) continue;
    const double high = sums ? (g.M + T.bm - 1) / T.bm : e.experts == 1 ? (e.rows + T.bm - 1) / T.bm : std::max(1.0, rows / experts / T.bm + 0.5);
    const long long n = (long long)((sums ? e.experts : experts) * high * (double)tiles_across(g, T));
    const double step = three && t == 1 && g.la == 0 && g.lb == 0 ? kStep3Along : T.step;
    const double stages = ((kbytes + T.kb - 1) / T.kb) * g.nseg * T.kb / 128;
    const long long slots = (long long)kCus * T.per_cu, full = n / slots, rest = n - full * slots;
    const double fixed = T.fixed + (sums && !three ? T.per_cu * T.bm * T.bn * 2 / 28e3 : 0);  // (results leave a compute unit at 28 KB a us)
    double cost = full * (fixed + stages * step);
    if (rest) cost += fixed + stages * (rest <= kCus ? T.step1 : step);
    if (cost < least) {
      least = cost;
      best = t;
    }
  }
  return best;
}

bool experts_fit(const GemmArgs& g, const Groups& e, bool sums, int tile) { return grid_of(g, e, sums, shape_of(g, sums, tile)) < 1 << 23; }

void tile_of_experts(const GemmArgs& g, bool sums, int tile, int* rows, int* cols, int* per_cu) {
  *rows = shape_of(g, sums, tile).bm;
  *cols = shape_of(g, sums, tile).bn;
  *per_cu = shape_of(g, sums, tile).per_cu;
}

hipError_t launch_gemm_experts(const GemmArgs& g, const Groups& e, bool sums, int tile, hipStream_t s) {
  Args a{};
  a.g = g;
  const TileShape& T = shape_of(g, sums, tile);
  const int kstep = T.kb / 2;
  a.tiles_m = sums ? (g.M + T.bm - 1) / T.bm : 1;  // (kRows: each expert's own)
  a.tiles_n = (int)tiles_across(g, T);
  a.ksteps = (g.K + kstep - 1) / kstep;
  a.splits = 1;
  a.offsets = e.offsets;
  a.experts = e.experts;
  a.rows = e.rows;
  a.index = e.index;
  a.x_rows = e.x_rows;
  const int n = (int)grid_of(g, e, sums, T);
  if (sums) launch_tiles<1, 1, 1, kSums>(a, tile, n, s);
  else if (g.gated) g.lb == 0 ? launch_tiles<0, 0, 2, kRows>(a, tile, n, s) : launch_tiles<0, 1, 2, kRows>(a, tile, n, s);
  else g.lb == 0 ? launch_tiles<0, 0, 1, kRows>(a, tile, n, s) : launch_tiles<0, 1, 1, kRows>(a, tile, n, s);
  return hipGetLastError();
}

}  // namespace ax
