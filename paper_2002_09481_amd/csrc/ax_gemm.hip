// Matrix products on the matrix cores: bf16 operands with float32 sums, int8 codes with int32 sums.
//
// A workgroup computes a tile of the result, 256 x 256 where the product is large: the two operands' parts of a stage meet
// 256 times each, so that memory and L2 keep up.  Copies go from memory to LDS past the registers; LDS is laid out so that
// neither plain nor transposing reads meet in a bank, which lets every operand be read as it lies.  Bound, large products: by
// the power that the card draws with random operands (the matrix cores are busy 65 % of the time; with zeros for operands
// the same product takes 692 us instead of 843).  Smaller ones: rounds of tiles that leave compute units idle,
// and each tile's first stage and stores, during which nothing multiplies.
//
// Measured (us): bf16 8192^3 815 to 930 (1180 to 1350 TF), 4096^3 103 to 110 (1250 to 1340 TF), gradient of a weight 8192^3 780 to
// 805 (1365 to 1400 TF);
// gated 8192 x 4096 -> 16384 with both projections stored 1735 to 1800 (1220 to 1270 TF); int8 8192^3 465 to 520 (2100 to 2370 TOP);
// float32 4096^3 690 to 700 (196 to 199 TF, six products each).
#include <algorithm>

#include "ax_gemm_tile.h"

namespace ax {
namespace {

// The slices' sums in their order, four loads at a time.
template <bool I8>
__device__ __forceinline__ f32x4 sum_slices(const float* p, long long step, int n) {
  typedef typename Acc<I8>::T T;
  T t = *(const T*)p;
  int k = 1;
  for (; k + 4 <= n; k += 4) {
    const T a = *(const T*)(p + k * step), b = *(const T*)(p + (k + 1) * step), c = *(const T*)(p + (k + 2) * step),
            d = *(const T*)(p + (k + 3) * step);
    t = t + a + b + c + d;
  }
  for (; k < n; ++k) t += *(const T*)(p + k * step);
  return __builtin_bit_cast(f32x4, t);
}

// Partial sums of the slices, added in their order, and the epilogue: eight columns a thread.  Bound by memory, a launch's
// latency where the sums are few (333 x 2048 in five slices 5 us, 4101 x 2048 in three 29).
template <bool I8, bool GATED>
__global__ __launch_bounds__(256) void gemm_join_kernel(const Args a) {
  const GemmArgs& g = a.g;
  const int groups = (int)(a.ldp >> 3);
  const int planes = GATED || g.dual ? 2 : 1;
  const int outs = g.dual ? 2 : 1;
  const long long plane = (long long)g.M * a.ldp;
  const long long total = (long long)outs * g.M * groups;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const int second = i >= (long long)g.M * groups;
    const long long r = i - (second ? (long long)g.M * groups : 0);
    const int m = (int)(r / groups), n = (int)(r - (long long)m * groups) * 8;
    Columns cols;
    load_columns<I8, GATED, kAnyOut>(g, n, cols);
    Ahead ahead;
    look_ahead<I8, GATED, kAnyOut>(g, m, n, ahead);
    f32x4 s[2][2];
#pragma unroll
    for (int pl = 0; pl < (GATED ? 2 : 1); ++pl)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float* p = a.part + (long long)(second + pl) * plane + (long long)m * a.ldp + n + 4 * h;
        s[pl][h] = sum_slices<I8>(p, (long long)planes * plane, a.splits);
      }
    finish<I8, GATED, kAnyOut>(g, cols, ahead, m, n, s[0], s[GATED ? 1 : 0], second);
  }
}

template <bool I8, int LA, int LB, int NB, int OT>
void launch_out(const Args& a, int tile, int grid, hipStream_t s) {
  switch (tile) {
    case 0: gemm_kernel<I8, 1, LA, LB, NB, 256, 256, 2, 4, 128, 2, 2, OT><<<grid, 512, 0, s>>>(a); break;
    case 1: gemm_kernel<I8, 1, LA, LB, NB, 128, 128, 2, 2, 128, 2, 2, OT><<<grid, 256, 0, s>>>(a); break;
    case 2: gemm_kernel<I8, 1, LA, LB, NB, 64, 128, 1, 4, 128, 3, 2, OT><<<grid, 256, 0, s>>>(a); break;
    default:  // (copies of 32 columns whose rows are the contraction would not fill the threads)
      if constexpr (LA == 0) gemm_kernel<I8, 1, LA, LB, NB, 32, 128, 1, 4, 128, 3, 2, OT><<<grid, 256, 0, s>>>(a);
      break;
  }
}
template <bool I8, int LA, int LB, int NB>
void launch_tile(const Args& a, int tile, int grid, hipStream_t s) {
  if constexpr (LA == 0) {  // (the weight's gradient has the operands' type)
    if (a.g.odt == AX_F32) return launch_out<I8, LA, LB, NB, AX_F32>(a, tile, grid, s);
  }
  launch_out<I8, LA, LB, NB, AX_BF16>(a, tile, grid, s);
}
template <int LA, int LB, int NB, int OT>
void launch_out3(const Args& a, int tile, int grid, hipStream_t s) {
  if constexpr (LA == 0 && LB == 0) {
    if (tile == 0) {
      gemm_kernel<false, 3, LA, LB, NB, 128, 128, 2, 4, 64, 3, 2, OT><<<grid, 512, 0, s>>>(a);
      return;
    }
  }
  gemm_kernel<false, 3, LA, LB, NB, 64, 128, 2, 2, 64, 2, 2, OT><<<grid, 256, 0, s>>>(a);
}
template <int LA, int LB, int NB>
void launch_tile3(const Args& a, int tile, int grid, hipStream_t s) {
  if constexpr (LA == 0) {
    if (a.g.odt == AX_BF16) return launch_out3<LA, LB, NB, AX_BF16>(a, tile, grid, s);
  }
  launch_out3<LA, LB, NB, AX_F32>(a, tile, grid, s);
}

constexpr int kMaxSplits = 16;

long long tiles_of(const GemmArgs& g, const TileShape& t) {
  const int bns = t.bn / (g.gated ? 2 : 1);
  return (long long)((g.M + t.bm - 1) / t.bm) * ((g.N + bns - 1) / bns) * (g.dual ? 2 : 1);
}
const TileShape& shape_of(const GemmArgs& g, int tile) { return g.pieces == 3 ? kTiles3[tile] : kTiles[tile]; }
long long part_pitch(const GemmArgs& g) { return ((long long)g.N + 7) / 8 * 8; }

}  // namespace

// The tile configuration and the slices of the contraction with the least estimated time: rounds of workgroups over the
// card, each a fixed part and its stages; the slices' partial sums (written and read once, at 6.5 bytes a picosecond) and the
// launch that adds them.  Large products get the large tiles, few tiles are cut along the contraction.
GemmPlan plan_gemm(const GemmArgs& g) {
  const long long kbytes = (long long)g.K * (g.i8 ? 1 : 2);
  const bool three = g.pieces == 3;
  const double outs = g.gated || g.dual ? 2 : 1;
  GemmPlan best{};
  double least = 1e300;
  for (int t = 0; t < (three ? kNumTiles3 : kNumTiles); ++t) {
    const TileShape& T = shape_of(g, t);
    if (T.bm == 32 && g.la != 0) continue;
    if (three && t == 0 && (g.la != 0 || g.lb != 0)) continue;
    const long long steps = (kbytes + T.kb - 1) / T.kb * g.nseg;
    const long long tiles = tiles_of(g, T);
    const double step = three && t == 1 && g.la == 0 && g.lb == 0 ? kStep3Along : T.step;
    if (t > 0 && tiles > kMaxGrid) continue;
    for (int sp = 1; sp <= kMaxSplits && (sp == 1 || sp * 2 <= steps); ++sp) {
      if (sp > 1 && tiles * sp > kMaxGrid) break;
      const long long n = tiles * sp, slots = (long long)kCus * T.per_cu;
      const long long full = n / slots, rest = n - full * slots;
      const double stages = (double)((steps + sp - 1) / sp) * T.kb / 128;
      const double fixed = T.fixed + (sp > 1 ? T.bm * T.bn * 4 / 20e3 : 0);  // (sums leave a compute unit at 20 KB a us)
      double cost = full * (fixed + stages * step);
      if (rest) cost += fixed + stages * (rest <= kCus ? T.step1 : step);
      if (sp > 1) cost += 3.0 + sp * outs * g.M * (double)g.N * 8.0 / 6.5e6;
      if (cost < least) {
        least = cost;
        best.tile = t;
        best.splits = sp;
      }
    }
  }
  best.part_bytes = best.splits > 1 ? (size_t)best.splits * (size_t)outs * (size_t)g.M * (size_t)part_pitch(g) * 4 : 0;
  return best;
}

void tile_of(const GemmArgs& g, const GemmPlan& p, int* rows, int* cols) {
  const TileShape& T = shape_of(g, p.tile);
  *rows = T.bm;
  *cols = T.bn;
}

hipError_t launch_gemm(const GemmArgs& g, const GemmPlan& p, void* part, hipStream_t s) {
  Args a;
  a.g = g;
  const TileShape& T = shape_of(g, p.tile);
  const int kstep = T.kb / (g.i8 ? 1 : 2);
  a.tiles_m = (g.M + T.bm - 1) / T.bm;
  a.tiles_n = (int)(tiles_of(g, T) / a.tiles_m);
  a.ksteps = (g.K + kstep - 1) / kstep;
  a.splits = p.splits;
  a.part = (float*)part;
  a.ldp = part_pitch(g);
  const long long grid = (long long)a.tiles_m * a.tiles_n * p.splits;
  if (grid <= 0 || grid >= 1 << 23) return hipErrorInvalidValue;
  const int n = (int)grid;
  if (g.pieces == 3) {
    if (g.gated) launch_tile3<0, 1, 2>(a, p.tile, n, s);
    else if (g.la == 0 && g.lb == 0) launch_tile3<0, 0, 1>(a, p.tile, n, s);
    else if (g.la == 0) launch_tile3<0, 1, 1>(a, p.tile, n, s);
    else launch_tile3<1, 1, 1>(a, p.tile, n, s);
  } else if (g.gated) {
    if (g.i8) launch_tile<true, 0, 0, 2>(a, p.tile, n, s);
    else launch_tile<false, 0, 1, 2>(a, p.tile, n, s);
  } else if (g.i8) {
    launch_tile<true, 0, 0, 1>(a, p.tile, n, s);
  } else if (g.la == 0 && g.lb == 0) {
    launch_tile<false, 0, 0, 1>(a, p.tile, n, s);
  } else if (g.la == 0) {
    launch_tile<false, 0, 1, 1>(a, p.tile, n, s);
  } else {
    launch_tile<false, 1, 1, 1>(a, p.tile, n, s);
  }
  const hipError_t rc = hipGetLastError();
  return rc != hipSuccess || p.splits == 1 ? rc : launch_join(g, p.splits, part, s);
}

hipError_t launch_join(const GemmArgs& g, int splits, void* part, hipStream_t s) {
  Args a{};
  a.g = g;
  a.splits = splits;
  a.part = (float*)part;
  a.ldp = part_pitch(g);
  const long long groups = (long long)(g.dual ? 2 : 1) * g.M * (a.ldp / 8);
  const int jg = (int)std::min<long long>((groups + 255) / 256, 8192);
  if (g.i8) g.gated ? gemm_join_kernel<true, true><<<jg, 256, 0, s>>>(a) : gemm_join_kernel<true, false><<<jg, 256, 0, s>>>(a);
  else g.gated ? gemm_join_kernel<false, true><<<jg, 256, 0, s>>>(a) : gemm_join_kernel<false, false><<<jg, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ax
