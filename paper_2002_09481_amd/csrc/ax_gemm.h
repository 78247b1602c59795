// Matrix products of the feed-forward operators: what ax_gemm.hip computes and how it is asked for.
#pragma once

#include "ax_internal.h"

namespace ax {

typedef __bf16 bf16;

// One factor pair of a product.  b2: the second projection of a gated pair, or the second right operand of a
// launch that computes two outputs from one left operand.
struct GemmSeg {
  const void* a;
  const void* b;
  const void* b2;
};

constexpr int kMaxSegs = 2;  // two in the gated block's input gradient

// y[M,N] = epilogue(sum over the segments of a[M,K] b[K,N]).
struct GemmArgs {
  GemmSeg seg[kMaxSegs];
  int nseg;
  int i8;         // 1: operands are int8 codes, sums int32; 0: bf16, sums float32
  int pieces;     // 3: float32 operands as three bf16 matrices each, a_plane and b_plane bytes apart; else 1
  int la, lb;     // operand layouts: 0 = the contraction is contiguous (a [M,K], b [N,K]), 1 = it is the row index (a [K,M], b [K,N])
  int M, N, K;
  long long lda, ldb;  // row pitches in bytes, multiples of 16
  long long a_plane, b_plane;
  int gated;      // h = act(a b) * (a b2)
  int dual;       // y = a b, y2 = a b2
  // epilogue
  int odt;        // type of everything below (AX_F32 or AX_BF16)
  int act;
  void* y;        // [M,N], rows of ldy elements
  void* y2;       // dual: the second output
  void* z;        // may be NULL: value before the activation (gated: the gate projection); rows of N elements
  void* z2;       // gated, may be NULL: the other projection
  const void* bias;  // may be NULL
  const void* res;   // may be NULL: added after the activation, rows of ldr elements
  long long ldy, ldr;
  const float* xs;   // int8: scale of every row of a, of every column of b, of b2
  const float* ws;
  const float* ws2;
};

// How a launch is cut: tile configuration, and slices of the contraction whose partial sums a second kernel adds.
struct GemmPlan {
  int tile;
  int splits;
  size_t part_bytes;  // partial sums (0 without slices)
};

GemmPlan plan_gemm(const GemmArgs& g);
void tile_of(const GemmArgs& g, const GemmPlan& p, int* rows, int* cols);
hipError_t launch_gemm(const GemmArgs& g, const GemmPlan& p, void* part, hipStream_t s);
// y from the partial sums [splits][planes][M][N rounded up to 8] of the slices, with the epilogue.
hipError_t launch_join(const GemmArgs& g, int splits, void* part, hipStream_t s);

// Products of rows grouped by expert (ax_gemm_experts.hip).  offsets [experts + 1] (device; null: one expert, all rows) are the
// experts' first rows; the experts' right operands lie one behind the other.  sums false: rows of a times the matrix of their
// expert, g.M = rows.  sums true: for every expert a^T b over its rows, g.K = rows, results one behind the other.  No slices,
// bf16 operands or pieces, results of the operands' type.
// index (rows by rows of bf16 alone; null: none): row of a for each of the rows, a has x_rows of them, in less than 2 GB.
struct Groups {
  const int32_t* offsets;
  int experts, rows;
  const int32_t* index;
  int x_rows;
};
int plan_experts(const GemmArgs& g, const Groups& e, bool sums);  // the tile configuration
bool experts_fit(const GemmArgs& g, const Groups& e, bool sums, int tile);  // whether its tiles are as many as one launch can have
void tile_of_experts(const GemmArgs& g, bool sums, int tile, int* rows, int* cols, int* per_cu);
hipError_t launch_gemm_experts(const GemmArgs& g, const Groups& e, bool sums, int tile, hipStream_t s);

// Products of few rows straight from the operands in their own type, at any element: int8 (g.i8), or dtype AX_BF16 or
// AX_F32.  g as above; seg holds the operands themselves, la is 0, dual is not taken.  Meant for up to 64 rows.
struct FewPlan {
  int slices;
  size_t part_bytes;
};
FewPlan plan_few(const GemmArgs& g, int dtype);
hipError_t launch_few(const GemmArgs& g, int dtype, const FewPlan& p, void* part, hipStream_t s);

// Few rows an expert, forward only: rows index[r] of x (null: row r; x_rows there are) straight from the operands.  g.M = rows.
hipError_t launch_few_experts(const GemmArgs& g, int dtype, const Groups& e, const int32_t* index, int x_rows, hipStream_t s);

}  // namespace ax
