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

// Products of few rows straight from the operands in their own type, at any element: int8 (g.i8), or dtype AX_BF16 or
// AX_F32.  g as above; seg holds the operands themselves, la is 0, dual is not taken.  Meant for up to 64 rows.
struct FewPlan {
  int slices;
  size_t part_bytes;
};
FewPlan plan_few(const GemmArgs& g, int dtype);
hipError_t launch_few(const GemmArgs& g, int dtype, const FewPlan& p, void* part, hipStream_t s);

}  // namespace ax
