// The tile kernel of the matrix products (ax_gemm.hip: products of whole matrices; ax_gemm_experts.hip: of rows grouped by
// expert) and the tile configurations that the planners choose from.
#pragma once

#include <type_traits>

#include "ax_float.h"
#include "ax_gemm.h"
#include "ax_group.h"

namespace ax {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

#define AX_INLINE __attribute__((always_inline))
#define AX_LDS(T) __attribute__((address_space(3))) T

constexpr uint32_t kOut = 0x80000000u;  // an offset behind every buffer: the load gives zeros

struct Args {
  GemmArgs g;
  int tiles_m, tiles_n;  // tiles_n counts both outputs of a dual launch
  int ksteps;            // stages per segment
  int splits;
  float* part;           // [splits][planes][M][ldp]
  long long ldp;
  const int32_t* offsets;  // rows grouped by expert: [experts + 1], of their first rows (null: one expert, all rows)
  int experts, rows;
  const int32_t* index;    // kFound: row of the left operand for each row, of x_rows
  int x_rows;
};

// What a launch's tiles belong to: one product, or products of rows grouped by expert, each with its own right operand (kRows;
// kFound: its rows of the left operand are found through an index), or the experts' weight gradients, each a sum over its own rows
// (kSums: the contraction is grouped).
enum Grouping { kWhole, kRows, kFound, kSums };

// ---- epilogue ----------------------------------------------------------------------------------

// Eight columns n .. n + 7 of a row, of which `left` are there.
__device__ __forceinline__ void load8(const void* p, long long i, int dt, int left, float (&v)[8]) {
  if (dt == AX_F32) load_elems<true, 8>(p, i, left, v);
  else load_elems<false, 8>(p, i, left, v);
}
__device__ __forceinline__ void store8(void* p, long long i, int dt, int left, const float (&v)[8]) {
  if (dt == AX_F32) store_elems<true, 8>(p, i, left, v);
  else store_elems<false, 8>(p, i, left, v);
}

// Type of the results, known to the kernel or not.  It decides the form of the activation: with both forms in the epilogue of
// a 256 x 256 tile the compiler no longer unrolls it, and the sums go through scratch memory.
constexpr int kAnyOut = 2;
template <int OT>
__device__ __forceinline__ int out_type(const GemmArgs& g) { return OT == kAnyOut ? g.odt : OT; }

// What the epilogue needs of eight columns, the same for all rows.
struct Columns {
  float bias[8], ws[8], ws2[8];
};
template <bool I8, bool GATED, int OT>
__device__ __forceinline__ void load_columns(const GemmArgs& g, int n, Columns& c) {
  const int left = g.N - n;
  if (!GATED && g.bias) load8(g.bias, n, out_type<OT>(g), left, c.bias);
  if (I8) load_elems<true, 8>(g.ws, n, left, c.ws);
  if (I8 && GATED) load_elems<true, 8>(g.ws2, n, left, c.ws2);
}
// Eight whole columns of the residual as they lie, asked for some rows ahead in int8 products: one row after the other, the
// latencies add up (8192 x 1024 -> 8192 139 us, 177 row by row; bf16 gains 2 % with a residual and loses as much without).
struct Ahead {
  u32x4 q[2];
};
template <bool I8, bool GATED, int OT>
__device__ __forceinline__ void look_ahead(const GemmArgs& g, int m, int n, Ahead& a) {
  if (!I8 || GATED || !g.res || n + 8 > g.N) return;
  const long long i = (long long)m * g.ldr + n;
  if (out_type<OT>(g) == AX_F32) {
    a.q[0] = load_any<u32x4>((const float*)g.res + i);
    a.q[1] = load_any<u32x4>((const float*)g.res + i + 4);
  } else {
    a.q[0] = load_any<u32x4>((const uint16_t*)g.res + i);
  }
}
// Columns n .. n + 7 of row m from their finished sums (GATED: of both projections; int8: sums as integers in s and s2).
// second: the second output of a dual launch.
template <bool I8, bool GATED, int OT>
__device__ __forceinline__ void finish(const GemmArgs& g, const Columns& c, const Ahead& a, int m, int n, const f32x4 (&s)[2], const f32x4 (&s2)[2], int second) {
  const int left = g.N - n, odt = out_type<OT>(g);
  float v[8], u[8];
  const float xs = I8 ? g.xs[m] : 1.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = I8 ? (float)__float_as_int(s[e >> 2][e & 3]) * (xs * c.ws[e]) : s[e >> 2][e & 3];
    if (GATED) u[e] = I8 ? (float)__float_as_int(s2[e >> 2][e & 3]) * (xs * c.ws2[e]) : s2[e >> 2][e & 3];
  }
  if (!GATED && g.bias) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += c.bias[e];
  }
  if (g.z) store8(g.z, (long long)m * g.N + n, odt, left, v);
  if (GATED && g.z2) store8(g.z2, (long long)m * g.N + n, odt, left, u);
  if (odt == AX_F32) apply_act<true>(v, g.act);
  else apply_act<false>(v, g.act);
  if (GATED) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= u[e];
  }
  if (!GATED && g.res) {
    if (!I8 || left < 8) {
      load8(g.res, (long long)m * g.ldr + n, odt, left, u);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        u[e] = odt == AX_F32 ? __uint_as_float(a.q[e >> 2][e & 3]) : bf16_to_f32((a.q[0][e >> 1] >> (16 * (e & 1))) & 0xffffu);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += u[e];
  }
  store8(!GATED && second ? g.y2 : g.y, (long long)m * g.ldy + n, odt, left, v);
}

// ---- main kernel -------------------------------------------------------------------------------

// A value that is the same in all lanes, in a scalar register: the quotients of scalars are worked out in vector ones.
template <typename T>
__device__ __forceinline__ T uniform(T x) { return (T)__builtin_amdgcn_readfirstlane((int)x); }

// 16 bytes per lane from memory to LDS at dst + 16 * lane (dst uniform over the wave).  Written as instructions: of a
// copy that it knows, the compiler makes every later LDS read wait, since it cannot tell the stages apart.  (m0 is reserved: the
// compiler keeps nothing there and sets it right in front of the instructions that read it, of which these kernels have no others.)
__device__ __forceinline__ void lds_copy(uint32_t dst, uint32_t off, const u32x4& rsrc) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(dst), "v"(off), "s"(rsrc) : "memory");
}
// At most N copies under way, LDS reads done (the built-in, not an instruction: the compiler then knows that it need not
// wait for those reads itself).
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | 0x70 | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wg_barrier() {
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Where a stage keeps a row's 16-byte chunk of the contraction: at chunk ^ swizzle(row).  A 16-byte LDS read is served in
// passes of 16 lanes, lanes 0-3, 12-15, 20-23 and 24-27 of 32 and their complement; lane l of a fragment reads row l % 16,
// chunk l / 16, and the swizzles give the 16 lanes of a pass 16 different slots of the 64 banks.
template <int KB>
__device__ __forceinline__ int swizzle(int row) {
  return KB == 128 ? (row >> 1) & 7 : (-(row >> 2)) & 3;
}

// Where a stage keeps a 32-byte pair of chunks of a row (of R elements, L = 1): at pair ^ pair_swizzle(row).  A transposing
// 8-byte read takes 32 bytes of rows 8 g + 0 .. 3 for g = 0 .. 3; the eight rows of either half of the wave get eight
// different slots (rows of 64 elements: two of them share a line of the banks).
template <int R>
__device__ __forceinline__ int pair_swizzle(int row) {
  return R >= 128 ? (row & 3) | ((row >> 1) & 4) : ((row >> 1) & 1) | ((row >> 2) & 2);
}

// One operand's share of the copies.  L = 0: R rows of KB bytes, contraction contiguous.  L = 1 (bf16): KB / 2 rows (the
// contraction) of R elements.
template <int L, int R, int KB, int THREADS>
struct Stager {
  static constexpr int kLoads = R * KB / 16 / THREADS;
  static_assert(kLoads >= 1 && kLoads * 16 * THREADS == R * KB, "whole copies per thread");
  static constexpr int kRowChunks = L == 0 ? KB / 16 : R / 8;
  static_assert(L == 0 || R >= 64, "four pairs a row at least");
  static_assert(THREADS / kRowChunks % 16 == 0, "the swizzle is the same in all copies of a thread");
  uint32_t off;   // of this thread's first copy; the others follow at `step`
  uint32_t step;  // uniform
  int chunk;      // L = 0: this thread's chunk (the same in all its copies)

  __device__ __forceinline__ void init(int t, long long ld, int cols_left) {
    const int row = t / kRowChunks, pos = t % kRowChunks;
    step = (uint32_t)(THREADS / kRowChunks * ld);
    if (L == 0) {
      chunk = pos ^ swizzle<KB>(row);
      off = (uint32_t)(row * ld + chunk * 16);
    } else {
      const int c = pos ^ (pair_swizzle<R>(row) << 1);
      off = c * 8 < cols_left ? (uint32_t)(row * ld + c * 16) : kOut;
    }
  }
  struct Copy {  // of one stage: kLoads pieces
    u32x4 rsrc;
    uint32_t off;
  };
  // base: first byte of the stage's tile, rem: bytes from there to the operand's end, kleft: bytes of the contraction
  // left in the segment (L = 0: chunks behind them are zeros; L = 1: rows behind them lie behind the end).
  __device__ __forceinline__ Copy begin(const char* base, long long rem, int kleft) const {
    const uint32_t n = rem > 0x7fffffffll ? 0x7fffffffu : (uint32_t)rem;
    return Copy{u32x4{uniform((uint32_t)(uintptr_t)base), uniform((uint32_t)((uintptr_t)base >> 32) & 0xffffu), uniform(n), 0x00020000u},
                L == 1 || chunk * 16 < kleft ? off : kOut};
  }
  __device__ __forceinline__ void piece(Copy& c, uint32_t lds, int i) const {
    lds_copy(lds + i * (THREADS * 16), c.off, c.rsrc);
    // (added here every time: kept in registers, the offsets of all pieces are many.  kOut stays behind every buffer: the
    // steps add up to less than 2^31.)
    if (i + 1 < kLoads) asm volatile("v_add_u32 %0, %1, %0" : "+v"(c.off) : "s"(step));
  }
};

// The left operand's share of the copies where its rows are found through an index: like L = 0, with an offset for each piece.
template <int R, int KB, int THREADS>
struct RowStager {
  static constexpr int kLoads = R * KB / 16 / THREADS, kRowChunks = KB / 16, kStep = THREADS / kRowChunks;
  static_assert(kLoads >= 1 && kLoads * 16 * THREADS == R * KB && kStep % 16 == 0, "whole copies, one swizzle per thread");
  uint32_t off[kLoads];
  int chunk;
  // rows `first` .. of the product, `left` of them this tile's
  __device__ __forceinline__ void init(int t, long long ld, const int32_t* index, int x_rows, int first, int left) {
    const int row = t / kRowChunks;
    chunk = (t % kRowChunks) ^ swizzle<KB>(row);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = row + i * kStep;
      const int k = r < left ? index[first + r] : -1;
      off[i] = k >= 0 && k < x_rows ? (uint32_t)(k * ld + chunk * 16) : kOut;
    }
  }
  struct Copy {
    u32x4 rsrc;
    bool in;
  };
  __device__ __forceinline__ Copy begin(const char* base, long long rem, int kleft) const {
    const uint32_t n = rem > 0x7fffffffll ? 0x7fffffffu : (uint32_t)rem;
    return Copy{u32x4{uniform((uint32_t)(uintptr_t)base), uniform((uint32_t)((uintptr_t)base >> 32) & 0xffffu), uniform(n), 0x00020000u},
                chunk * 16 < kleft};
  }
  __device__ __forceinline__ void piece(Copy& c, uint32_t lds, int i) const { lds_copy(lds + i * (THREADS * 16), c.in ? off[i] : kOut, c.rsrc); }
};

// The matrix instruction's operand for 16 rows starting at r0, bytes 16 g .. of 64-byte part ks of a stage.
template <int L, int R, int KB>
__device__ __forceinline__ u32x4 fragment(uint32_t lds, int r0, int ks, int lane) {
  const int r = lane & 15, g = lane >> 4;
  if (L == 0) {
    const uint32_t a = lds + (uint32_t)((r0 + r) * KB + (((ks * 4 + g) ^ swizzle<KB>(r)) << 4));
    return *(const AX_LDS(u32x4)*)(uintptr_t)a;
  }
  const int kr = r >> 2, sp = pair_swizzle<R>(8 * g + kr);
  const uint32_t a = lds + (uint32_t)((ks * 32 + g * 8 + kr) * (R * 2) + (((r0 >> 4) ^ sp) << 5) + 8 * (lane & 3));
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((AX_LDS(s16x4)*)(uintptr_t)a);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((AX_LDS(s16x4)*)(uintptr_t)(a + 4 * R * 2));
  const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(u32x4, v);
}

template <bool I8>
struct Acc {
  typedef f32x4 T;
  static __device__ __forceinline__ f32x4 mma(const u32x4& a, const u32x4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Acc<true> {
  typedef i32x4 T;
  static __device__ __forceinline__ i32x4 mma(const u32x4& a, const u32x4& b, const i32x4& c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

// I8: int8 codes.  LA, LB: operand layouts.  NB: 2 for the gated pair (the tile's BN columns are BN/2 columns of both
// projections).  WM x WN waves; STAGES stages of KB contraction bytes in LDS.
//
// The wave holds the fragments of 64 bytes of the contraction in registers and reads the next ones while the matrix
// instructions of these run.  Where the next ones are another stage's, a barrier in front of that says that they have arrived
// and that this stage's place is free, and the copies of stage + STAGES are asked for.
//
// P = 3: float32 operands as three bf16 pieces, a = a1 + a2 + a3 and b alike.  A stage holds all pieces of its part of both,
// and each fragment is used in several of the six products of pieces that can pass 2^-24 of a b, the smallest added first:
// half the copies and a third of the LDS reads that six passes over pairs of pieces would take.
// OT: type of the results.
// GR: grouping by experts, whose matrices (right operands, kSums: results) lie one behind the other.
template <bool I8, int P, int LA, int LB, int NB, int BM, int BN, int WM, int WN, int KB, int STAGES, int OCC, int OT, Grouping GR = kWhole>
__global__ __launch_bounds__(64 * WM * WN, OCC) void gemm_kernel(const Args a) {
  constexpr int THREADS = 64 * WM * WN;
  constexpr int BNS = BN / NB;                // columns of one right operand
  constexpr int MF = BM / WM / 16, NF = BN / WN / 16;
  constexpr int KK = KB / 64;                 // matrix instructions' contraction steps per stage
  constexpr int kABytes = BM * KB, kBBytes = BNS * KB;
  constexpr int kBAt = P * kABytes;           // right operands: [weight][piece]
  constexpr int kStage = P * (kABytes + NB * kBBytes);
  constexpr bool kIndexed = GR == kFound;
  typedef typename std::conditional<kIndexed, RowStager<BM, KB, THREADS>, Stager<LA, BM, KB, THREADS>>::type SA;
  typedef Stager<LB, BNS, KB, THREADS> SB;
  constexpr int kLoads = P * (SA::kLoads + NB * SB::kLoads);
  __shared__ __align__(1024) unsigned char smem[STAGES * kStage];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(AX_LDS(unsigned char)*)smem;

  const GemmArgs& g = a.g;
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave % WM, wn = wave / WM;

  // Tiles XCD by XCD: workgroups b, b + 8, ... share an XCD (and its L2) and take a contiguous run of tiles (of all
  // experts' tiles; the weights' gradients: of each expert's); runs go down blocks of eight row tiles before they move to the next column tile.
  constexpr int kElem = I8 ? 1 : 2;
  constexpr int kStepK = KB / kElem;
  int M = g.M, K = g.K, ksteps = a.ksteps, tiles_m = a.tiles_m;
  int row_at = 0;                    // of the results
  long long a_at = 0, b_at = 0;      // bytes from the operands' beginnings
  int tile, split = 0;
  if constexpr (GR == kWhole) {
    tile = xcd_run(blockIdx.x, a.tiles_m * a.tiles_n * a.splits);
    split = uniform(tile / (a.tiles_m * a.tiles_n));
    tile -= split * (a.tiles_m * a.tiles_n);
  } else if constexpr (GR == kRows || GR == kFound) {
    GroupTile e;
    if (!find_tile(a.offsets, a.experts, a.rows, BM, a.tiles_n, blockIdx.x, e)) return;
    tile = uniform(e.tile);
    M = uniform(e.count);
    row_at = uniform(e.first);
    tiles_m = uniform((M + BM - 1) / BM);
    a_at = kIndexed ? 0 : row_at * g.lda;
    b_at = (long long)uniform(e.expert) * (LB == 0 ? g.N : g.K) * g.ldb;
  } else {
    // (the experts with most rows begin first: the launch does not end with them)
    const int per = a.tiles_m * a.tiles_n, i = uniform(blockIdx.x / per);
    Span rows;
    const int e = uniform(by_size(a.offsets, a.experts, a.rows, i, rows));
    tile = xcd_run(blockIdx.x - i * per, per);
    K = uniform(rows.count);
    ksteps = (K + kStepK - 1) / kStepK;
    row_at = e * M;
    a_at = uniform(rows.first) * g.lda;
    b_at = uniform(rows.first) * g.ldb;
  }
  int tm, tn;
  {
    const int band = 8 * a.tiles_n, b = uniform(tile / band), r = tile - b * band;
    const int h = min(8, tiles_m - 8 * b);
    tn = uniform(r / h);
    tm = 8 * b + r - tn * h;
  }
  int second = 0;
  if (NB == 1 && g.dual) {
    const int half = a.tiles_n >> 1;
    second = tn >= half;
    tn -= second * half;
  }
  const int m0 = tm * BM, n0 = tn * BNS;

  const int steps = g.nseg * ksteps, splits = GR == kWhole ? a.splits : 1;
  const int s_beg = uniform((int)((long long)steps * split / splits)), s_end = uniform((int)((long long)steps * (split + 1) / splits));
  const int n_st = s_end - s_beg;

  SA sa;
  SB sb;
  if constexpr (kIndexed) sa.init(t, g.lda, a.index, a.x_rows, row_at + m0, M - m0);
  else sa.init(t, g.lda, M - m0);
  sb.init(t, g.ldb, g.N - n0);

  // the next stage to copy: segment, stage within it, operand positions
  const long long a_step = LA == 0 ? KB : kStepK * g.lda, b_step = LB == 0 ? KB : kStepK * g.ldb;
  // bytes from the tile's first element to the operand's end; rows are whole 16-byte chunks, and a chunk that only began
  // in front of the end would not be loaded at all
  const long long row_bytes = ((long long)K * kElem + 15) & ~15ll;
  const long long a_all = LA == 0 ? (long long)(kIndexed ? a.x_rows - 1 : M - 1 - m0) * g.lda + row_bytes
                                  : (long long)(K - 1) * g.lda + (long long)(((M + 7) & ~7) - m0) * kElem;
  const long long b_all = LB == 0 ? (long long)(g.N - 1 - n0) * g.ldb + row_bytes
                                  : (long long)(K - 1) * g.ldb + (long long)(((g.N + 7) & ~7) - n0) * kElem;
  int seg = GR == kWhole ? uniform(s_beg / ksteps) : 0, ks = s_beg - seg * ksteps;
  const char *pa, *pb, *pb2;
  long long ra, rb;
  auto at_segment = [&]() AX_INLINE {
    const long long ao = LA == 0 ? (kIndexed ? 0 : (long long)m0 * g.lda) : (long long)m0 * kElem;
    const long long bo = LB == 0 ? (long long)n0 * g.ldb : (long long)n0 * kElem;
    pa = (const char*)g.seg[seg].a + a_at + ao + ks * a_step;
    pb = (const char*)(second ? g.seg[seg].b2 : g.seg[seg].b) + b_at + bo + ks * b_step;
    if (NB == 2) pb2 = (const char*)g.seg[seg].b2 + b_at + bo + ks * b_step;
    ra = a_all - ks * a_step;
    rb = b_all - ks * b_step;
  };
  at_segment();
  struct Copies {
    typename SA::Copy a[P];
    typename SB::Copy b[NB][P];
    uint32_t lds;
  };
  auto copies_begin = [&](int buf) AX_INLINE {
    const int kleft = (K - ks * kStepK) * kElem;
    Copies c;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      c.a[p] = sa.begin(pa + p * g.a_plane, ra, kleft);
      c.b[0][p] = sb.begin(pb + p * g.b_plane, rb, kleft);
      if (NB == 2) c.b[NB - 1][p] = sb.begin(pb2 + p * g.b_plane, rb, kleft);
    }
    c.lds = uniform(lds0 + (uint32_t)(buf * kStage + wave * 1024));
    return c;
  };
  auto copies_piece = [&](Copies& c, int i) AX_INLINE {
    if (i < P * SA::kLoads) {
      const int p = i / SA::kLoads;
      sa.piece(c.a[p], c.lds + p * kABytes, i % SA::kLoads);
    } else {
      const int k = (i - P * SA::kLoads) / SB::kLoads;
      sb.piece(c.b[k / P][k % P], c.lds + kBAt + k * kBBytes, (i - P * SA::kLoads) % SB::kLoads);
    }
  };
  auto copies_end = [&]() AX_INLINE {  // the next stage
    if (++ks == ksteps) {
      ks = 0;
      if (++seg < g.nseg) at_segment();
    } else {
      pa += a_step;
      pb += b_step;
      if (NB == 2) pb2 += b_step;
      ra -= a_step;
      rb -= b_step;
    }
  };

  typename Acc<I8>::T acc[MF][NF];
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) acc[i][j] = typename Acc<I8>::T{};

  const int wrow = wm * (BM / WM), wcol = wn * (BNS / WN);
  struct Fragments {
    u32x4 a[P][MF], b[P][NF];
  };
  constexpr int kFrags = P * (MF + NF);
  auto read = [&](Fragments& f, int buf, int kk, int i) AX_INLINE {  // fragment i of kFrags
    const uint32_t la = lds0 + (uint32_t)(buf * kStage), lb = la + kBAt;
    if (i < P * NF) {
      const int p = i / NF, j = i % NF;
      f.b[p][j] = NB == 2 ? fragment<LB, BNS, KB>(lb + ((j & 1) * P + p) * kBBytes, wcol + 16 * (j >> 1), kk, lane)
                          : fragment<LB, BNS, KB>(lb + p * kBBytes, wcol + 16 * j, kk, lane);
    } else {  // (row by row: the first rows' products can start before the last rows' pieces are there)
      const int k = i - P * NF;
      f.a[k % P][k / P] = fragment<LA, BM, KB>(la + (k % P) * kABytes, wrow + 16 * (k / P), kk, lane);
    }
  };
  auto multiply = [&](const Fragments& f, int i) AX_INLINE {  // row i of blocks
    constexpr int kPairs = P == 1 ? 1 : 6;
    constexpr int qa[6] = {P - 1, 0, P / 2, P / 2, 0, 0}, qb[6] = {0, P - 1, P / 2, 0, P / 2, 0};
#pragma unroll
    for (int q = 0; q < kPairs; ++q)
#pragma unroll
      for (int j = 0; j < NF; ++j) acc[i][j] = Acc<I8>::mma(f.b[qb[q]][j], f.a[qa[q]][i], acc[i][j]);
  };

  // Stages asked for: it + STAGES when stage it is multiplied.
#pragma unroll
  for (int s = 0; s < STAGES; ++s)
    if (s < n_st) {
      Copies c = copies_begin(s);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) copies_piece(c, i);
      copies_end();
    }
  int buf = 0;
  Fragments f0, f1;
  if (n_st >= STAGES) wait_copies<(STAGES - 1) * kLoads>();
  else wait_copies<0>();
  wg_barrier();
#pragma unroll
  for (int i = 0; i < kFrags; ++i) read(f0, 0, 0, i);
  // Part kk of stage `it`, whose fragments `now` holds; `next` gets those of the part behind it.  steady: there is a stage
  // it + STAGES to ask for.  Copies and LDS reads are spread evenly among the matrix instructions, row by row.
  auto turn = [&](auto steady, int it, int kk, const Fragments& now, Fragments& next) AX_INLINE {
    const bool last = kk + 1 == KK;
    const int nbuf = !last ? buf : buf + 1 == STAGES ? 0 : buf + 1;
    const bool more = !last || steady || it + 1 < n_st;
    if (last && more) {
      // behind stage it + 1, STAGES - 2 have been asked for (fewer at the end)
      if (steady || it + STAGES <= n_st) wait_copies<(STAGES - 2) * kLoads>();
      else wait_copies<0>();
      wg_barrier();
    }
    if constexpr (steady) {
      Copies c;
      if (last) c = copies_begin(buf);
#pragma unroll
      for (int i = 0; i < MF; ++i) {
#pragma unroll
        for (int k = i * kLoads / MF; k < (i + 1) * kLoads / MF; ++k)
          if (last) copies_piece(c, k);
#pragma unroll
        for (int k = i * kFrags / MF; k < (i + 1) * kFrags / MF; ++k) read(next, nbuf, last ? 0 : kk + 1, k);
        multiply(now, i);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (last) copies_end();
    } else {
      if (last && it + STAGES < n_st) {
        Copies c = copies_begin(buf);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) copies_piece(c, k);
        copies_end();
      }
      if (more) {
#pragma unroll
        for (int k = 0; k < kFrags; ++k) read(next, nbuf, last ? 0 : kk + 1, k);
      }
#pragma unroll
      for (int i = 0; i < MF; ++i) multiply(now, i);
    }
    buf = nbuf;
  };
  // stages in pairs, so that each part finds its fragments in the same registers every time
  auto two = [&](auto steady, int it) AX_INLINE {
    if constexpr (KK == 1) {
      turn(steady, it, 0, f0, f1);
      if (steady || it + 1 < n_st) turn(steady, it + 1, 0, f1, f0);
    } else {
      turn(steady, it, 0, f0, f1);
      turn(steady, it, 1, f1, f0);
    }
  };
  constexpr int PER = KK == 1 ? 2 : 1;
  int it = 0;
  for (; it + STAGES + PER - 1 < n_st; it += PER) two(std::true_type{}, it);
  for (; it < n_st; it += PER) two(std::false_type{}, it);

  // ---- epilogue: a lane holds row m, columns n .. n + 3 of every 16 x 16 block.  Through LDS (a part of it for each wave)
  // so that rows are stored in whole lines: eight columns a lane, the wave's columns of a row side by side.
  constexpr int COLS = NF * 16, OUT = COLS / NB;    // columns in LDS, of the result
  constexpr int PITCH = COLS * 4 + 16;
  constexpr int ROUND = MF >= 2 ? 32 : 16;          // rows a turn
  constexpr int LPR = OUT / 8, RPI = 64 / LPR;      // lanes a row, rows a pass
  static_assert(ROUND * PITCH * WM * WN <= STAGES * kStage && ROUND % RPI == 0, "a part of LDS for each wave");
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  wg_barrier();  // the stages are read
  const uint32_t mine = lds0 + (uint32_t)(wave * ROUND * PITCH);
  const int lm = lane & 15, lq = lane >> 4;
  const int orow = lane / LPR, ocol = lane % LPR * 8;
  const int n = n0 + wcol + ocol;
  Columns cols;
  if (splits == 1 && n < g.N) load_columns<I8, NB == 2, OT>(g, n, cols);
#pragma unroll
  for (int i0 = 0; i0 < MF; i0 += ROUND / 16) {
#pragma unroll
    for (int i = 0; i < ROUND / 16; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        const int c = NB == 2 ? (j & 1) * OUT + 16 * (j >> 1) : 16 * j;
        *(AX_LDS(u32x4)*)(uintptr_t)(mine + (uint32_t)((16 * i + lm) * PITCH + (c + 4 * lq) * 4)) =
            __builtin_bit_cast(u32x4, acc[i0 + i][j]);
      }
    Ahead ahead[ROUND / RPI];
#pragma unroll
    for (int r = 0; r < ROUND / RPI; ++r) {
      const int m = m0 + wrow + 16 * i0 + r * RPI + orow;
      if (splits == 1 && m < M && n < g.N) look_ahead<I8, NB == 2, OT>(g, row_at + m, n, ahead[r]);
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int r = 0; r < ROUND; r += RPI) {
      const int m = m0 + wrow + 16 * i0 + r + orow;
      const uint32_t at = mine + (uint32_t)((r + orow) * PITCH + ocol * 4);
      f32x4 s[2], s2[2];
      s[0] = *(const AX_LDS(f32x4)*)(uintptr_t)at;
      s[1] = *(const AX_LDS(f32x4)*)(uintptr_t)(at + 16);
      if (NB == 2) {
        s2[0] = *(const AX_LDS(f32x4)*)(uintptr_t)(at + OUT * 4);
        s2[1] = *(const AX_LDS(f32x4)*)(uintptr_t)(at + OUT * 4 + 16);
      }
      if (m >= M || n >= g.N) continue;
      if (splits > 1) {  // (rows of ldp, a multiple of eight)
        const long long plane = (long long)M * a.ldp;
        const int planes = NB == 2 || g.dual ? 2 : 1;
        float* p = a.part + ((long long)split * planes + second) * plane + (long long)m * a.ldp + n;
        *(f32x4*)p = s[0];
        *(f32x4*)(p + 4) = s[1];
        if (NB == 2) {
          *(f32x4*)(p + plane) = s2[0];
          *(f32x4*)(p + plane + 4) = s2[1];
        }
      } else {
        finish<I8, NB == 2, OT>(g, cols, ahead[r / RPI], row_at + m, n, s, s2, second);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Tile configurations.  kb: contraction bytes (of a bf16 or int8 operand) per stage, per_cu: workgroups that fit a compute
// unit (LDS).  Times in us, measured on products that fill the card with one kind of tile: of a workgroup (prologue,
// epilogue), and of 128 contraction bytes with one workgroup per compute unit and with per_cu of them.
struct TileShape {
  int bm, bn, kb, per_cu;
  double fixed, step1, step;
};
constexpr int kNumTiles = 4;
constexpr TileShape kTiles[kNumTiles] = {{256, 256, 128, 1, 6.0, 1.50, 1.50},
                                         {128, 128, 128, 2, 3.0, 0.70, 0.95},
                                         {64, 128, 128, 2, 2.5, 0.39, 0.65},
                                         {32, 128, 128, 2, 2.0, 0.30, 0.45}};
// float32 operands (three pieces; six products in the time).  Two of the small ones in a compute unit take the time of a large
// one, which therefore pays only where they read both operands along the contraction: kStep3Along (1531 x 1000 -> 2048: 54.8 us
// a call with the large tile, 60.7 with the small one; 2000 x 2048 -> 2048 101.8 and 121.6).
constexpr int kNumTiles3 = 2;
constexpr TileShape kTiles3[kNumTiles3] = {{128, 128, 64, 1, 5.0, 2.1, 2.1}, {64, 128, 64, 2, 4.0, 1.25, 2.1}};
constexpr double kStep3Along = 2.6;

constexpr int kCus = 256;
constexpr long long kMaxGrid = 1 << 22;  // workgroups: a launch counts its threads in 32 bits

}  // namespace
}  // namespace ax
