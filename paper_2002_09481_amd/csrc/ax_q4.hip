// Products with weights of 4 bits and a scale for every group of a row:
//
//   w[n, k] = scale[n, k / group] c[n, k],  c in -8 .. 7, scale bf16, group 32, 64 or 128
//   y = act(x w^T + bias) + residual        h = act(x wg^T) (x wu^T)
//
// Layout.  A block holds 16 rows and 128 columns of the weights in 1 KB, as the matrix instruction wants them: lane (r, q) of a wave
// has 16 bytes, word s of which holds columns 32 s + 8 q .. + 7 of row r (in the order of q4_shift).  Blocks of a row of
// blocks follow one another, then those of the next 16 rows, then those of the next expert.  Scales in the same order of blocks:
// [4 quads of rows][groups of the block][4 rows], a quad's side by side for the lanes that hold its sums.  What lies behind the last
// row or column has codes and scales of zero.
//
// Few rows of x (q4_kernel).  Bound by reading the weights once, half a byte each.  A wave reads whole blocks, 1 KB at
// a time, and turns words into operands of the matrix instruction in registers: codes are whole numbers that bf16 holds, so
// the products with x (float32: its three bf16 pieces) are exact, and each group's sum in float32 is multiplied by its
// scale in float32.  No weight is rounded.  The waves of a workgroup share the contraction and meet in LDS.  Measured (us at rows / K / N,
// group, a replayed graph over four sets of weights; in brackets the bytes at the rate of a large copy): bf16 1/4096/4096, 128 5.1 (1.7),
// 8/8192/8192, 32 13.3 (7.4), gated 1/4096/14336, 128 16.2 (11.8), gated 68 rows of 32 experts, 28 of them with rows, 2048/1409, 32 32.6 (18), 22 with rows
// 23.8 (14), 64/4096/4096, 128 18.6 (1.9), 256/4096/4096, 128 25.1 (2.5); float32 1/4096/4096, 128 7.9 (1.7), 64/4096/4096 22 (2.1), 256/4096/4096 80 (3.3), gated
// 68 rows of 28 experts 60 (18).  What is left: a workgroup's way from its launch to its first block, and the meeting at its end (the gated pair
// of many experts: two blocks a wave between them); from 64 rows on the conversion of codes, 14 instructions for eight; float32: x cut in
// pieces once for 16 to 64 columns.
//
// More rows: ax_q4_tile.hip, with the weights exact as well.  Very many rows of bf16: the weights are written out once, in the
// workspace, and multiplied by the tiles of ax_gemm_experts.hip, which lose nothing to scales and codes: every weight, scale
// times code, is rounded to bf16 (2^-9 of it at most; codes and scales have eleven significant bits together), an error of 1.1e-3 of a result's
// root mean square, where the rounding of the result alone gives 1.7e-3.  A row's result then depends on how many rows its call has.
#include <algorithm>
#include <type_traits>

#include "ax_float.h"
#include "ax_group.h"
#include "ax_operand.h"
#include "ax_q4.h"
#include "axconv_probe.h"

namespace ax {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kBlockRows = 16, kBlockCols = 128, kBlockBytes = 1024;

// Sizes of the weights of one expert.
struct Shape {
  long long tiles, blocks;  // of 16 rows, of 128 columns
  int groups;               // of columns, to the end of the last block
};
inline Shape shape_of(long long N, long long K, int group) {
  Shape s;
  s.tiles = (N + kBlockRows - 1) / kBlockRows;
  s.blocks = (K + kBlockCols - 1) / kBlockCols;
  s.groups = (int)(s.blocks * (kBlockCols / group));
  return s;
}

// Scale of row r of a tile of rows for group g of block `at` (tile * blocks + block), per groups a block.
__device__ __forceinline__ long long scale_at(long long at, int per, int g, int r) { return (at * per * 4 + (r >> 2) * per + g) * 4 + (r & 3); }

struct Args {
  const void* x;
  Q4Weights w;
  const void* bias;
  const void* res;
  void* y;
  const int32_t* index;
  Groups e;
  long long lda, ldr, ldy;  // elements
  int N, K, x_rows, act;
  int wide;  // workgroups along the columns
};

// Eight float32 values in three pieces of bf16, cut instead of rounded: all products of the pieces with a code are taken, so their sum is
// exact either way, and cutting is a quarter of the instructions.  An infinity is its first piece alone, so that it comes out as the product
// of a float32 infinity does; a NaN is in one of them.  (Float32 calls take 2 to 10 % longer for it, 1/4096/4096 8.5 us instead of 7.7; with
// a branch on all eight values 10 to 40 %.)
__device__ __forceinline__ void cut_in_pieces(const float (&v)[8], u32x4 (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo = v[2 * i], hi = v[2 * i + 1];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      p[k][i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
      if (k < 2) {
        lo -= __uint_as_float(__float_as_uint(lo) & 0xffff0000u);
        hi -= __uint_as_float(__float_as_uint(hi) & 0xffff0000u);
        if (k == 0) {
          lo = __builtin_isinf(v[2 * i]) ? 0.f : lo;
          hi = __builtin_isinf(v[2 * i + 1]) ? 0.f : hi;
        }
      }
    }
  }
}

// Eight elements of x at any alignment, `left` of them there, as operands: themselves, or three pieces.
template <bool F32>
struct XPart {
  u32x4 p[F32 ? 3 : 1];
  template <bool FULL>
  __device__ __forceinline__ void load(const void* x, long long i, int left) {
    if constexpr (F32) {
      float v[8];
      load_elems<true, 8>(x, i, FULL ? 8 : left, v);
      cut_in_pieces(v, p);
    } else {
      const uint16_t* s = (const uint16_t*)x + i;
      if (FULL || left >= 8) {
        p[0] = load_any<u32x4>(s);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          p[0][e] = (2 * e < left ? (uint32_t)s[2 * e] : 0u) | ((2 * e + 1 < left ? (uint32_t)s[2 * e + 1] : 0u) << 16);
      }
    }
  }
};

template <bool F32>
__device__ __forceinline__ f32x4 mma(const u32x4& w, const XPart<F32>& x, f32x4 c) {
#pragma unroll
  for (int i = F32 ? 2 : 0; i >= 0; --i)  // (the smallest piece first)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x.p[i]), c, 0, 0, 0);
  return c;
}

// NB: 2 for the gated pair.  MFR: fragments of 16 rows of x.  CF: tiles of 16 columns of the result.  G: columns of a group.
// WAVES of a workgroup share the contraction, block by block.
template <bool F32, int NB, int MFR, int CF, int G, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void q4_kernel(const Args a) {
  constexpr int COLS = 16 * CF, SCALES = kBlockCols / G;
  __shared__ __align__(16) float part[WAVES][NB][16 * MFR][COLS + 4];
  const int t = threadIdx.x, lane = t & 63, r = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  GroupTile e;
  if (!find_tile(a.e.offsets, a.e.experts, a.e.rows, 16 * MFR, a.wide, blockIdx.x, e)) return;
  // (workgroups of an XCD take neighbouring columns, and all rows of these)
  const int bands = e.tiles / a.wide, k = e.tile;
  const int m0 = __builtin_amdgcn_readfirstlane(k % bands) * 16 * MFR, tile = __builtin_amdgcn_readfirstlane(k / bands) * CF;
  const int M = __builtin_amdgcn_readfirstlane(e.count), row_at = __builtin_amdgcn_readfirstlane(e.first);
  const int expert = __builtin_amdgcn_readfirstlane(e.expert);

  long long x_at[MFR];
  bool there[MFR], all = true;
#pragma unroll
  for (int i = 0; i < MFR; ++i) {
    const int m = row_at + min(m0 + 16 * i + r, M - 1), row = a.index ? a.index[m] : m;
    there[i] = row >= 0 && row < a.x_rows;  // (another index stands for a row of zeros)
    x_at[i] = there[i] ? row * a.lda : 0;
    all = all && __ballot(there[i]) == ~0ull;
  }

  f32x4 acc[NB][MFR][CF];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < MFR; ++i)
#pragma unroll
      for (int j = 0; j < CF; ++j) acc[b][i][j] = f32x4{0, 0, 0, 0};

  auto run = [&](int kb, auto full) __attribute__((always_inline)) {
    u32x4 w[NB][CF];
    typedef uint32_t Scales __attribute__((ext_vector_type(2 * SCALES)));
    Scales sc[NB][CF];
    XPart<F32> x[4][MFR];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int j = 0; j < CF; ++j) {
        const long long row = (long long)expert * a.w.tiles + min(tile + j, a.w.tiles - 1);  // (tiles behind the last: not stored)
        w[b][j] = *(const u32x4*)(a.w.codes[b] + (row * a.w.blocks + kb) * kBlockBytes + lane * 16);
        sc[b][j] = *(const Scales*)(a.w.scales[b] + scale_at(row * a.w.blocks + kb, SCALES, 0, 4 * q));
      }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int c = kb * kBlockCols + 32 * s + 8 * q;
#pragma unroll
      for (int i = 0; i < MFR; ++i) x[s][i].template load<full>(a.x, x_at[i] + c, there[i] ? a.K - c : 0);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int j = 0; j < CF; ++j) {
        f32x4 sum[MFR];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const u32x4 v = widen(w[b][j][s]);
          const bool first = s % (G / 32) == 0, last = (s + 1) % (G / 32) == 0;
          const uint32_t g0 = sc[b][j][s * 32 / G * 2], g1 = sc[b][j][s * 32 / G * 2 + 1];
          f32x4 g;
          if (last) {
            g[0] = bf16_to_f32(g0 & 0xffffu);
            g[1] = __uint_as_float(g0 & 0xffff0000u);
            g[2] = bf16_to_f32(g1 & 0xffffu);
            g[3] = __uint_as_float(g1 & 0xffff0000u);
          }
#pragma unroll
          for (int i = 0; i < MFR; ++i) {
            sum[i] = mma<F32>(v, x[s][i], first ? f32x4{0, 0, 0, 0} : sum[i]);
            if (last) {
#pragma unroll
              for (int h = 0; h < 4; ++h) acc[b][i][j][h] = __builtin_fmaf(sum[i][h], g[h], acc[b][i][j][h]);
            }
          }
        }
      }
  };
  const int whole = all ? a.K / kBlockCols : 0;  // blocks that x has whole
  int kb = wave;
  for (; kb < whole; kb += WAVES) run(kb, std::true_type{});
  for (; kb < a.w.blocks; kb += WAVES) run(kb, std::false_type{});

  // lane: row r of a fragment of x, columns 4 q .. 4 q + 3 of a tile
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < MFR; ++i)
#pragma unroll
      for (int j = 0; j < CF; ++j) *(f32x4*)&part[wave][b][16 * i + r][16 * j + 4 * q] = acc[b][i][j];
  __syncthreads();
  for (int o = t; o < 16 * MFR * COLS; o += 64 * WAVES) {
    const int row = o / COLS, c = o - row * COLS, n = tile * 16 + c;
    if (m0 + row >= M || n >= a.N) continue;
    const long long m = row_at + m0 + row;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s[b] += part[w][b][row][c];
    s[0] *= 16.f;  // (codes came as sixteenths)
    s[1] *= 16.f;
    auto get = [&](const void* p, long long i) { return F32 ? ((const float*)p)[i] : bf16_to_f32(((const uint16_t*)p)[i]); };
    float v[1] = {s[0]};
    if (NB == 1 && a.bias) v[0] += get(a.bias, n);
    apply_act<F32>(v, a.act);
    if (NB == 2) v[0] *= s[1];
    if (NB == 1 && a.res) v[0] += get(a.res, m * a.ldr + n);
    if (F32) ((float*)a.y)[m * a.ldy + n] = v[0];
    else ((uint16_t*)a.y)[m * a.ldy + n] = (uint16_t)f32_to_bf16(v[0]);
  }
}

// ---- the layout --------------------------------------------------------------------------------

struct LayoutArgs {
  const void* w;          // quantize: [experts N, K]
  const int8_t* codes_in;  // pack: [experts N, K]
  const uint16_t* scales_in;  // pack: [experts N, groups given]
  uint8_t* codes;
  uint16_t* scales;
  void* out;              // values, or operands of the products at `pitch`
  long long ld, pitch;
  long long tiles_all;    // of all experts
  int N, K, group, tiles, blocks, given;
};

// A wave a block: lane (r, q) of it has columns 32 s + 8 q .. + 7 of row r.  The largest of a group is that of 4 lanes of the
// row and one, two or four words.  4096 x 4096, group 128: float32 21.5 us (14.8 at the rate of a large copy), bf16 17.8 (8.2), 32 matrices of
// 1408 x 2048 in float32 96 (81).
template <bool F32>
__global__ __launch_bounds__(256) void quantize_kernel(const LayoutArgs a) {
  const long long at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= a.tiles_all * a.blocks) return;
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const long long tile = at / a.blocks;
  const int kb = (int)(at - tile * a.blocks);
  const long long expert = tile / a.tiles;
  const int n = (int)(tile - expert * a.tiles) * kBlockRows + r;
  float v[4][8], top[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int c = kb * kBlockCols + 32 * s + 8 * q;
    load_elems<F32, 8>(a.w, (expert * a.N + n) * a.ld + c, n < a.N ? a.K - c : 0, v[s]);
    top[s] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float m = fabsf(v[s][i]);
      top[s] = m > top[s] || m != m ? m : top[s];  // (a NaN stays)
    }
#pragma unroll
    for (int d = 16; d < 64; d <<= 1) {
      const float m = __shfl_xor(top[s], d);
      top[s] = m > top[s] || m != m ? m : top[s];
    }
  }
  const int per = a.group / 32;
  u32x4 words;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i / per == s / per) m = top[i] > m || top[i] != top[i] ? top[i] : m;
    // rounded to bf16 before the codes are made for it
    const uint32_t half = f32_to_bf16(m / 7.f);
    const float scale = bf16_to_f32(half);
    const bool sound = scale > 0.f && scale < __builtin_inff();
    uint32_t d = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = sound ? fminf(7.f, fmaxf(-8.f, rintf(v[s][i] / scale))) : 0.f;
      d |= (uint32_t)((int)c + 8) << q4_shift(i);
    }
    words[s] = d;
    if (q == 0 && s % per == 0) a.scales[scale_at(at, 4 / per, s / per, r)] = (uint16_t)half;
  }
  *(u32x4*)(a.codes + at * kBlockBytes + lane * 16) = words;
}

// Bound by its loads of single codes: 33 us for 4096 x 4096, where the bytes would take 5.  Once in a weight's life.
__global__ __launch_bounds__(256) void pack_kernel(const LayoutArgs a) {
  const long long at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= a.tiles_all * a.blocks) return;
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const long long tile = at / a.blocks;
  const int kb = (int)(at - tile * a.blocks);
  const long long expert = tile / a.tiles;
  const int n = (int)(tile - expert * a.tiles) * kBlockRows + r;
  const long long row = expert * a.N + n;
  const int per = a.group / 32;
  u32x4 words;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int c = kb * kBlockCols + 32 * s + 8 * q;
    uint32_t d = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      int v = n < a.N && c + i < a.K ? a.codes_in[row * a.K + c + i] : 0;
      v = min(7, max(-8, v));
      d |= (uint32_t)(v + 8) << q4_shift(i);
    }
    words[s] = d;
    if (q == 0 && s % per == 0) {
      const int g = kb * (4 / per) + s / per;
      a.scales[scale_at(at, 4 / per, s / per, r)] = n < a.N && g < a.given ? a.scales_in[row * a.given + g] : 0;
    }
  }
  *(u32x4*)(a.codes + at * kBlockBytes + lane * 16) = words;
}

// The weights, float32 [rows, K] (VALUES), or bf16 as the tiles read them.  Bound by memory: 4096 x 4096 in float32 18 us (14.8 at the rate of a
// large copy), in bf16 11 (8.2).
template <bool VALUES>
__global__ __launch_bounds__(256) void unpack_kernel(const LayoutArgs a) {
  const long long at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= a.tiles_all * a.blocks) return;
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const long long tile = at / a.blocks;
  const int kb = (int)(at - tile * a.blocks);
  const long long expert = tile / a.tiles;
  const int n = (int)(tile - expert * a.tiles) * kBlockRows + r;
  if (n >= a.N) return;
  const long long row = expert * a.N + n;
  const u32x4 words = *(const u32x4*)(a.codes + at * kBlockBytes + lane * 16);
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int c = kb * kBlockCols + 32 * s + 8 * q;
    if (c >= a.K) continue;
    const float scale = bf16_to_f32(a.scales[scale_at(at, kBlockCols / a.group, c % kBlockCols / a.group, r)]);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)((int)(words[s] >> q4_shift(i) & 15u) - 8) * scale;
    if constexpr (VALUES) {
      store_elems<true, 8>(a.out, row * a.K + c, a.K - c, v);
    } else {  // (rounded for the matrix instruction; whole chunks: the codes behind the last column are zero)
      *(u32x4*)((uint16_t*)a.out + row * a.pitch + c) =
          u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    }
  }
}

LayoutArgs layout_args(long long experts, long long N, long long K, int group) {
  LayoutArgs a{};
  const Shape s = shape_of(N, K, group);
  a.tiles_all = experts * s.tiles;
  a.N = (int)N;
  a.K = (int)K;
  a.group = group;
  a.tiles = (int)s.tiles;
  a.blocks = (int)s.blocks;
  a.given = (int)((K + group - 1) / group);
  return a;
}
int grid_of(const LayoutArgs& a) { return (int)((a.tiles_all * a.blocks + 3) / 4); }

// ---- checks and plans --------------------------------------------------------------------------

int check_weights(int64_t experts, int64_t N, int64_t K, int group) {
  if (group != 32 && group != 64 && group != 128) return AX_ERR_OPTION;
  if (experts < 1 || experts > kMaxExperts || N < 1 || K < 1 || N > kMaxDim || K > kMaxDim || experts * N >= 1ll << 31) return AX_ERR_SHAPE;
  const Shape s = shape_of(N, K, group);
  return experts * s.tiles * s.blocks < 1ll << 24 ? AX_OK : AX_ERR_SHAPE;  // (a wave a block: a launch counts its threads in 32 bits)
}

int check_q4(const ax_q4_desc_t* d, bool gated, bool residual) {
  if (!d) return AX_ERR_NULL;
  if (!dtype_ok(d->dtype) || d->act < AX_ACT_NONE || d->act > AX_ACT_GELU || (d->indexed & ~1) || (d->unaligned & ~1)) return AX_ERR_OPTION;
  if (int rc = check_weights(d->experts, d->N, d->K, d->group)) return rc;
  const int e = elem_bytes(d->dtype);
  if (d->rows < 0 || d->x_rows < 0 || d->rows > kMaxDim || d->x_rows > kMaxDim || (!d->indexed && d->x_rows != d->rows) ||
      !pitch_ok(d->x_ld, d->K, e) || !pitch_ok(d->y_ld, d->N, e) || (residual && !pitch_ok(d->residual_ld, d->N, e)))
    return AX_ERR_SHAPE;
  return AX_OK;
}

enum Way { kFew, kTiles, kWritten };
struct Plan {
  Way way;
  bool found;   // more rows: through the index, in place
  PackJob job;  // or copied
  Operand w[2];  // kWritten
  int tile;
  GemmArgs g;
  Groups e;
  size_t bytes;
};

// us at rows / K / N, q4_kernel : q4_tile_kernel : written out.  A few units of 64 rows by 16 columns, or few rows of an expert: the first, which
// needs none of the others' stages.
//   256/4096/4096 26 : 43 : 39      350/4096/4096 41 : 43 : 42   gated 256/4096/4096 42 : 43     500/2048/11264 58 : 42 : 47
//   8 experts, 2048/1408: 512 rows 17 : 23, 4096 rows 68 : 47 : 49   600/1024/3000 17 : 14 : 20  float32 256/4096/4096 80 : 79, 300/4096/4096 100 : 79
// Many rows of an expert: the weights pay for being written once.
//   512/4096/4096 41 : 42 : 42      600/4096/4096 62 : 58 : 51   1027/4096/4096 86 : 75 : 56     2048/4096/4096 151 : 85 : 75
//   16 experts, 2048/1408: 4096 rows 64 : 45 : 56
// float32 is never written out, in pieces: 2048/4096/4096 228, the six products of pieces alone would be 340.
Way way_of(const ax_q4_desc_t* d, bool gated) {
  const long long used = std::max<long long>(1, std::min<long long>(d->experts, d->rows)), tiles = (d->N + 15) / 16;
  const long long units = used * ((d->rows + 64 * used - 1) / (64 * used)) * tiles * (gated ? 2 : 1);
  if ((d->rows <= 32 * used || units <= 1024) && (d->rows / 16 + used) * tiles < 1 << 21) return kFew;  // (a launch counts its threads in 32 bits)
  if (d->dtype == AX_BF16 && d->rows > 600 * used) return kWritten;
  return kTiles;
}

Plan make_plan(const ax_q4_desc_t* d, bool gated, const void* x, const int32_t* offsets, void* ws) {
  Plan p{};
  Arena ar(ws);
  p.way = way_of(d, gated);
  p.e = Groups{offsets, d->experts, (int)d->rows, nullptr, 0};
  if (p.way == kFew) return p;
  p.found = d->indexed && d->x_rows > 0 && d->dtype == AX_BF16 && !d->unaligned && d->K % 8 == 0 && d->x_ld % 8 == 0 &&
            d->x_rows * d->x_ld * 2 < 1ll << 31;
  const Operand a = make_operand(x, p.found ? d->x_rows : d->rows, d->K, d->x_ld, d->dtype, d->unaligned || (d->indexed && !p.found), ar, &p.job);
  GemmArgs& g = p.g;
  if (p.way == kWritten) {
    PackJob unused;
    for (int b = 0; b < (gated ? 2 : 1); ++b) p.w[b] = make_operand(nullptr, d->experts * d->N, d->K, d->K, AX_BF16, true, ar, &unused);
  }
  add_segment(&g, a, p.w[0], gated ? &p.w[1] : nullptr);
  g.M = (int)d->rows;
  g.N = (int)d->N;
  g.K = (int)a.cols;
  g.gated = gated;
  g.odt = d->dtype;
  g.act = d->act;
  g.ldy = d->y_ld;
  g.ldr = d->residual_ld;
  if (p.way == kWritten) p.tile = plan_experts(g, p.e, false);
  p.bytes = ar.used;
  return p;
}

// A workgroup's columns, 16, 32 or 64 of them: as many as leave work for two thirds of the compute units, since each reads all
// rows of x (us with 16 / 32 / 64: 64/2048/11264 26 / 23 / 18, 64/4096/4096 18 / 19 / 24, 256/4096/4096 61 / 36 / 25).  float32 pays for the
// pieces of x in each workgroup as well: 68 rows of 16 experts, 1024/4096 30 / 21 / 17, gated 32 experts, 2048/1409 55 / 53 / 50, 8 experts,
// 2048/4096 30 / 25 / 27.  Its waves: 16 where a wave of eight would have four blocks or more and no compute unit gets a second workgroup,
// else eight.  (us with 8 : 16, one row, K / N: 2048/4096 3.8 : 4.1, 4096/2048 4.5 : 4.6, 4096/4096 5.2 : 5.1, 5120/4096 5.8 : 5.4, 8192/4096
// 7.3 : 6.7, 16384/2048 10.7 : 9.6, float32 8192/1024 12.2 : 11.5; 320 workgroups, which sixteen waves each would take in two turns: 2048/5120
// 4.6 : 5.7, 4096/5120 6.5 : 7.6, 16384/5120 15.6 : 16.6; 20 rows, 4096/2048 8.5 : 8.7, 16384/4096 25.6 : 26.0, 4096/5120 14.6 : 15.5.)
constexpr long long kLeast = 170, kUnits = 256;  // two thirds of the compute units, all
struct FewShape {
  int bands, cols, waves;  // rows and columns by 16
};
FewShape few_shape(bool f32, bool gated, const Groups& e, const Q4Weights& w) {
  const long long used = std::max(1, e.offsets ? std::min(e.experts, e.rows) : 1), rows = e.rows;
  const int bands = rows <= 16 * used ? 1 : f32 || rows <= 32 * used ? 2 : 4;  // (three pieces of 64 rows leave no registers)
  // tiles of 16 columns by bands of rows that there can be expected
  const long long work = w.tiles * used * ((rows + 16 * bands * used - 1) / (16 * bands * used));
  const bool deep = w.blocks >= 32;
  if (bands == 1) {
    if (f32 && !gated && work >= 2048) return {1, 4, 8};
    if ((deep || f32) && work >= 512) return {1, 2, 8};
    return {1, 1, deep && work <= kUnits ? 16 : 8};
  }
  if (bands == 2) {
    if (work >= 2 * kLeast) return {2, 2, 8};
    return {2, 1, deep && !f32 && work <= kUnits ? 16 : 8};
  }
  if (!gated && work >= 4 * kLeast) return {4, 4, 4};
  return {4, work >= 2 * kLeast ? 2 : 1, 8};
}
template <bool F32, int NB, int G>
void launch_rows(Args& a, hipStream_t s) {
  const FewShape f = few_shape(F32, NB == 2, a.e, a.w);
  auto go = [&](auto mfr, auto cf, auto waves) {
    constexpr int MFR = decltype(mfr)::value, CF = decltype(cf)::value, WAVES = decltype(waves)::value;
    const long long used = std::max(1, a.e.offsets ? std::min(a.e.experts, a.e.rows) : 1), rows = a.e.rows;
    a.wide = (a.w.tiles + CF - 1) / CF;
    const long long bands = a.e.offsets ? rows / (16 * MFR) + used : (rows + 16 * MFR - 1) / (16 * MFR);
    q4_kernel<F32, NB, MFR, CF, G, WAVES><<<(int)(bands * a.wide), 64 * WAVES, 0, s>>>(a);
  };
  constexpr auto one = std::integral_constant<int, 1>{};
  constexpr auto two = std::integral_constant<int, 2>{};
  constexpr auto four = std::integral_constant<int, 4>{};
  constexpr auto eight = std::integral_constant<int, 8>{};
  constexpr auto sixteen = std::integral_constant<int, 16>{};
  if (f.bands == 1) {
    if constexpr (F32 && NB == 1) {
      if (f.cols == 4) return go(one, four, eight);
    }
    if (f.cols == 2) go(one, two, eight);
    else if (f.waves == 16) go(one, one, sixteen);
    else go(one, one, eight);
  } else if (f.bands == 2) {
    if constexpr (!F32) {
      if (f.waves == 16) return go(two, one, sixteen);
    }
    if (f.cols == 2) go(two, two, eight);
    else go(two, one, eight);
  } else if constexpr (!F32) {
    if constexpr (NB == 1) {
      if (f.cols == 4) return go(four, four, four);
    }
    if (f.cols == 2) go(four, two, eight);
    else go(four, one, eight);
  }
}
template <bool F32, int NB>
hipError_t launch_group(Args& a, int group, hipStream_t s) {
  if (group == 32) launch_rows<F32, NB, 32>(a, s);
  else if (group == 64) launch_rows<F32, NB, 64>(a, s);
  else launch_rows<F32, NB, 128>(a, s);
  return hipGetLastError();
}

Q4Weights weights_of(const ax_q4_desc_t* d, const uint8_t* const (&codes)[2], const void* const (&scales)[2]) {
  const Shape sh = shape_of(d->N, d->K, d->group);
  Q4Weights w{};
  for (int b = 0; b < 2; ++b) {
    w.codes[b] = codes[b];
    w.scales[b] = (const uint16_t*)scales[b];
  }
  w.tiles = (int)sh.tiles;
  w.blocks = (int)sh.blocks;
  w.group = d->group;
  return w;
}

int run(const ax_q4_desc_t* d, bool gated, const void* x, const int32_t* index, const int32_t* offsets, const uint8_t* const (&codes)[2],
        const void* const (&scales)[2], const void* bias, const void* residual, void* y, void* ws, size_t ws_bytes, hipStream_t s) {
  Plan p = make_plan(d, gated, x, offsets, ws);
  if ((p.way == kTiles && !q4_tiles_fit(p.g, p.e)) || (p.way == kWritten && !experts_fit(p.g, p.e, false, p.tile))) return AX_ERR_SHAPE;
  if (!ws_ok(ws, ws_bytes, p.bytes)) return AX_ERR_WORKSPACE;
  const bool f32 = d->dtype == AX_F32;
  const Q4Weights w = weights_of(d, codes, scales);
  if (p.way == kFew) {
    Args a{};
    a.x = x;
    a.w = w;
    a.bias = bias;
    a.res = residual;
    a.y = y;
    a.index = index;
    a.e = p.e;
    a.lda = d->x_ld;
    a.ldr = d->residual_ld;
    a.ldy = d->y_ld;
    a.N = (int)d->N;
    a.K = (int)d->K;
    a.x_rows = (int)d->x_rows;
    a.act = d->act;
    const hipError_t rc = f32 ? (gated ? launch_group<true, 2>(a, d->group, s) : launch_group<true, 1>(a, d->group, s))
                              : (gated ? launch_group<false, 2>(a, d->group, s) : launch_group<false, 1>(a, d->group, s));
    return rc == hipSuccess ? AX_OK : AX_ERR_HIP;
  }
  if (p.found) {
    p.e.index = index;
    p.e.x_rows = (int)d->x_rows;
  } else {
    p.job.index = index;
    p.job.src_rows = (int)d->x_rows;
  }
  const bool wanted[1] = {true};
  PackBatch copies{};
  const int blocks = fill_pack(&copies, &p.job, wanted, 1);
  if (run_pack(copies, blocks, s) != hipSuccess) return AX_ERR_HIP;
  p.g.y = y;
  p.g.bias = bias;
  p.g.res = residual;
  if (p.way == kTiles) return launch_q4_tiles(p.g, p.e, w, s) == hipSuccess ? AX_OK : AX_ERR_HIP;
  for (int b = 0; b < (gated ? 2 : 1); ++b) {
    LayoutArgs l = layout_args(d->experts, d->N, d->K, d->group);
    l.codes = (uint8_t*)codes[b];
    l.scales = (uint16_t*)scales[b];
    l.out = (void*)p.w[b].p;
    l.pitch = p.w[b].ld / 2;
    unpack_kernel<false><<<grid_of(l), 256, 0, s>>>(l);
    if (hipGetLastError() != hipSuccess) return AX_ERR_HIP;
  }
  return launch_gemm_experts(p.g, p.e, false, p.tile, s) == hipSuccess ? AX_OK : AX_ERR_HIP;
}

// What all products check of their pointers.
int check_rows(const ax_q4_desc_t* d, const void* x, const int32_t* index, const int32_t* offsets) {
  if ((d->indexed != 0) != (index != nullptr) || (!x && d->x_rows > 0) || (!offsets && d->experts > 1)) return AX_ERR_NULL;
  if (!aligned_to(offsets, 4) || !aligned_to(index, 4)) return AX_ERR_ALIGN;
  return operand_aligned(x, elem_bytes(d->dtype), d->unaligned, d->K, d->x_ld, d->dtype) ? AX_OK : AX_ERR_ALIGN;
}

}  // namespace
}  // namespace ax

using namespace ax;

extern "C" size_t ax_q4_codes_bytes(int64_t experts, int64_t N, int64_t K) {
  if (check_weights(experts, N, K, 128) != AX_OK) return 0;
  const Shape s = shape_of(N, K, 128);
  return (size_t)(experts * s.tiles * s.blocks) * kBlockBytes;
}
extern "C" size_t ax_q4_scales_bytes(int64_t experts, int64_t N, int64_t K, int32_t group) {
  if (check_weights(experts, N, K, group) != AX_OK) return 0;
  const Shape s = shape_of(N, K, group);
  return (size_t)(experts * s.tiles * s.groups) * kBlockRows * 2;
}

extern "C" int ax_quantize_q4(const void* w, int32_t dtype, int64_t w_ld, int64_t experts, int64_t N, int64_t K, int32_t group,
                              uint8_t* codes_out, void* scales_out, void* hip_stream) {
  if (!dtype_ok(dtype)) return AX_ERR_OPTION;
  if (int rc = check_weights(experts, N, K, group)) return rc;
  if (!pitch_ok(w_ld, K, elem_bytes(dtype))) return AX_ERR_SHAPE;
  if (!w || !codes_out || !scales_out) return AX_ERR_NULL;
  if (!aligned_to(w, elem_bytes(dtype)) || !aligned_to(codes_out, 16) || !aligned_to(scales_out, 16)) return AX_ERR_ALIGN;
  LayoutArgs a = layout_args(experts, N, K, group);
  a.w = w;
  a.ld = w_ld;
  a.codes = codes_out;
  a.scales = (uint16_t*)scales_out;
  const hipStream_t s = (hipStream_t)hip_stream;
  if (dtype == AX_F32) quantize_kernel<true><<<grid_of(a), 256, 0, s>>>(a);
  else quantize_kernel<false><<<grid_of(a), 256, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? AX_OK : AX_ERR_HIP;
}

extern "C" int ax_pack_q4(const int8_t* codes, const void* scales, int64_t experts, int64_t N, int64_t K, int32_t group,
                          uint8_t* codes_out, void* scales_out, void* hip_stream) {
  if (int rc = check_weights(experts, N, K, group)) return rc;
  if (!codes || !scales || !codes_out || !scales_out) return AX_ERR_NULL;
  if (!aligned_to(scales, 2) || !aligned_to(codes_out, 16) || !aligned_to(scales_out, 16)) return AX_ERR_ALIGN;
  LayoutArgs a = layout_args(experts, N, K, group);
  a.codes_in = codes;
  a.scales_in = (const uint16_t*)scales;
  a.codes = codes_out;
  a.scales = (uint16_t*)scales_out;
  pack_kernel<<<grid_of(a), 256, 0, (hipStream_t)hip_stream>>>(a);
  return hipGetLastError() == hipSuccess ? AX_OK : AX_ERR_HIP;
}

extern "C" int ax_q4_values(const uint8_t* codes, const void* scales, int64_t experts, int64_t N, int64_t K, int32_t group, float* values_out,
                            void* hip_stream) {
  if (int rc = check_weights(experts, N, K, group)) return rc;
  if (!codes || !scales || !values_out) return AX_ERR_NULL;
  if (!aligned_to(codes, 16) || !aligned_to(scales, 16) || !aligned_to(values_out, 4)) return AX_ERR_ALIGN;
  LayoutArgs a = layout_args(experts, N, K, group);
  a.codes = (uint8_t*)codes;
  a.scales = (uint16_t*)scales;
  a.out = values_out;
  unpack_kernel<true><<<grid_of(a), 256, 0, (hipStream_t)hip_stream>>>(a);
  return hipGetLastError() == hipSuccess ? AX_OK : AX_ERR_HIP;
}

extern "C" size_t ax_matmul_q4_workspace_bytes(const ax_q4_desc_t* d) {
  if (check_q4(d, false, false) != AX_OK || d->rows == 0) return 0;
  return make_plan(d, false, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_matmul_q4(const ax_q4_desc_t* d, const void* x, const int32_t* index, const int32_t* offsets, const uint8_t* codes,
                            const void* scales, const void* bias, const void* residual, void* y_out, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_q4(d, false, residual != nullptr)) return rc;
  if (d->rows == 0) return AX_OK;
  if (int rc = check_rows(d, x, index, offsets)) return rc;
  if (!codes || !scales || !y_out) return AX_ERR_NULL;
  if (!aligned_to(codes, 16) || !aligned_to(scales, 16)) return AX_ERR_ALIGN;
  for (const void* p : {bias, residual, (const void*)y_out})
    if (!aligned_to(p, elem_bytes(d->dtype))) return AX_ERR_ALIGN;
  return run(d, false, x, index, offsets, {codes, nullptr}, {scales, nullptr}, bias, residual, y_out, workspace, workspace_bytes,
             (hipStream_t)hip_stream);
}

extern "C" size_t ax_gated_q4_workspace_bytes(const ax_q4_desc_t* d) {
  if (check_q4(d, true, false) != AX_OK || d->rows == 0) return 0;
  return make_plan(d, true, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_gated_q4(const ax_q4_desc_t* d, const void* x, const int32_t* index, const int32_t* offsets, const uint8_t* g_codes,
                           const void* g_scales, const uint8_t* u_codes, const void* u_scales, void* h_out, void* workspace,
                           size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_q4(d, true, false)) return rc;
  if (d->rows == 0) return AX_OK;
  if (int rc = check_rows(d, x, index, offsets)) return rc;
  if (!g_codes || !g_scales || !u_codes || !u_scales || !h_out) return AX_ERR_NULL;
  for (const void* p : {(const void*)g_codes, g_scales, (const void*)u_codes, u_scales})
    if (!aligned_to(p, 16)) return AX_ERR_ALIGN;
  if (!aligned_to(h_out, elem_bytes(d->dtype))) return AX_ERR_ALIGN;
  return run(d, true, x, index, offsets, {g_codes, u_codes}, {g_scales, u_scales}, nullptr, nullptr, h_out, workspace, workspace_bytes,
             (hipStream_t)hip_stream);
}

extern "C" int ax_probe_q4_plan(const ax_q4_desc_t* d, int gated, int* kernel, int* rows, int* cols, int* waves) {
  if (gated & ~1) return AX_ERR_OPTION;
  if (int rc = check_q4(d, gated != 0, false)) return rc;
  int k = 0, r = 0, c = 0, n = 0, unused;
  if (d->rows > 0) {
    static const int32_t grouped = 0;  // (asked only whether there are any)
    const Plan p = make_plan(d, gated != 0, nullptr, d->experts > 1 ? &grouped : nullptr, nullptr);
    k = p.way;
    if (k == kFew) {
      const FewShape f = few_shape(d->dtype == AX_F32, gated != 0, p.e, weights_of(d, {nullptr, nullptr}, {nullptr, nullptr}));
      r = 16 * f.bands;
      c = 16 * f.cols;
      n = f.waves;
    } else if (k == kTiles) {
      r = q4_tile_rows(p.g, p.e);
      c = gated ? 128 : 256;
    } else {
      tile_of_experts(p.g, false, p.tile, &r, &c, &unused);
    }
  }
  if (kernel) *kernel = k;
  if (rows) *rows = r;
  if (cols) *cols = c;
  if (waves) *waves = n;
  return AX_OK;
}
