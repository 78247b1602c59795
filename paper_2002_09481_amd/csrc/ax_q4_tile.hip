// Products of many rows with weights of 4 bits (layout: ax_q4.hip), the weights exact as for few rows: codes are operands of the matrix
// instruction, a group's sum in float32 is multiplied by its scale in float32.
//
// A workgroup of four waves computes 64 or 32 rows by 256 columns (gated: 128 of each weight), a wave 64 columns of all rows.  x passes through
// LDS as in ax_gemm.hip, for all waves; codes and scales pass through LDS as well, each wave's own, since that way all copies
// are asynchronous and counted together.  The words of codes lie as the instruction wants them and are widened once for the rows
// of the workgroup.  Scales are applied every 64 columns of the contraction (32 where the group is 32): one more level of sums in registers
// would leave none for the operands.  bf16: codes are widened with 24 added (a third of the instructions), and the product of x with -24
// stands in front of every sum; sums round as those of terms up to six times as large.  float32: x in its three pieces, codes as they are.
//
// Bound: vector instructions (widening, scales) and matrix instructions, 63 and 49 % of the cycles at 8192/4096/4096, next to each
// other only in part.  Measured (us at rows / K / N, group): bf16 300/4096/4096, 64 43, 512/4096/4096 44, 600/4096/4096 59, 1027/4096/4096, 64 75,
// 2048/4096/4096, 128 85, 2048 rows of 32 experts, 2048/1408, 64 33, 4096 of them 47; float32 512/4096/4096, 128 81, 2048/4096/4096 244.  Dropped: parts read a turn ahead in registers (they spill, or gain
// nothing), three to six stages (0 to 50 % slower: fewer workgroups a compute unit), 128 rows a workgroup (one wave a SIMD, twice the time).
#include <algorithm>
#include <cmath>

#include "ax_gemm_tile.h"
#include "ax_q4.h"

namespace ax {
namespace {

struct TileArgs {
  GemmArgs g;
  Groups e;
  Q4Weights w;
  int wide;  // workgroups along the columns
};

template <int P, int NB, int MF, int G, bool FOUND>
__global__ __launch_bounds__(256, P == 3 ? 1 : 2) void q4_tile_kernel(const TileArgs a) {
  constexpr int BM = 16 * MF, THREADS = 256, OT = P == 3 ? AX_F32 : AX_BF16;
  constexpr int SC = 128 / G, PER = 4 / NB;              // groups of a block; tiles of 16 columns a wave has of each weight
  constexpr int U = G == 32 ? 1 : 2;                     // words of codes under one scale at a time
  constexpr int kHalf = BM * 128;                        // 64 columns of the contraction, one plane
  constexpr int kCodesAt = P * 2 * kHalf, kScalesAt = kCodesAt + 4 * 4096, kStage = kScalesAt + 4 * 512;
  typedef typename std::conditional<FOUND, RowStager<BM, 128, THREADS>, Stager<0, BM, 128, THREADS>>::type SA;
  constexpr int kLoads = P * 2 * SA::kLoads + 4 + NB;    // copies of a thread for a stage
  __shared__ __align__(1024) unsigned char smem[2 * kStage];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(AX_LDS(unsigned char)*)smem;

  const GemmArgs& g = a.g;
  const int t = threadIdx.x, lane = t & 63, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  GroupTile e;
  if (!find_tile(a.e.offsets, a.e.experts, a.e.rows, BM, a.wide, blockIdx.x, e)) return;
  // (neighbouring workgroups of an XCD: all rows of the same columns)
  const int bands = e.tiles / a.wide, k = e.tile;
  const int m0 = uniform(k % bands) * BM, n0 = uniform(k / bands) * (64 * PER);
  const int M = uniform(e.count), row_at = uniform(e.first);
  const long long tile_at = (long long)uniform(e.expert) * a.w.tiles;

  SA sa;
  if constexpr (FOUND) sa.init(t, g.lda, a.e.index, a.e.x_rows, row_at + m0, M - m0);
  else sa.init(t, g.lda, M - m0);
  const long long row_bytes = ((long long)g.K * 2 + 15) & ~15ll;
  const char* pa = (const char*)g.seg[0].a + (FOUND ? 0 : (long long)(row_at + m0) * g.lda);
  long long ra = (long long)(FOUND ? a.e.x_rows - 1 : M - 1 - m0) * g.lda + row_bytes;

  // codes and scales of this wave's tiles (those behind the last: the last's again, not stored)
  const int tile = n0 / 16 + wave * PER;
  const int first = min(tile, a.w.tiles - 1);
  uint32_t code_off[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) code_off[j] = (uint32_t)((min(tile + j, a.w.tiles - 1) - first) * a.w.blocks * 1024 + lane * 16);
  const int sj = lane / (2 * SC);
  const uint32_t scale_off = sj < PER ? (uint32_t)((min(tile + sj, a.w.tiles - 1) - first) * a.w.blocks * (SC * 32) + lane % (2 * SC) * 16) : kOut;
  const uint32_t code_end = uniform((uint32_t)min(a.w.tiles - first, PER) * (uint32_t)a.w.blocks * 1024u);
  const uint32_t scale_end = uniform((uint32_t)min(a.w.tiles - first, PER) * (uint32_t)a.w.blocks * (SC * 32u));

  auto copies = [&](int kb, int buf) AX_INLINE {
    const uint32_t at = uniform(lds0 + (uint32_t)(buf * kStage));
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // (a half behind the last column: nothing of it is there)
        typename SA::Copy c = sa.begin(pa + p * g.a_plane + h * 128, max(ra - h * 128, 0ll), (g.K - kb * 128 - h * 64) * 2);
#pragma unroll
        for (int i = 0; i < SA::kLoads; ++i) sa.piece(c, uniform(at + (uint32_t)((p * 2 + h) * kHalf + wave * 1024)), i);
      }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const long long block = (tile_at + first) * a.w.blocks + kb;
      const char* codes = (const char*)a.w.codes[b] + block * 1024;
      const char* scales = (const char*)a.w.scales[b] + block * (SC * 32);
      const u32x4 rc{uniform((uint32_t)(uintptr_t)codes), uniform((uint32_t)((uintptr_t)codes >> 32) & 0xffffu), uniform(code_end - (uint32_t)kb * 1024u), 0x00020000u};
      const u32x4 rs{uniform((uint32_t)(uintptr_t)scales), uniform((uint32_t)((uintptr_t)scales >> 32) & 0xffffu), uniform(scale_end - (uint32_t)kb * (SC * 32u)), 0x00020000u};
#pragma unroll
      for (int j = 0; j < PER; ++j) lds_copy(uniform(at + (uint32_t)(kCodesAt + wave * 4096 + (b * PER + j) * 1024)), code_off[j], rc);
      if (lane < 2 * SC * PER) lds_copy(uniform(at + (uint32_t)(kScalesAt + wave * 512 + b * PER * SC * 32)), scale_off, rs);
    }
    pa += 256;
    ra -= 256;
  };

  f32x4 acc[MF][4];  // [rows][weight, tile]
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

  // Words of codes under one scale (of a group of 128, half of them), their scales, and what they meet.
  typedef uint32_t Words __attribute__((ext_vector_type(U)));
  struct Part {
    Words word[4];
    u32x2 scale[4];
    u32x4 x[MF][U][P];
  };
  auto read = [&](Part& part, int buf, int u) AX_INLINE {
    const uint32_t at = uniform(lds0 + (uint32_t)(buf * kStage));
#pragma unroll
    for (int j = 0; j < 4; ++j) part.word[j] = *(const AX_LDS(Words)*)(uintptr_t)(at + (uint32_t)(kCodesAt + wave * 4096 + j * 1024 + lane * 16 + u * 4));
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int s = 0; s < U; ++s)
#pragma unroll
        for (int p = 0; p < P; ++p) part.x[i][s][p] = fragment<0, BM, 128>(at + (uint32_t)((p * 2 + (u >> 1)) * kHalf), 16 * i, U == 2 ? s : u & 1, lane);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      part.scale[j] = *(const AX_LDS(u32x2)*)(uintptr_t)(at + (uint32_t)(kScalesAt + wave * 512 + j * SC * 32 + (q * SC + u * 32 / G) * 8));
  };
  auto multiply = [&](const Part& part) AX_INLINE {
    f32x4 less[MF];
#pragma unroll
    for (int i = 0; i < MF; ++i) less[i] = f32x4{0, 0, 0, 0};
    if constexpr (P == 1) {
#pragma unroll
      for (int s = 0; s < U; ++s)
#pragma unroll
        for (int i = 0; i < MF; ++i) less[i] = Acc<false>::mma(u32x4{kQ4Less, kQ4Less, kQ4Less, kQ4Less}, part.x[i][s][0], less[i]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u32x4 w[U];
#pragma unroll
      for (int s = 0; s < U; ++s) {
        const uint32_t d = part.word[j][s];
        w[s] = P == 3 ? widen(d) : widen_more(d);
      }
      f32x4 sum[MF];
#pragma unroll
      for (int s = 0; s < U; ++s)
#pragma unroll
        for (int p = P - 1; p >= 0; --p)  // (the smallest piece first)
#pragma unroll
          for (int i = 0; i < MF; ++i) sum[i] = Acc<false>::mma(w[s], part.x[i][s][p], s == 0 && p == P - 1 ? less[i] : sum[i]);
      const f32x4 sc{bf16_to_f32(part.scale[j][0] & 0xffffu), __uint_as_float(part.scale[j][0] & 0xffff0000u),
                     bf16_to_f32(part.scale[j][1] & 0xffffu), __uint_as_float(part.scale[j][1] & 0xffff0000u)};
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[i][j][c] = __builtin_fmaf(sum[i][c], sc[c], acc[i][j][c]);
    }
  };

#pragma unroll
  for (int b = 0; b < 2; ++b)
    if (b < a.w.blocks) copies(b, b);
  int buf = 0;
  for (int kb = 0; kb < a.w.blocks; ++kb) {
    if (kb + 2 <= a.w.blocks) wait_copies<kLoads>();
    else wait_copies<0>();
    wg_barrier();
    // (not unrolled: operands of two parts leave the registers)
#pragma unroll 1
    for (int u = 0; u < 4; u += U) {
      Part part;
      read(part, buf, u);
      multiply(part);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wg_barrier();  // the stage is read
    if (kb + 2 < a.w.blocks) copies(kb + 2, buf);
    buf ^= 1;
  }

  // a lane holds row lane % 16 of each 16, columns 4 q .. 4 q + 3 of each tile: through LDS, so that rows are stored in whole lines
  constexpr int OUT = 16 * PER, PITCH = 64 * 4 + 16, LPR = OUT / 8, RPI = 64 / LPR;
  static_assert(16 * PITCH * 4 <= 2 * kStage && 16 % RPI == 0, "a part of LDS for each wave");
  const uint32_t mine = lds0 + (uint32_t)(wave * 16 * PITCH);
  const int orow = lane / LPR, ocol = lane % LPR * 8, n = n0 + wave * OUT + ocol;
  Columns cols;
  if (n < g.N) load_columns<false, NB == 2, OT>(g, n, cols);
#pragma unroll
  for (int i = 0; i < MF; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j)  // (float32: codes came as sixteenths)
      *(AX_LDS(f32x4)*)(uintptr_t)(mine + (uint32_t)((lane & 15) * PITCH + (16 * j + 4 * q) * 4)) = P == 3 ? acc[i][j] * 16.f : acc[i][j];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int r = 0; r < 16; r += RPI) {
      const int m = m0 + 16 * i + r + orow;
      const uint32_t from = mine + (uint32_t)((r + orow) * PITCH + ocol * 4);
      f32x4 s[2], s2[2];
      s[0] = *(const AX_LDS(f32x4)*)(uintptr_t)from;
      s[1] = *(const AX_LDS(f32x4)*)(uintptr_t)(from + 16);
      if (NB == 2) {
        s2[0] = *(const AX_LDS(f32x4)*)(uintptr_t)(from + OUT * 4);
        s2[1] = *(const AX_LDS(f32x4)*)(uintptr_t)(from + OUT * 4 + 16);
      }
      if (m < M && n < g.N) finish<false, NB == 2, OT>(g, cols, Ahead{}, row_at + m, n, s, s2, 0);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

long long grid_of(const Groups& e, int height, int wide) {
  return (e.offsets ? e.rows / height + std::min(e.experts, e.rows) : ((long long)e.rows + height - 1) / height) * wide;
}
int wide_of(long long N, bool gated) { return (int)((N + (gated ? 127 : 255)) / (gated ? 128 : 256)); }

template <int P, int NB, int MF, bool FOUND>
void launch_group(const TileArgs& a, int grid, hipStream_t s) {
  switch (a.w.group) {
    case 32: q4_tile_kernel<P, NB, MF, 32, FOUND><<<grid, 256, 0, s>>>(a); break;
    case 64: q4_tile_kernel<P, NB, MF, 64, FOUND><<<grid, 256, 0, s>>>(a); break;
    default: q4_tile_kernel<P, NB, MF, 128, FOUND><<<grid, 256, 0, s>>>(a); break;
  }
}

}  // namespace

// 64 rows a workgroup or 32: rounds of workgroups over the card, in us for 4096 columns of the contraction.  (300/4096/4096 64 : 32 rows 58 : 42,
// 1027/4096/4096 80 : 77, 2048/4096/4096 87 : 108, 2048 rows of 32 experts, 2048/1408 44 : 34; float32 512/4096/4096 107 : 77, 2048/4096/4096 228 : 285.)
int q4_tile_rows(const GemmArgs& g, const Groups& e) {
  const bool f32 = g.pieces == 3;
  const int wide = wide_of(g.N, g.gated != 0);
  const double experts = (double)std::max(1, e.offsets ? std::min(e.experts, e.rows) : 1), each = e.rows / experts;
  auto count = [&](int height) {
    return (long long)(wide * (e.experts == 1 ? std::ceil(each / height) : experts * std::max(1.0, each / height + 0.5)));
  };
  auto rounds = [](long long n, long long slots) { return (double)((n + slots - 1) / slots); };
  const long long n4 = count(64), n2 = count(32);
  const double cost4 = f32 ? 100 * rounds(n4, 256) : n4 <= 256 ? 57 : 84 * rounds(n4, 512);
  const double cost2 = f32 ? 70 * rounds(n2, 256) : n2 <= 256 ? 42 : 76 * rounds(n2, 768);
  return cost2 < cost4 ? 32 : 64;
}

bool q4_tiles_fit(const GemmArgs& g, const Groups& e) { return grid_of(e, q4_tile_rows(g, e), wide_of(g.N, g.gated != 0)) < 1 << 23; }

hipError_t launch_q4_tiles(const GemmArgs& g, const Groups& e, const Q4Weights& w, hipStream_t s) {
  TileArgs a{g, e, w, wide_of(g.N, g.gated != 0)};
  const bool f32 = g.pieces == 3, low = q4_tile_rows(g, e) == 32;
  const int n = (int)grid_of(e, low ? 32 : 64, a.wide);
  auto go = [&](auto p, auto nb, auto found) {
    constexpr int P = decltype(p)::value, NB = decltype(nb)::value;
    low ? launch_group<P, NB, 2, decltype(found)::value>(a, n, s) : launch_group<P, NB, 4, decltype(found)::value>(a, n, s);
  };
  constexpr auto one = std::integral_constant<int, 1>{};
  constexpr auto two = std::integral_constant<int, 2>{};
  constexpr auto three = std::integral_constant<int, 3>{};
  if (f32) g.gated ? go(three, two, std::false_type{}) : go(three, one, std::false_type{});
  else if (e.index) g.gated ? go(one, two, std::true_type{}) : go(one, one, std::true_type{});
  else g.gated ? go(one, two, std::false_type{}) : go(one, one, std::false_type{});
  return hipGetLastError();
}

}  // namespace ax
