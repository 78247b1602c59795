// Products with few rows on the left (a token, or a handful decoded together): every weight is read once and met by all rows.
//
// Bound by memory: 2 M operations for each weight.  So nothing is staged: a workgroup of 16 waves takes 16 to 64 columns
// of the result, its waves take turns along the contraction, and a lane loads weights straight into the registers that the
// matrix instruction wants (16 columns x 32 of the contraction, 64 for int8), several steps ahead of their use.  The
// waves' sums meet in LDS, in the waves' order, and the epilogue follows there: one launch, no partial sums in memory.  Only
// where the columns would leave compute units idle is the contraction cut, and a second launch joins the slices' sums.
//
// More than 32 rows (16 in one fragment) are several workgroups, neighbours, so that one reads what the other has brought to L2.
//
// Measured, weights from memory (us at rows / K / N): bf16 [N, K] 1/4096/4096 9.6 (3.5 TB/s), [K, N] 1/2048/8192 10.3
// (3.3 TB/s), float32 [K, N] 17/8192/8192 71.5 (3.75 TB/s); slices: float32 [K, N] 16/8192/512 13.5, uncut 45.
//
// Weights [N, K]: a lane holds 8 (int8: 16) consecutive elements of a row, what the instruction wants.  Weights [K, N]: a
// lane loads V neighbouring columns of eight rows, and the eight values of a column are put together by byte permutes;
// lane r of a fragment then stands for columns V r .. V r + V - 1, one for each of V matrix instructions.  float32 operands
// are cut into their three bf16 pieces in registers.
#include <algorithm>

#include "ax_float.h"
#include "ax_gemm.h"
#include "ax_group.h"

namespace ax {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 16, kThreads = 64 * kWaves;
enum Kind { kBf16, kInt8, kF32 };

struct Args {
  GemmArgs g;
  int blocks;   // of the contraction, per segment
  int tiles;    // workgroups along the columns
  int bands;    // of 16 MFR rows
  int slices;   // of the contraction, each `per` turns of a wave (over all segments)
  int per;
  float* part;  // [slices][NB][M][ldp] with slices, as the joining kernel reads them
  long long ldp;
  Groups e;                // rows grouped by expert
  const int32_t* index;    // of the grouped rows into those of x (null: the same)
  int x_rows;
  long long next;          // bytes from one expert's weights to the next one's
};

// One operand of the matrix instruction: bf16 or int8 as they are, float32 as three pieces.
template <Kind KD>
struct Frag {
  u32x4 p[KD == kF32 ? 3 : 1];
};

template <Kind KD, typename Acc>
__device__ __forceinline__ Acc mma(const Frag<KD>& a, const Frag<KD>& b, Acc c) {
  if constexpr (KD == kInt8) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a.p[0]), __builtin_bit_cast(i32x4, b.p[0]), c, 0, 0, 0);
  } else if constexpr (KD == kBf16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.p[0]), __builtin_bit_cast(bf16x8, b.p[0]), c, 0, 0, 0);
  } else {
    constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
    for (int i = 0; i < 6; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.p[pa[i]]), __builtin_bit_cast(bf16x8, b.p[pb[i]]), c, 0, 0, 0);
    return c;
  }
}

// A lane's share of a row with the contraction contiguous: raw bytes (32 for float32), `left` elements of them there.
// ODD: rows may start inside a word.  Reads of 16 bytes off the words cost two to three times as much (us at rows / K / N of
// [N, K], with and without ODD: bf16 16/4097/4096 18.1 : 28.5, int8 9.2 : 17.4), so the words that hold the bytes are read, and
// shifted when they are used.  No word is read that holds none of the row's elements.
template <Kind KD, bool ODD>
struct Along {
  u32x4 q[KD == kF32 ? 2 : 1];
  uint32_t next, shift;
  template <bool FULL>
  __device__ __forceinline__ void load(const char* row, int k, int left) {
    constexpr int E = KD == kInt8 ? 16 : 8, B = KD == kInt8 ? 1 : KD == kBf16 ? 2 : 4;
    const char* p = row + (long long)k * B;
    if (ODD && FULL) {
      shift = (uint32_t)(uintptr_t)row & 3u;  // (k elements are whole words)
      const char* words = p - shift;
      q[0] = load_any<u32x4>(words);
      next = *(const uint32_t*)(words + (shift ? 16 : 12));
      return;
    }
    if (ODD) shift = next = 0;
    if (FULL || left >= E) {
      q[0] = load_any<u32x4>(p);
      if (KD == kF32) q[KD == kF32 ? 1 : 0] = load_any<u32x4>(p + 16);
      return;
    }
#pragma unroll
    for (int w = 0; w < E * B / 4; ++w) {
      uint32_t v = 0;
#pragma unroll
      for (int e = 0; e < 4 / B; ++e) {
        const int i = w * (4 / B) + e;
        if (i < left) {
          if (B == 1) v |= (uint32_t)((const uint8_t*)p)[i] << (8 * e);
          else if (B == 2) v |= (uint32_t)((const uint16_t*)p)[i] << (16 * e);
          else v = ((const uint32_t*)p)[i];
        }
      }
      q[w >> 2][w & 3] = v;
    }
  }
  __device__ __forceinline__ void clear() {
    q[0] = u32x4{0, 0, 0, 0};
    if (KD == kF32) q[KD == kF32 ? 1 : 0] = q[0];
  }
  __device__ __forceinline__ void fragment(Frag<KD>& f) const {
    if constexpr (KD == kF32) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(q[e >> 2][e & 3]);
      pieces_of(v, f.p);
    } else if constexpr (ODD) {
#pragma unroll
      for (int w = 0; w < 4; ++w) f.p[0][w] = __builtin_amdgcn_alignbyte(w < 3 ? q[0][w < 3 ? w + 1 : 0] : next, q[0][w], shift);
    } else {
      f.p[0] = q[0];
    }
  }
};

// A lane's share of eight rows of V columns.
template <Kind KD, int V>
struct Across {
  static constexpr int W = V * (KD == kF32 ? 4 : 2) / 4;  // words a row
  uint32_t d[8][W];
  // p: first row's first column; rows_left, cols_left: how many of each there are
  template <bool FULL>
  __device__ __forceinline__ void load(const char* p, long long ld, int rows_left, int cols_left) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const char* r = p + j * ld;
      if (FULL) {
        typedef uint32_t words __attribute__((ext_vector_type(W)));
        const words v = load_any<words>(r);
#pragma unroll
        for (int w = 0; w < W; ++w) d[j][w] = W == 1 ? ((const uint32_t*)&v)[0] : v[w];
        continue;
      }
#pragma unroll
      for (int w = 0; w < W; ++w) d[j][w] = 0;
#pragma unroll
      for (int c = 0; c < V; ++c)
        if (j < rows_left && c < cols_left) {
          if (KD == kF32) d[j][c] = ((const uint32_t*)r)[c];
          else d[j][c >> 1] |= (uint32_t)((const uint16_t*)r)[c] << (16 * (c & 1));
        }
    }
  }
  __device__ __forceinline__ void fragment(int v, Frag<KD>& f) const {
    if constexpr (KD == kF32) {
      float t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = __uint_as_float(d[e][v]);
      pieces_of(t, f.p);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        f.p[0][e] = __builtin_amdgcn_perm(d[2 * e + 1][v >> 1], d[2 * e][v >> 1], (v & 1) ? 0x07060302u : 0x05040100u);
    }
  }
};

// LB: 0 = weights [N, K], 1 = [K, N].  NB: 2 for the gated pair.  MFR: fragments of 16 rows.  CF: fragments of 16 columns
// of one weight (LB = 1: neighbouring columns a lane).  U: steps of the contraction a wave loads at a time.
// ODD: rows may start inside a word (not for float32).  GR: rows grouped by expert; a workgroup has up to 16 MFR of one expert.
template <Kind KD, int LB, int NB, int MFR, int CF, int U, bool ODD, bool GR = false>
__global__ __launch_bounds__(kThreads) void few_kernel(const Args a) {
  constexpr int KS = KD == kInt8 ? 64 : 32, LANE = KS / 4;  // contraction of a step, of a lane
  constexpr int ES = KD == kInt8 ? 1 : KD == kBf16 ? 2 : 4;
  constexpr int COLS = 16 * CF;
  typedef typename std::conditional<KD == kInt8, i32x4, f32x4>::type Acc;
  __shared__ __align__(16) float part[kWaves][NB][16 * MFR][COLS + 4];
  const GemmArgs& g = a.g;
  const int t = threadIdx.x, lane = t & 63, r = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  // workgroups b, b + 8, ... share an XCD: they take neighbouring columns, which may share lines of memory
  int tile, slice = 0, m0 = 0, M = g.M, row_at = 0;
  long long w_at = 0;
  if constexpr (GR) {  // (the columns of one expert: workgroups of an XCD take neighbours)
    GroupTile e;
    if (!find_tile(a.e.offsets, a.e.experts, a.e.rows, 16 * MFR, a.tiles, blockIdx.x, e)) return;
    const int bands = e.tiles / a.tiles, k = e.tile;
    m0 = __builtin_amdgcn_readfirstlane(k % bands) * 16 * MFR;
    tile = __builtin_amdgcn_readfirstlane(k / bands);
    M = __builtin_amdgcn_readfirstlane(e.count);
    row_at = __builtin_amdgcn_readfirstlane(e.first);
    w_at = __builtin_amdgcn_readfirstlane(e.expert) * a.next;
  } else {
    const int b = blockIdx.x, x = b & 7, i = b >> 3, total = gridDim.x, per = total >> 3, more = total & 7;
    tile = x * per + min(x, more) + i;
    if (a.bands > 1) {  // neighbours: the weights come from memory once
      const int band = tile % a.bands;
      tile /= a.bands;
      m0 = band * 16 * MFR;
    }
    slice = a.slices > 1 ? tile / a.tiles : 0;
    tile -= slice * a.tiles;
  }
  const int n0 = tile * COLS;

  Acc acc[NB][MFR][CF];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < MFR; ++i)
#pragma unroll
      for (int j = 0; j < CF; ++j) acc[b][i][j] = Acc{};

  // grouped: where this lane's rows of x are
  long long x_at[GR ? MFR : 1];
  bool there[GR ? MFR : 1];
  if constexpr (GR) {
#pragma unroll
    for (int i = 0; i < MFR; ++i) {
      const int m = row_at + min(m0 + 16 * i + r, M - 1), k = a.index ? a.index[m] : m;
      there[i] = k >= 0 && k < a.x_rows;  // (another index stands for a row of zeros)
      x_at[i] = there[i] ? k * g.lda : 0;
    }
  }

  const bool all_cols = n0 + COLS <= g.N;
  const int groups = (a.blocks + U - 1) / U;
  const int behind = min((slice + 1) * a.per, groups * g.nseg);
  for (int it = slice * a.per + wave; it < behind; it += kWaves) {
    const int seg = __builtin_amdgcn_readfirstlane(g.nseg == 1 ? 0 : it / groups);
    const int k0 = (it - seg * groups) * U * KS;
    const char* x = (const char*)g.seg[seg].a;
    const char* w[2] = {(const char*)g.seg[seg].b + w_at, (const char*)g.seg[seg].b2 + w_at};
    auto run = [&](auto full) __attribute__((always_inline)) {
      Along<KD, ODD> xa[U][MFR];
      typename std::conditional<LB == 0, Along<KD, ODD>, Across<KD == kInt8 ? kBf16 : KD, CF>>::type wa[U][NB][LB == 0 ? CF : 1];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = k0 + u * KS + LANE * q, left = g.K - k;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if constexpr (LB == 0) {
#pragma unroll
            for (int j = 0; j < CF; ++j) {  // (rows behind the last: their results are not stored)
              const int n = min(n0 + 16 * j + r, g.N - 1);
              wa[u][b][j].template load<full>(w[b] + n * g.ldb, k, left);
            }
          } else {
            const int c = n0 + CF * r;
            wa[u][b][0].template load<full>(w[b] + k * g.ldb + (long long)c * ES, g.ldb, left, g.N - c);
          }
        }
#pragma unroll
        for (int i = 0; i < MFR; ++i) {
          if constexpr (GR) xa[u][i].template load<full>(x + x_at[i], k, left);
          else xa[u][i].template load<full>(x + min(m0 + 16 * i + r, g.M - 1) * g.lda, k, left);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        Frag<KD> fx[MFR];
#pragma unroll
        for (int i = 0; i < MFR; ++i) {
          if constexpr (GR) {
            if (!there[i]) xa[u][i].clear();
          }
          xa[u][i].fragment(fx[i]);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int j = 0; j < CF; ++j) {
            Frag<KD> fw;
            if constexpr (LB == 0) wa[u][b][j].fragment(fw);
            else wa[u][b][0].fragment(j, *(Frag<KD == kInt8 ? kBf16 : KD>*)&fw);
#pragma unroll
            for (int i = 0; i < MFR; ++i) acc[b][i][j] = mma<KD>(fw, fx[i], acc[b][i][j]);
          }
      }
    };
    if (k0 + U * KS <= g.K && (LB == 0 || all_cols)) run(std::true_type{});
    else run(std::false_type{});
  }

  // lane: row m = r of the fragment, weight rows 4 q .. 4 q + 3 of it
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < MFR; ++i)
#pragma unroll
      for (int j = 0; j < CF; ++j) {
        const f32x4 v = __builtin_bit_cast(f32x4, acc[b][i][j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) part[wave][b][16 * i + r][LB == 0 ? 16 * j + 4 * q + e : CF * (4 * q + e) + j] = v[e];
      }
  __syncthreads();
  for (int o = t; o < 16 * MFR * COLS; o += kThreads) {
    const int row = o / COLS, c = o - row * COLS, n = n0 + c, m = row_at + m0 + row;
    if (m0 + row >= M || n >= g.N) continue;
    float s[2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (KD == kInt8) {
        int32_t v = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += __float_as_int(part[w][b][row][c]);
        s[b] = a.slices > 1 ? __int_as_float(v) : (float)v * (g.xs[m] * (b ? g.ws2 : g.ws)[n]);
      } else {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += part[w][b][row][c];
        s[b] = v;
      }
    }
    if (a.slices > 1) {
#pragma unroll
      for (int b = 0; b < NB; ++b) a.part[((long long)(slice * NB + b) * g.M + m) * a.ldp + n] = s[b];
      continue;
    }
    auto put = [&](void* p, long long i, float v) {
      if (g.odt == AX_F32) ((float*)p)[i] = v;
      else ((uint16_t*)p)[i] = (uint16_t)f32_to_bf16(v);
    };
    auto get = [&](const void* p, long long i) { return g.odt == AX_F32 ? ((const float*)p)[i] : bf16_to_f32(((const uint16_t*)p)[i]); };
    float v[1] = {s[0]};
    if (NB == 1 && g.bias) v[0] += get(g.bias, n);
    if (g.z) put(g.z, (long long)m * g.N + n, v[0]);
    if (NB == 2 && g.z2) put(g.z2, (long long)m * g.N + n, s[1]);
    if (g.odt == AX_F32) apply_act<true>(v, g.act);
    else apply_act<false>(v, g.act);
    if (NB == 2) v[0] *= s[1];
    if (NB == 1 && g.res) v[0] += get(g.res, (long long)m * g.ldr + n);
    put(g.y, (long long)m * g.ldy + n, v[0]);
  }
}

// Fragments of 16 columns a workgroup takes: as many as leave a workgroup for every compute unit (wider pieces of a line,
// fewer reads of x).
constexpr int cols_of(Kind kd, int lb, int nb, int mfr, int n) {
  const bool wide = kd == kF32 && mfr == 2;  // (the pieces of 32 rows leave few registers)
  if (lb == 0) return mfr * nb < 4 && !wide && n >= 8192 ? 2 : 1;
  if (wide && nb == 2) return 1;
  return kd == kBf16 && mfr * nb == 1 && n >= 16384 ? 4 : 2;
}
// Steps of the contraction that a wave loads at a time: what 128 registers a lane hold.
constexpr int steps_of(Kind kd, int lb, int nb, int mfr) {
  if (kd == kF32) return nb == 2 || (lb == 1 && mfr == 2) ? 1 : 2;
  return 4 / nb;
}

template <Kind KD, int LB, int NB, int MFR>
void launch_cols(Args& a, hipStream_t s) {
  constexpr int U = steps_of(KD, LB, NB, MFR);
  uintptr_t low = (uintptr_t)a.g.lda;
  if (LB == 0) low |= (uintptr_t)a.g.ldb;
  for (int i = 0; i < a.g.nseg; ++i) {
    low |= (uintptr_t)a.g.seg[i].a;
    if (LB == 0) low |= (uintptr_t)a.g.seg[i].b | (uintptr_t)a.g.seg[i].b2;
  }
  const bool odd = KD != kF32 && (low & 3);
  auto go = [&](auto cf) {
    constexpr int CF = decltype(cf)::value;
    a.tiles = (a.g.N + 16 * CF - 1) / (16 * CF);
    a.bands = (a.g.M + 16 * MFR - 1) / (16 * MFR);
    a.per = ((a.blocks + U - 1) / U * a.g.nseg + a.slices - 1) / a.slices;
    const int n = a.tiles * a.slices * a.bands;
    if constexpr (KD != kF32 && CF < 4) {
      if (odd) {
        few_kernel<KD, LB, NB, MFR, CF, U, true><<<n, kThreads, 0, s>>>(a);
        return;
      }
    }
    few_kernel<KD, LB, NB, MFR, CF, U, false><<<n, kThreads, 0, s>>>(a);
  };
  const int cf = cols_of(KD, LB, NB, MFR, a.g.N);
  constexpr int most = cols_of(KD, LB, NB, MFR, 1 << 20), least = cols_of(KD, LB, NB, MFR, 1);
  if constexpr (most != least) {
    if (cf == most && (most < 4 || !odd)) return go(std::integral_constant<int, most>{});
  }
  go(std::integral_constant<int, least>{});
}
template <Kind KD, int LB, int NB>
void launch_rows(Args& a, hipStream_t s) {
  if (a.g.M > 16) return launch_cols<KD, LB, NB, 2>(a, s);
  launch_cols<KD, LB, NB, 1>(a, s);
}

// Grouped: 16 rows of an expert a workgroup, or 32 where an expert can expect more.
template <Kind KD, int LB, int NB, int MFR>
void launch_group(Args& a, hipStream_t s) {
  constexpr int U = steps_of(KD, LB, NB, MFR), CF = cols_of(KD, LB, NB, MFR, 1);
  a.tiles = (a.g.N + 16 * CF - 1) / (16 * CF);
  a.per = (a.blocks + U - 1) / U;
  const long long grid = (a.e.rows / (16 * MFR) + std::min(a.e.experts, a.e.rows)) * (long long)a.tiles;
  few_kernel<KD, LB, NB, MFR, CF, U, false, true><<<(int)grid, kThreads, 0, s>>>(a);
}
template <Kind KD, int LB, int NB>
void launch_group_rows(Args& a, hipStream_t s) {
  if (a.e.rows > 16 * std::min(a.e.experts, a.e.rows)) return launch_group<KD, LB, NB, 2>(a, s);
  launch_group<KD, LB, NB, 1>(a, s);
}

Kind kind_of(const GemmArgs& g, int dtype) { return g.i8 ? kInt8 : dtype == AX_BF16 ? kBf16 : kF32; }
int blocks_of(const GemmArgs& g) { return (g.K + (g.i8 ? 63 : 31)) / (g.i8 ? 64 : 32); }

}  // namespace

// A compute unit takes in some 18 KB a us from memory, whatever the others do, so few columns leave most of the card's rate
// unused: the contraction is cut where the workgroups' rounds, with the launch that joins their sums, come out shorter.  (The
// launch, the kernel and the workspace are 8 us a call to a program that calls the operators one by one: bf16 [K, N]
// 1/4096/4096 in two slices 13.9 us a call, uncut 11.4.)
FewPlan plan_few(const GemmArgs& g, int dtype) {
  const Kind kd = kind_of(g, dtype);
  const int nb = g.gated ? 2 : 1, mfr = g.M > 16 ? 2 : 1, cols = 16 * cols_of(kd, g.lb, nb, mfr, g.N), steps = steps_of(kd, g.lb, nb, mfr);
  const long long tiles = (long long)((g.N + cols - 1) / cols) * ((g.M + 16 * mfr - 1) / (16 * mfr)), groups = (long long)(blocks_of(g) + steps - 1) / steps * g.nseg;
  const double turn = kWaves * steps * (kd == kF32 ? 128.0 : 64.0) * (nb * cols + 0.5 * std::min(g.M, 32)) / 18e3;  // (x from the caches)
  FewPlan best{1, 0};
  double least = 1e300;
  for (int n = 1; n <= 16 && (n == 1 || n * kWaves < groups + kWaves); ++n) {
    const long long turns = ((groups + n - 1) / n + kWaves - 1) / kWaves;
    const double sums = n > 1 ? 8.0 + n * nb * g.M * (double)g.N * 8.0 / 4e6 : 0.0;
    const double cost = (double)((tiles * n + 255) / 256) * (turns * turn + 2.0) + sums;
    if (cost < least) {
      least = cost;
      best.slices = n;
    }
  }
  if (best.slices > 1) best.part_bytes = (size_t)best.slices * nb * g.M * (((size_t)g.N + 7) / 8 * 8) * 4;
  return best;
}

hipError_t launch_few(const GemmArgs& g, int dtype, const FewPlan& p, void* part, hipStream_t s) {
  Args a{};
  a.g = g;
  a.blocks = blocks_of(g);
  a.slices = p.slices;
  a.part = (float*)part;
  a.ldp = ((long long)g.N + 7) / 8 * 8;
  switch (kind_of(g, dtype)) {
    case kInt8: g.gated ? launch_rows<kInt8, 0, 2>(a, s) : launch_rows<kInt8, 0, 1>(a, s); break;
    case kBf16:
      if (g.gated) launch_rows<kBf16, 1, 2>(a, s);
      else g.lb == 0 ? launch_rows<kBf16, 0, 1>(a, s) : launch_rows<kBf16, 1, 1>(a, s);
      break;
    case kF32:
      if (g.gated) launch_rows<kF32, 1, 2>(a, s);
      else g.lb == 0 ? launch_rows<kF32, 0, 1>(a, s) : launch_rows<kF32, 1, 1>(a, s);
      break;
  }
  const hipError_t rc = hipGetLastError();
  return rc != hipSuccess || p.slices == 1 ? rc : launch_join(g, p.slices, part, s);
}

hipError_t launch_few_experts(const GemmArgs& g, int dtype, const Groups& e, const int32_t* index, int x_rows, hipStream_t s) {
  Args a{};
  a.g = g;
  a.blocks = blocks_of(g);
  a.slices = 1;
  a.e = e;
  a.index = index;
  a.x_rows = x_rows;
  a.next = (long long)(g.lb == 0 ? g.N : g.K) * g.ldb;
  if (kind_of(g, dtype) == kBf16) {
    if (g.gated) launch_group_rows<kBf16, 1, 2>(a, s);
    else g.lb == 0 ? launch_group_rows<kBf16, 0, 1>(a, s) : launch_group_rows<kBf16, 1, 1>(a, s);
  } else {
    if (g.gated) launch_group_rows<kF32, 1, 2>(a, s);
    else g.lb == 0 ? launch_group_rows<kF32, 0, 1>(a, s) : launch_group_rows<kF32, 1, 1>(a, s);
  }
  return hipGetLastError();
}

}  // namespace ax
