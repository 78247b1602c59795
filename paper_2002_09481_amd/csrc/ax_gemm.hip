// Matrix products on the matrix cores: bf16 operands with float32 sums, int8 codes with int32 sums.
#include <algorithm>

#include "ax_float.h"
#include "ax_gemm.h"

namespace ax {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

#define AX_LDS(T) __attribute__((address_space(3))) T

constexpr int kStepBytes = 128;  // contraction bytes per stage: 64 bf16 or 128 int8
constexpr uint32_t kOut = 0x80000000u;  // an offset behind every buffer: the load gives zeros

struct Args {
  GemmArgs g;
  int tiles_m, tiles_n;  // tiles_n counts both outputs of a dual launch
  int ksteps;            // stages per segment
  int splits;
  float* part;           // [splits][planes][M][ldp]
  long long ldp;
};

// ---- epilogue ----------------------------------------------------------------------------------

__device__ __forceinline__ void load4(const void* p, long long i, int dt, int left, float (&v)[4]) {
  if (dt == AX_F32) load_elems<true, 4>(p, i, left, v);
  else load_elems<false, 4>(p, i, left, v);
}
__device__ __forceinline__ void store4(void* p, long long i, int dt, int left, const float (&v)[4]) {
  if (dt == AX_F32) store_elems<true, 4>(p, i, left, v);
  else store_elems<false, 4>(p, i, left, v);
}

// Columns n .. n + 3 of row m from the finished sums (int8: already scaled).  second: the second output of a dual launch.
__device__ __forceinline__ void finish(const GemmArgs& g, int m, int n, const float (&s)[4], int second) {
  const int left = g.N - n;
  float v[4];
  for (int e = 0; e < 4; ++e) v[e] = s[e];
  if (g.bias) {
    float b[4];
    load4(g.bias, n, g.odt, left, b);
    for (int e = 0; e < 4; ++e) v[e] += b[e];
  }
  if (g.z) store4(g.z, (long long)m * g.N + n, g.odt, left, v);
  if (g.act != AX_ACT_NONE)
    for (int e = 0; e < 4; ++e) v[e] = act_of(v[e], g.act);
  if (g.res) {
    float r[4];
    load4(g.res, (long long)m * g.ldr + n, g.odt, left, r);
    for (int e = 0; e < 4; ++e) v[e] += r[e];
  }
  if (second) store4(g.y2, (long long)m * g.ldy + n, g.odt, left, v);
  else store4(g.y, (long long)m * g.ldy + n, g.odt, left, v);
}
__device__ __forceinline__ void finish_gated(const GemmArgs& g, int m, int n, const float (&a)[4], const float (&u)[4]) {
  const int left = g.N - n;
  if (g.z) store4(g.z, (long long)m * g.N + n, g.odt, left, a);
  if (g.z2) store4(g.z2, (long long)m * g.N + n, g.odt, left, u);
  float v[4];
  for (int e = 0; e < 4; ++e) v[e] = act_of(a[e], g.act) * u[e];
  store4(g.y, (long long)m * g.ldy + n, g.odt, left, v);
}
// int8: scales of four columns and of a row.
__device__ __forceinline__ void scaled4(const int32_t (&c)[4], float xs, const float* ws, int n, int N, float (&v)[4]) {
  for (int e = 0; e < 4; ++e) v[e] = (float)c[e] * (xs * (n + e < N ? ws[n + e] : 0.f));
}

// ---- main kernel -------------------------------------------------------------------------------

// 16 bytes per lane from memory to LDS at dst + 16 * lane (dst uniform over the wave).  Written as instructions: of a
// copy that it knows, the compiler makes every later LDS read wait, since it cannot tell the stages apart.
__device__ __forceinline__ void lds_copy(uint32_t dst, uint32_t off, const u32x4& rsrc) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(dst), "v"(off), "s"(rsrc) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(N) : "memory");
}
__device__ __forceinline__ void wg_barrier() {
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// One operand's share of the copies.  L = 0: rows of kStepBytes, contraction contiguous; a row's eight 16-byte chunks
// are stored at chunk ^ ((row >> 1) & 7), which gives the 16 lanes of each pass of a 16-byte LDS read 16 different
// slots of the 64 banks.  L = 1 (bf16): 64 rows (the contraction) of R elements; 32-byte chunk pairs are stored at
// pair ^ (bits 0, 1 and 3 of the row), for the transposing 8-byte reads.
template <int L, int R, int THREADS>
struct Stager {
  static constexpr int kLoads = R * kStepBytes / 16 / THREADS;
  static_assert(kLoads >= 1, "a copy per thread at least");
  static constexpr int kRowChunks = L == 0 ? 8 : R / 8;
  static constexpr int kPairMask = R / 16 - 1;  // L = 1
  uint32_t off[kLoads];
  int chunk;  // L = 0: this thread's chunk (the same in all its copies)

  __device__ __forceinline__ void init(int t, long long ld, int cols_left) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int q = i * THREADS + t;
      const int row = q / kRowChunks, pos = q % kRowChunks;
      if (L == 0) {
        chunk = pos ^ ((row >> 1) & 7);
        off[i] = (uint32_t)(row * ld + chunk * 16);
      } else {
        const int sp = ((row & 3) | ((row >> 1) & 4)) & kPairMask;
        const int c = pos ^ (sp << 1);
        off[i] = c * 8 < cols_left ? (uint32_t)(row * ld + c * 16) : kOut;
      }
    }
  }
  // base: first byte of the stage's tile, rem: bytes from there to the operand's end, kleft: bytes of the contraction
  // left in the segment (L = 0: chunks behind them are zeros; L = 1: rows behind them lie behind the end).
  __device__ __forceinline__ void copy(uint32_t lds, const char* base, long long rem, int kleft) const {
    const uint32_t n = rem > 0x7fffffffll ? 0x7fffffffu : (uint32_t)rem;
    const u32x4 rsrc = {(uint32_t)(uintptr_t)base, (uint32_t)((uintptr_t)base >> 32) & 0xffffu, n, 0x00020000u};
    const bool mine = L == 1 || chunk * 16 < kleft;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) lds_copy(lds + i * (THREADS * 16), mine ? off[i] : kOut, rsrc);
  }
};

// The matrix instruction's operand for 16 rows starting at r0, contraction elements 16 g .. (bytes) of half ks.
template <int L, int R>
__device__ __forceinline__ u32x4 fragment(uint32_t lds, int r0, int ks, int lane) {
  const int r = lane & 15, g = lane >> 4;
  if (L == 0) {
    const uint32_t a = lds + (uint32_t)((r0 + r) * kStepBytes + (((ks * 4 + g) ^ ((r >> 1) & 7)) << 4));
    return *(const AX_LDS(u32x4)*)(uintptr_t)a;
  }
  const int kr = r >> 2;
  const int sp = (kr | ((g & 1) << 2)) & (R / 16 - 1);
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
// projections).  WM x WN waves, STAGES stages of LDS.
template <bool I8, int LA, int LB, int NB, int BM, int BN, int WM, int WN, int STAGES, int OCC>
__global__ __launch_bounds__(64 * WM * WN, OCC) void gemm_kernel(const Args a) {
  constexpr int THREADS = 64 * WM * WN;
  constexpr int BNS = BN / NB;                // columns of one right operand
  constexpr int MF = BM / WM / 16, NF = BN / WN / 16;
  constexpr int kABytes = BM * kStepBytes, kBBytes = BNS * kStepBytes;
  constexpr int kStage = kABytes + NB * kBBytes;
  typedef Stager<LA, BM, THREADS> SA;
  typedef Stager<LB, BNS, THREADS> SB;
  constexpr int kLoads = SA::kLoads + NB * SB::kLoads;
  __shared__ __align__(1024) unsigned char smem[STAGES * kStage];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(AX_LDS(unsigned char)*)smem;

  const GemmArgs& g = a.g;
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave % WM, wn = wave / WM;

  // Tiles XCD by XCD: workgroups b, b + 8, ... share an XCD (and its L2) and take a contiguous run of tiles; runs go
  // down blocks of eight row tiles before they move to the next column tile.
  const int total = a.tiles_m * a.tiles_n * a.splits;
  int tile;
  {
    const int b = blockIdx.x, x = b & 7, i = b >> 3, per = total >> 3, more = total & 7;
    tile = x * per + min(x, more) + i;
  }
  const int split = tile / (a.tiles_m * a.tiles_n);
  tile -= split * (a.tiles_m * a.tiles_n);
  int tm, tn;
  {
    const int band = 8 * a.tiles_n, b = tile / band, r = tile - b * band;
    const int h = min(8, a.tiles_m - 8 * b);
    tm = 8 * b + r % h;
    tn = r / h;
  }
  int second = 0;
  if (NB == 1 && g.dual) {
    const int half = a.tiles_n >> 1;
    second = tn >= half;
    tn -= second * half;
  }
  const int m0 = tm * BM, n0 = tn * BNS;

  const int steps = g.nseg * a.ksteps;
  const int s_beg = (int)((long long)steps * split / a.splits), s_end = (int)((long long)steps * (split + 1) / a.splits);
  const int n_st = s_end - s_beg;

  SA sa;
  SB sb;
  sa.init(t, g.lda, g.M - m0);
  sb.init(t, g.ldb, g.N - n0);

  // the next stage to copy: segment, stage within it, operand positions
  constexpr int kElem = I8 ? 1 : 2;
  constexpr int kStepK = kStepBytes / kElem;
  const long long a_step = LA == 0 ? kStepBytes : kStepK * g.lda, b_step = LB == 0 ? kStepBytes : kStepK * g.ldb;
  // bytes from the tile's first element to the operand's end; rows are whole 16-byte chunks, and a chunk that only began
  // in front of the end would not be loaded at all
  const long long row_bytes = ((long long)g.K * kElem + 15) & ~15ll;
  const long long a_all = LA == 0 ? (long long)(g.M - 1 - m0) * g.lda + row_bytes
                                  : (long long)(g.K - 1) * g.lda + (long long)(((g.M + 7) & ~7) - m0) * kElem;
  const long long b_all = LB == 0 ? (long long)(g.N - 1 - n0) * g.ldb + row_bytes
                                  : (long long)(g.K - 1) * g.ldb + (long long)(((g.N + 7) & ~7) - n0) * kElem;
  int seg = s_beg / a.ksteps, ks = s_beg - seg * a.ksteps;
  const char *pa, *pb, *pb2;
  long long ra, rb;
  auto at_segment = [&]() {
    const long long ao = LA == 0 ? (long long)m0 * g.lda : (long long)m0 * kElem;
    const long long bo = LB == 0 ? (long long)n0 * g.ldb : (long long)n0 * kElem;
    pa = (const char*)g.seg[seg].a + ao + ks * a_step;
    pb = (const char*)(second ? g.seg[seg].b2 : g.seg[seg].b) + bo + ks * b_step;
    if (NB == 2) pb2 = (const char*)g.seg[seg].b2 + bo + ks * b_step;
    ra = a_all - ks * a_step;
    rb = b_all - ks * b_step;
  };
  at_segment();
  auto issue = [&](int buf) {
    const uint32_t l = lds0 + (uint32_t)(buf * kStage + wave * 1024);
    const int kleft = (g.K - ks * kStepK) * kElem;
    sa.copy(l, pa, ra, kleft);
    sb.copy(l + kABytes, pb, rb, kleft);
    if (NB == 2) sb.copy(l + kABytes + kBBytes, pb2, rb, kleft);
    if (++ks == a.ksteps) {
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
  auto compute = [&](int buf) {
    const uint32_t la = lds0 + (uint32_t)(buf * kStage), lb = la + kABytes;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      u32x4 fb[NF], fa[MF];
#pragma unroll
      for (int j = 0; j < NF; ++j)
        fb[j] = NB == 2 ? fragment<LB, BNS>(lb + (j & 1) * kBBytes, wcol + 16 * (j >> 1), kk, lane)
                        : fragment<LB, BNS>(lb, wcol + 16 * j, kk, lane);
#pragma unroll
      for (int i = 0; i < MF; ++i) fa[i] = fragment<LA, BM>(la, wrow + 16 * i, kk, lane);
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = Acc<I8>::mma(fb[j], fa[i], acc[i][j]);
    }
  };

#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s)
    if (s < n_st) issue(s);
  int buf = 0;
  for (int it = 0; it < n_st; ++it) {
    if (n_st - 1 - it >= STAGES - 2) wait_copies<(STAGES - 2) * kLoads>();
    else wait_copies<0>();
    wg_barrier();
    if (it + STAGES - 1 < n_st) issue(buf == 0 ? STAGES - 1 : buf - 1);
    compute(buf);
    buf = buf + 1 == STAGES ? 0 : buf + 1;
  }

  // lane: row m, columns n .. n + 3 of every 16 x 16 block
  const int lm = lane & 15, ln = (lane >> 4) * 4;
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int m = m0 + wrow + 16 * i + lm;
    if (m >= g.M) continue;
#pragma unroll
    for (int j = 0; j < NF; j += NB) {
      const int n = n0 + wcol + 16 * (j / NB) + ln;
      if (n >= g.N) continue;
      if (a.splits > 1) {
        const long long plane = (long long)g.M * a.ldp;
        const int planes = NB == 2 || g.dual ? 2 : 1;
        float* p = a.part + ((long long)split * planes + second) * plane + (long long)m * a.ldp + n;
        *(u32x4*)p = __builtin_bit_cast(u32x4, acc[i][j]);
        if (NB == 2) *(u32x4*)(p + plane) = __builtin_bit_cast(u32x4, acc[i][j + NB - 1]);
        continue;
      }
      float v[4], u[4];
      if (I8) {
        const float xs = g.xs[m];
        int32_t c[4], c2[4];
        for (int e = 0; e < 4; ++e) {
          c[e] = (int32_t)acc[i][j][e];
          c2[e] = (int32_t)acc[i][j + NB - 1][e];
        }
        scaled4(c, xs, g.ws, n, g.N, v);
        if (NB == 2) scaled4(c2, xs, g.ws2, n, g.N, u);
      } else {
        for (int e = 0; e < 4; ++e) {
          v[e] = (float)acc[i][j][e];
          u[e] = (float)acc[i][j + NB - 1][e];
        }
      }
      if (NB == 2) finish_gated(g, m, n, v, u);
      else finish(g, m, n, v, second);
    }
  }
}

// Partial sums of the slices, added in their order, and the epilogue: four columns a thread.
template <bool I8>
__global__ __launch_bounds__(256) void gemm_join_kernel(const Args a) {
  const GemmArgs& g = a.g;
  const int quads = (int)(a.ldp >> 2);
  const int planes = g.gated || g.dual ? 2 : 1;
  const int outs = g.dual ? 2 : 1;
  const long long plane = (long long)g.M * a.ldp;
  const long long total = (long long)outs * g.M * quads;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const int second = i >= (long long)g.M * quads;
    const long long r = i - (second ? (long long)g.M * quads : 0);
    const int m = (int)(r / quads), n = (int)(r - (long long)m * quads) * 4;
    float v[2][4];
#pragma unroll
    for (int pl = 0; pl < 2; ++pl) {
      if (pl && !g.gated) break;
      const float* p = a.part + (long long)(second + pl) * plane + (long long)m * a.ldp + n;
      if (I8) {
        i32x4 s = {0, 0, 0, 0};
        for (int k = 0; k < a.splits; ++k) s += *(const i32x4*)(p + (long long)k * planes * plane);
        int32_t c[4] = {s[0], s[1], s[2], s[3]};
        scaled4(c, g.xs[m], pl ? g.ws2 : g.ws, n, g.N, v[pl]);
      } else {
        f32x4 s = *(const f32x4*)p;
        for (int k = 1; k < a.splits; ++k) s += *(const f32x4*)(p + (long long)k * planes * plane);
        for (int e = 0; e < 4; ++e) v[pl][e] = s[e];
      }
    }
    if (g.gated) finish_gated(g, m, n, v[0], v[1]);
    else finish(g, m, n, v[0], second);
  }
}

struct TileShape {
  int bm, bn, wgs;  // wgs: workgroups per compute unit
};
constexpr TileShape kTiles[3] = {{256, 256, 1}, {128, 128, 2}, {32, 128, 2}};

template <bool I8, int LA, int LB, int NB>
void launch_tile(const Args& a, int tile, int grid, hipStream_t s) {
  switch (tile) {
    case 0: gemm_kernel<I8, LA, LB, NB, 256, 256, 2, 4, 2, 2><<<grid, 512, 0, s>>>(a); break;
    case 1: gemm_kernel<I8, LA, LB, NB, 128, 128, 2, 2, 2, 2><<<grid, 256, 0, s>>>(a); break;
    default:
      if constexpr (LA == 0) gemm_kernel<I8, LA, LB, NB, 32, 128, 1, 4, 3, 2><<<grid, 256, 0, s>>>(a);
      break;
  }
}

}  // namespace

GemmPlan plan_gemm(const GemmArgs& g) {
  const int elem = g.i8 ? 1 : 2, kstep = kStepBytes / elem;
  const int ksteps = (g.K + kstep - 1) / kstep, steps = ksteps * g.nseg;
  const int cus = 256;
  GemmPlan best{};
  double best_t = 1e30;
  for (int t = 0; t < 3; ++t) {
    if (t == 2 && g.la != 0) continue;
    const TileShape& T = kTiles[t];
    const int bns = T.bn / (g.gated ? 2 : 1);
    const long long tiles = (long long)((g.M + T.bm - 1) / T.bm) * ((g.N + bns - 1) / bns) * (g.dual ? 2 : 1);
    const long long slots = (long long)cus * T.wgs;
    for (int sp = 1; sp <= 16 && sp * 4 <= std::max(4, steps); sp *= 2) {
      const long long rounds = (tiles * sp + slots - 1) / slots;
      // a stage of the tile, in units of a 128 x 128 x 64 step of a workgroup that has its unit half for itself
      const double step = t == 0 ? 1.75 : t == 1 ? 1.0 : 0.55;
      double cost = rounds * ((steps + sp - 1) / sp * step + 6.0);
      if (sp > 1) cost += 8.0 + sp * (double)g.M * g.N * (g.gated || g.dual ? 2 : 1) * 8.0 / 4e6;
      if (cost < best_t) {
        best_t = cost;
        best.tile = t;
        best.splits = sp;
      }
    }
  }
  const long long ldp = (g.N + 3) / 4 * 4;
  best.part_bytes = best.splits > 1 ? (size_t)best.splits * (g.gated || g.dual ? 2 : 1) * g.M * ldp * 4 : 0;
  return best;
}

hipError_t launch_gemm(const GemmArgs& g, const GemmPlan& p, void* part, hipStream_t s) {
  Args a;
  a.g = g;
  const TileShape& T = kTiles[p.tile];
  const int bns = T.bn / (g.gated ? 2 : 1);
  const int kstep = kStepBytes / (g.i8 ? 1 : 2);
  a.tiles_m = (g.M + T.bm - 1) / T.bm;
  a.tiles_n = (g.N + bns - 1) / bns * (g.dual ? 2 : 1);
  a.ksteps = (g.K + kstep - 1) / kstep;
  a.splits = p.splits;
  a.part = (float*)part;
  a.ldp = (g.N + 3) / 4 * 4;
  const long long grid = (long long)a.tiles_m * a.tiles_n * p.splits;
  if (grid <= 0 || grid > 0x7fffffffll) return hipErrorInvalidValue;
  const int n = (int)grid;
  if (g.gated) {
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
  hipError_t rc = hipGetLastError();
  if (rc != hipSuccess || p.splits == 1) return rc;
  const long long quads = (long long)(g.dual ? 2 : 1) * g.M * (a.ldp / 4);
  const int jg = (int)std::min<long long>((quads + 255) / 256, 4096);
  if (g.i8) gemm_join_kernel<true><<<jg, 256, 0, s>>>(a);
  else gemm_join_kernel<false><<<jg, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ax
