// Matrix products with a fused epilogue, the gated feed-forward block, and their gradients: validation, operand
// preparation and the launches of ax_gemm.hip.
//
//   z = x w + bias,  y = act(z) + residual         gz = gy act'(z),  gx = gz w^T,  gw = x^T gz,  gb = sum of gz
//   g = x wg,  u = x wu,  h = act(g) u             gg = gh u act'(g),  gu = gh act(g),  gx = gg wg^T + gu wu^T, ...
//
// The matrix instructions take bf16 (or int8) operands.  float32 operands are cut into three bf16 pieces,
// a = a1 + a2 + a3 exactly (eight significant bits each), and six of the nine products of pieces are added: what is left out
// is within 2^-24 (1 + 2^-8) of a b, of either sign.  That is 6 / 16 of the cost of the float32 matrix instruction, at its precision.
#include <algorithm>

#include "ax_float.h"
#include "ax_norm.h"
#include "ax_operand.h"
#include "axconv_probe.h"

namespace ax {
namespace {

// Rows copied into the form the products read: eight elements (16 bytes of output; int8: 16) a thread, all the operands of a
// product in one launch.  Bound by memory: 4 bytes read and 6 written per float32 element (28 M of them 45 us, 6.3 TB/s with
// part of it in the caches).
template <int DT>
__device__ __forceinline__ void pack_rows(const PackBatch& b, int block) {
  constexpr int E = DT == kI8 ? 16 : 8;
  const int k = block >= b.first[2] ? 2 : block >= b.first[1] ? 1 : 0;
  const PackJob& j = b.job[k];
  const long long groups = j.pcols / E, total = j.rows * groups;
  for (long long i = (long long)(block - b.first[k]) * 256 + threadIdx.x; i < total; i += (long long)b.blocks[k] * 256) {
    const long long r = i / groups, c = (i - r * groups) * E;
    long long left = j.cols - c, from = r;
    if (j.index) {
      from = j.index[r];
      if (from < 0 || from >= j.src_rows) from = left = 0;
    }
    if (DT == AX_F32) {
      float v[8];
      load_elems<true, 8>(j.src, from * j.ld + c, (int)min(left, 8ll), v);
      u32x4 q[3];
      pieces_of(v, q);
#pragma unroll
      for (int p = 0; p < 3; ++p) *(u32x4*)((uint16_t*)j.dst + (p * j.rows + r) * j.pitch + c) = q[p];
    } else if (DT == AX_BF16) {
      const uint16_t* s = (const uint16_t*)j.src + from * j.ld + c;
      u32x4 q;
      if (left >= 8) q = load_any<u32x4>(s);
      else for (int e = 0; e < 4; ++e)
        q[e] = (2 * e < left ? (uint32_t)s[2 * e] : 0u) | ((2 * e + 1 < left ? (uint32_t)s[2 * e + 1] : 0u) << 16);
      *(u32x4*)((uint16_t*)j.dst + r * j.pitch + c) = q;
    } else {
      const uint8_t* s = (const uint8_t*)j.src + from * j.ld + c;
      u32x4 q;
      if (left >= 16) q = load_any<u32x4>(s);
      else for (int e = 0; e < 4; ++e) {
        q[e] = 0;
        for (int x = 0; x < 4; ++x) q[e] |= (4 * e + x < left ? (uint32_t)s[4 * e + x] : 0u) << (8 * x);
      }
      *(u32x4*)((uint8_t*)j.dst + r * j.pitch + c) = q;
    }
  }
}

template <int DT>
__global__ __launch_bounds__(256) void pack_kernel(const PackBatch b) {
  pack_rows<DT>(b, blockIdx.x);
}

}  // namespace

int fill_pack(PackBatch* b, const PackJob* jobs, const bool* wanted, int n) {
  int k = 0, grid = 0;
  for (int i = 0; i < 3; ++i) b->first[i] = 0x7fffffff;
  for (int i = 0; i < n; ++i) {
    const PackJob& j = jobs[i];
    if (!wanted[i] || !j.dst || j.rows == 0) continue;
    b->job[k] = j;
    b->first[k] = grid;
    b->blocks[k] = grid_for(j.rows * (j.pcols / (j.dtype == kI8 ? 16 : 8)));
    grid += b->blocks[k++];
  }
  return grid;
}
hipError_t run_pack(const PackBatch& b, int grid, hipStream_t s) {
  if (grid == 0) return hipSuccess;
  const int dtype = b.job[0].dtype;  // the same for all operands of an operation
  if (dtype == AX_F32) pack_kernel<AX_F32><<<grid, 256, 0, s>>>(b);
  else if (dtype == AX_BF16) pack_kernel<AX_BF16><<<grid, 256, 0, s>>>(b);
  else pack_kernel<kI8><<<grid, 256, 0, s>>>(b);
  return hipGetLastError();
}

namespace {

// ---- elementwise part of the gradients ---------------------------------------------------------------------------
//
// gz = gy act'(z) (GATED: gg and gu) in the form the products read, and the sums of gz over blocks of rows.  A
// workgroup takes 256 columns (eight a thread) and `rows_per` rows, eight at a time.  Bound by memory: gated, 4101 x 5512
// bf16, 226 MB in 46 us, 4.9 TB/s.
//
// bf16: gz is rounded to bf16, since the matrix instructions take 16-bit operands.  The products' error grows from that of their
// results' own rounding, 1.7e-3 in the 2-norm, to 2.3e-3 (gated gradients, 4101 x 2048 -> 5512); as two pieces gz would double
// both products (380 of 460 us).  The sums of gz, and outer_kernel's weight gradients, take it unrounded.
template <int DT>
__device__ __forceinline__ void write_planes(void* dst, long long rows, long long pitch, long long r, long long c, const float (&v)[8]) {
  if (DT == AX_F32) {
    u32x4 q[3];
    pieces_of(v, q);
#pragma unroll
    for (int k = 0; k < 3; ++k) *(u32x4*)((uint16_t*)dst + (k * rows + r) * pitch + c) = q[k];
  } else {
    *(uint4*)((uint16_t*)dst + r * pitch + c) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
}

// The copies that the products need as well come in the same launch, behind: neither waits for the other (us of all gradients
// at rows / K / N, together : in two launches: bf16 64/501/701 17.8 : 20.0, float32 333/2001/1003 48.0 : 51.9).
template <int DT, bool GATED>
__global__ __launch_bounds__(256) void act_grad_kernel(const GradArgs a, const PackBatch copies) {
  if ((int)blockIdx.x >= a.blocks) {
    pack_rows<DT>(copies, blockIdx.x - a.blocks);
    return;
  }
  const int by = blockIdx.x / a.wide, bx = blockIdx.x - by * a.wide;
  const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
  const long long c = ((long long)bx * 32 + cx) * 8;
  const int r0 = by * a.rows_per, r1 = min(a.M, r0 + a.rows_per);
  const int left = (int)max(0ll, min(8ll, a.N - c));
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c < a.pcols) {
    for (int r = r0 + ry; r < r1; r += 8) {
      float gy[8], z[8], u[8];
      load_elems<DT == AX_F32, 8>(a.gy, (long long)r * a.ldy + c, left, gy);
      if (GATED || a.z) load_elems<DT == AX_F32, 8>(a.z, (long long)r * a.N + c, left, z);
      if (GATED || a.z) {
        float v[8], sl[8];
        act_and_slope<DT == AX_F32>(z, a.act, v, sl);
        if (GATED) {
          load_elems<DT == AX_F32, 8>(a.u, (long long)r * a.N + c, left, u);
          for (int e = 0; e < 8; ++e) {
            v[e] *= gy[e];
            gy[e] = gy[e] * u[e] * sl[e];
          }
          write_planes<DT>(a.gu, a.M, a.pitch, r, c, v);
        } else {
          for (int e = 0; e < 8; ++e) gy[e] *= sl[e];
        }
      }
      if (a.gz) write_planes<DT>(a.gz, a.M, a.pitch, r, c, gy);
      if (!GATED)
        for (int e = 0; e < 8; ++e) sum[e] += gy[e];
    }
  }
  if (GATED || !a.part) return;
  __shared__ float red[8][32][9];
  for (int e = 0; e < 8; ++e) red[ry][cx][e] = sum[e];
  __syncthreads();
  const int x = threadIdx.x >> 3, e = threadIdx.x & 7;
  const long long col = ((long long)bx * 32 + x) * 8 + e;
  if (col >= a.N) return;
  float t = 0.f;
  for (int y = 0; y < 8; ++y) t += red[y][x][e];
  a.part[(long long)by * a.N + col] = t;
}

// ---- gradients of few rows -----------------------------------------------------------------------------------------
//
// With few rows the weight's gradient is a sum of that many outer products: bound by writing it, no work for the matrix
// instructions.  outer_kernel computes gz where it needs it (GATED: gg for one weight, gu for the other, blockIdx.z), and
// leaves it and its sum over the rows for the input's gradient and the bias's: two launches in all.
// A workgroup has 32 rows of the gradient and 512 columns, a lane eight of each; both factors come from LDS, which holds
// ROWS rows (16 or 32) of them.  3 x 97 x 2920 float32: 5 us, of 8 x 616 x 11679 gated bf16 both 19.
struct OuterArgs {
  const void* x;   // [M, K]
  const void* gy;  // [M, N] (GATED: gh)
  const void* z;   // [M, N] pitch N; null: gz = gy
  const void* u;   // GATED
  void* gw[2];     // [K, N], or [N, K] where transposed; may be null
  void* gz[2];     // [M, N], may be null
  float* gb;       // may be null
  long long x_ld, gy_ld, gw_ld;
  int M, N, K, act, transposed;
};
template <int DT, bool GATED, int ROWS>
__global__ __launch_bounds__(256) void outer_kernel(const OuterArgs a) {
  constexpr bool F32 = DT == AX_F32;
  constexpr int R = 32, C = 512;
  __shared__ __align__(16) float rows[ROWS][R], cols[ROWS][C];
  const int which = GATED ? blockIdx.z : 0;
  const int r0 = blockIdx.y * R, c0 = blockIdx.x * C;
  const int nr = a.transposed ? a.N : a.K, nc = a.transposed ? a.K : a.N;
  // eight values m, i .. i + 7 of gz
  auto grad8 = [&](int m, int i, float (&g)[8]) {
    const int left = a.N - i;
    load_elems<F32, 8>(a.gy, m * a.gy_ld + i, left, g);
    if (!a.z) return;
    float z[8], v[8], sl[8];
    load_elems<F32, 8>(a.z, (long long)m * a.N + i, left, z);
    act_and_slope<DT == AX_F32>(z, a.act, v, sl);
    if (GATED) {
      float u[8];
      load_elems<F32, 8>(a.u, (long long)m * a.N + i, left, u);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] *= which ? v[e] : u[e] * sl[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] *= sl[e];
    }
  };
  auto stage = [&](float* dst, int width, int i0, bool grad, bool first) {
    for (int t = threadIdx.x; t < a.M * (width / 8); t += 256) {
      const int m = t / (width / 8), i = (t - m * (width / 8)) * 8;
      float v[8];
      if (grad) {
        grad8(m, i0 + i, v);
        if (first && a.gz[which]) store_elems<F32, 8>(a.gz[which], (long long)m * a.N + i0 + i, a.N - i0 - i, v);
      } else {
        load_elems<F32, 8>(a.x, m * a.x_ld + i0 + i, a.K - i0 - i, v);
      }
      *(f32x4*)(dst + m * width + i) = f32x4{v[0], v[1], v[2], v[3]};
      *(f32x4*)(dst + m * width + i + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
  };
  const bool first = a.transposed ? blockIdx.x == 0 : blockIdx.y == 0;  // of the workgroups that share a piece of gz
  if (a.transposed || a.gw[which]) stage(&rows[0][0], R, r0, a.transposed, first);
  if (!a.transposed || a.gw[which]) stage(&cols[0][0], C, c0, !a.transposed, first);
  __syncthreads();
  if (!GATED && a.gb && first) {
    const float* v = a.transposed ? &rows[0][0] : &cols[0][0];
    const int width = a.transposed ? R : C, n0 = a.transposed ? r0 : c0;
    for (int i = threadIdx.x; i < width && n0 + i < a.N; i += 256) {
      float t = 0.f;
      for (int m = 0; m < a.M; ++m) t += v[m * width + i];
      a.gb[n0 + i] = t;
    }
  }
  if (!a.gw[which]) return;
  const int r = (threadIdx.x >> 6) * 8, c = (threadIdx.x & 63) * 8;
  float acc[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
  for (int m = 0; m < a.M; ++m) {
    float x[8], y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = rows[m][r + i];
      y[i] = cols[m][c + i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[i][j] = __builtin_fmaf(x[i], y[j], acc[i][j]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (r0 + r + i < nr) store_elems<F32, 8>(a.gw[which], (long long)(r0 + r + i) * a.gw_ld + c0 + c, nc - c0 - c, acc[i]);
}

// rows x cols elements of `bytes` bytes at pitch ld set to zero.
__global__ __launch_bounds__(256) void zero_rows_kernel(uint8_t* p, long long rows, long long row_bytes, long long ld_bytes) {
  const long long total = rows * (row_bytes / 2);
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const long long r = i / (row_bytes / 2);
    *(uint16_t*)(p + r * ld_bytes + (i - r * (row_bytes / 2)) * 2) = 0;
  }
}

// ---- checks ------------------------------------------------------------------------------------------------------

int check_desc(const ax_matmul_desc_t* d, bool q8, bool backward, bool gated) {
  if (!d) return AX_ERR_NULL;
  if (!dtype_ok(d->out_dtype) || (!q8 && !dtype_ok(d->dtype))) return AX_ERR_OPTION;
  if (backward && d->out_dtype != d->dtype) return AX_ERR_OPTION;
  if (d->act < AX_ACT_NONE || d->act > AX_ACT_GELU) return AX_ERR_OPTION;
  if ((d->w_transposed & ~1) || (d->unaligned & ~1)) return AX_ERR_OPTION;
  if (q8 && !d->w_transposed) return AX_ERR_OPTION;
  if (gated && !q8 && d->w_transposed) return AX_ERR_OPTION;
  if (d->M < 0 || d->N < 1 || d->K < 1 || d->M > kMaxDim || d->N > kMaxDim || d->K > kMaxDim) return AX_ERR_SHAPE;
  const int e = q8 ? 1 : elem_bytes(d->dtype), oe = elem_bytes(d->out_dtype);
  if (!pitch_ok(d->x_ld, d->K, e) || !pitch_ok(d->w_ld, d->w_transposed ? d->K : d->N, e) || !pitch_ok(d->y_ld, d->N, oe)) return AX_ERR_SHAPE;
  if (q8 && d->K > 131071) return AX_ERR_K_OVERFLOW;  // 131072 * 128 * 128 = 2^31
  return AX_OK;
}
// ---- forward -----------------------------------------------------------------------------------------------------

struct Forward {
  PackJob jobs[3];
  int njobs;
  bool few;  // launch_few, on the operands themselves
  int dtype;
  GemmArgs g;
  GemmPlan plan;
  FewPlan few_plan;
  void* part;
  size_t bytes;
};

// Whether a product of M rows is worth launch_few, which reads the weights once and as they lie, against tiles with slices
// of the contraction and the launch that adds them.  A rule on the sizes alone: a view gives the bits of its copy.  Times in us
// at rows / K / N, weights from memory, few : tiles.
//   float32 (no copies in pieces)       1/4096/4096 20 : 71      32/2048/2048 11 : 25     32/8192/8192 78 : 224
//                                       64/2048/2048 14 : 25     64/8192/8192 132 : 231   96/512/8192 gated 39 : 32
//       [N, K]                          64/2048/2048 16 : 26     64/8192/8192 200 : 261   96/2048/2048 31 : 26
//       [N, K], rows off 16 bytes       32/4097/4097 53 : 57     64/4097/4097 95 : 57
//   weights [N, K]                      1/4096/4096 9.6 : 17.8   24/4096/4096 14.7 : 14.9 int8 32/4096/4096 9.0 : 12.8
//   bf16 [K, N], rows of one workgroup far apart: short contractions, small weights
//                                       1/2048/2048 6.6 : 9.9    32/2048/8192 12.7 : 13.7
//                                       8/4096/4096 13.8 : 14.9  16/4096/4096 14.7 : 13.7 1/4096/12288 31 : 25
//                                       16/4096/2048 11.1 : 11.8 32/4096/1024 11.7 : 11.0 8/8192/2048 15.0 : 14.5
//       gated                           16/4096/4096 22.6 : 24.4 32/4096/4096 23.9 : 20.8 32/4096/2048 14.3 : 14.8
//     or rows that tiles would have laid out anew
//                                       16/4097/4097 21 : 28     32/8191/1001 29 : 22     gated 32/8191/1001 25 : 29
//   int8 gated, where one launch of tiles has enough of them, of rows that are read in place
//                                       1/4096/4096 7.8 : 14.7   16/2048/6000 8.9 : 9.0   17/4096/10240 23.3 : 17.3
bool few_fits(int dtype, bool along, bool gated, long long M, long long N, long long K) {
  if (M > (dtype == AX_F32 ? 64 : 32) || N > 1 << 20) return false;
  if (dtype == AX_F32) return M <= 32 || !along || K % 4 == 0;
  if (dtype == kI8 && gated) return K % 16 != 0 || (N <= 8192 && M * N <= 98304);
  if (along || K <= 2048 || (N % 8 != 0 && (gated || M <= 16))) return true;
  const int m = (int)M / (gated ? 2 : 1);
  return K * N <= (m <= 8 ? 1 << 24 : m <= 16 ? 1 << 23 : 0);
}

// x [M, K] times w as it lies.
GemmArgs few_args(const ax_matmul_desc_t* d, bool q8, const void* x, const void* w, const void* w2) {
  GemmArgs g{};
  const int esz = q8 ? 1 : elem_bytes(d->dtype);
  g.seg[g.nseg++] = GemmSeg{x, w, w2};
  g.i8 = q8;
  g.lb = d->w_transposed ? 0 : 1;
  g.M = (int)d->M;
  g.N = (int)d->N;
  g.K = (int)d->K;
  g.lda = d->x_ld * esz;
  g.ldb = d->w_ld * esz;
  g.odt = d->out_dtype;
  g.act = d->act;
  g.ldy = d->y_ld;
  return g;
}

Forward make_forward(const ax_matmul_desc_t* d, bool q8, bool gated, const void* x, const void* w, const void* w2, void* ws) {
  Forward f{};
  Arena ar(ws);
  const int dt = q8 ? kI8 : d->dtype;
  const long long wr = d->w_transposed ? d->N : d->K, wc = d->w_transposed ? d->K : d->N;
  f.dtype = dt;
  f.few = few_fits(dt, d->w_transposed, gated, d->M, d->N, d->K);
  if (f.few) {
    f.g = few_args(d, q8, x, w, w2);
    f.g.gated = gated;
    f.g.ldr = d->residual_ld;
    f.few_plan = plan_few(f.g, dt);
    f.part = ar.take(f.few_plan.part_bytes);
    f.bytes = ar.used;
    return f;
  }
  const Operand a = make_operand(x, d->M, d->K, d->x_ld, dt, d->unaligned, ar, &f.jobs[0]);
  const Operand b = make_operand(w, wr, wc, d->w_ld, dt, d->unaligned, ar, &f.jobs[1]);
  Operand b2{};
  f.njobs = 2;
  if (gated) b2 = make_operand(w2, wr, wc, d->w_ld, dt, d->unaligned, ar, &f.jobs[f.njobs++]);
  GemmArgs& g = f.g;
  add_segment(&g, a, b, gated ? &b2 : nullptr);
  g.i8 = q8;
  g.la = 0;
  g.lb = d->w_transposed ? 0 : 1;
  g.M = (int)d->M;
  g.N = (int)d->N;
  // contraction: whole chunks where both operands have them contiguous (zeros behind the end), rows of w otherwise
  g.K = (int)(d->w_transposed ? a.cols : d->K);
  g.gated = gated;
  g.odt = d->out_dtype;
  g.act = d->act;
  g.ldy = d->y_ld;
  g.ldr = d->residual_ld;
  f.plan = plan_gemm(g);
  f.part = ar.take(f.plan.part_bytes);
  f.bytes = ar.used;
  return f;
}

int run_forward(Forward& f, hipStream_t s) {
  if (f.few) return launch_few(f.g, f.dtype, f.few_plan, f.part, s) == hipSuccess ? AX_OK : AX_ERR_HIP;
  const bool all[3] = {true, true, true};
  PackBatch copies{};
  const int copy_blocks = fill_pack(&copies, f.jobs, all, f.njobs);
  if (run_pack(copies, copy_blocks, s) != hipSuccess) return AX_ERR_HIP;
  return launch_gemm(f.g, f.plan, f.part, s) == hipSuccess ? AX_OK : AX_ERR_HIP;
}

// ---- backward ----------------------------------------------------------------------------------------------------

struct Backward {
  PackJob jobs[3];  // x, w, wu
  GradArgs ga;
  bool elementwise;  // act_grad_kernel runs for the products (it runs for gb alone too)
  int row_blocks;
  float* part;       // of gb
  bool few;          // gx by launch_few
  GemmArgs gx, gw;
  GemmPlan px, pw;
  FewPlan pf;
  void *partx, *partw;
  size_t bytes;
};

Backward make_backward(const ax_matmul_desc_t* d, bool gated, const void* gy, const void* x, const void* w, const void* w2,
                       const void* z, const void* u, void* ws) {
  Backward b{};
  Arena ar(ws);
  const int dt = d->dtype;
  const long long wr = d->w_transposed ? d->N : d->K, wc = d->w_transposed ? d->K : d->N;
  const Operand ox = make_operand(x, d->M, d->K, d->x_ld, dt, d->unaligned, ar, &b.jobs[0]);
  b.few = dt == AX_BF16 && few_fits(dt, !d->w_transposed, false, d->M, d->K, d->N);
  Operand ow{}, ow2{};
  if (!b.few) {
    ow = make_operand(w, wr, wc, d->w_ld, dt, d->unaligned, ar, &b.jobs[1]);
    if (gated) ow2 = make_operand(w2, wr, wc, d->w_ld, dt, d->unaligned, ar, &b.jobs[2]);
  }
  // gz as an operand: gy itself where nothing is multiplied to it and it can be read in place
  PackJob unused;
  Operand oz{}, ou{};
  const bool plain = !gated && d->act == AX_ACT_NONE;
  const bool in_place = plain && dt == AX_BF16 && !d->unaligned && d->N % 8 == 0 && d->y_ld % 8 == 0;
  const long long pcols = (d->N + 7) / 8 * 8;
  if (in_place) {
    oz = make_operand(gy, d->M, d->N, d->y_ld, dt, false, ar, &unused);
  } else {  // (unaligned: a buffer of its own)
    oz = make_operand(gy, d->M, d->N, d->y_ld, dt, true, ar, &unused);
    b.ga.gz = unused.dst;
    if (gated) {
      ou = make_operand(gy, d->M, d->N, d->y_ld, dt, true, ar, &unused);
      b.ga.gu = unused.dst;
    }
  }
  b.elementwise = !in_place;
  b.ga.gy = gy;
  b.ga.z = plain ? nullptr : z;
  b.ga.u = u;
  b.ga.ldy = d->y_ld;
  b.ga.pcols = pcols;
  b.ga.pitch = oz.ld / 2;
  b.ga.M = (int)d->M;
  b.ga.N = (int)d->N;
  b.ga.act = d->act;
  b.ga.rows_per = rows_per_block((int)d->M, (int)d->N);
  b.row_blocks = (int)((d->M + b.ga.rows_per - 1) / b.ga.rows_per);
  b.ga.wide = (int)((pcols + 255) / 256);
  b.ga.blocks = b.ga.wide * b.row_blocks;
  if (!gated) b.part = (float*)ar.take((size_t)b.row_blocks * d->N * 4);

  GemmArgs& gx = b.gx;  // gx [M, K] = gz [M, N] w^T
  if (b.few) {
    gx.seg[gx.nseg++] = GemmSeg{oz.p, w, nullptr};
    if (gated) gx.seg[gx.nseg++] = GemmSeg{ou.p, w2, nullptr};
  } else {
    add_segment(&gx, oz, ow, nullptr);
    if (gated) add_segment(&gx, ou, ow2, nullptr);
  }
  gx.la = 0;
  gx.lb = d->w_transposed ? 1 : 0;
  gx.M = (int)d->M;
  gx.N = (int)d->K;
  gx.K = (int)(d->w_transposed || b.few ? d->N : pcols);
  if (b.few) {
    gx.lda = oz.ld;
    gx.ldb = d->w_ld * 2;
  }
  gx.odt = dt;
  gx.ldy = d->x_ld;
  if (b.few) b.pf = plan_few(gx, dt);
  else b.px = plan_gemm(gx);

  GemmArgs& gw = b.gw;  // gw [K, N] = x^T gz, or [N, K] = gz^T x
  if (d->w_transposed) add_segment(&gw, oz, ox, nullptr);
  else add_segment(&gw, ox, oz, gated ? &ou : nullptr);
  gw.la = gw.lb = 1;
  gw.M = (int)(d->w_transposed ? d->N : d->K);
  gw.N = (int)(d->w_transposed ? d->K : d->N);
  gw.K = (int)d->M;
  gw.dual = gated;
  gw.odt = dt;
  gw.ldy = d->w_ld;
  if (d->M > 0) b.pw = plan_gemm(gw);
  // one after the other on one stream: the partial sums may share their place
  b.partx = b.partw = ar.take(std::max({b.px.part_bytes, b.pf.part_bytes, b.pw.part_bytes}));
  b.bytes = ar.used;
  return b;
}

template <bool GATED>
void run_act_grad(const GradArgs& a, const PackBatch& copies, int grid, int dtype, hipStream_t s) {
  if (dtype == AX_F32) act_grad_kernel<AX_F32, GATED><<<grid, 256, 0, s>>>(a, copies);
  else act_grad_kernel<AX_BF16, GATED><<<grid, 256, 0, s>>>(a, copies);
}

}  // namespace

hipError_t launch_act_grad(const GradArgs& a, bool gated, const PackBatch& copies, int copy_blocks, int dtype, hipStream_t s) {
  const int grid = a.blocks + copy_blocks;
  gated ? run_act_grad<true>(a, copies, grid, dtype, s) : run_act_grad<false>(a, copies, grid, dtype, s);
  return hipGetLastError();
}

namespace {

struct FewBackward {
  OuterArgs o;
  GemmArgs gx;
  FewPlan plan;
  void* part;
  size_t bytes;
};

// Whether the gradients are those of few rows.  Times in us of all three at rows / K / N, few : tiles.
//   float32    8/2048/2048 22 : 39   16/97/2920 20 : 25       32/2048/2048 36 : 39   20/512/8192 28 : 49   32/97/2920 31 : 26
//   bf16       8/2048/1000 12 : 14   16/2048/2048 17.5 : 18.3 16/2048/1000 16.4 : 14.5                     32/4096/4096 53 : 39
bool few_backward_fits(const ax_matmul_desc_t* d) {
  if (d->K > 1 << 20 || d->N > 1 << 20 || !few_fits(d->dtype, !d->w_transposed, false, d->M, d->K, d->N)) return false;
  if (d->dtype == AX_F32) return d->M <= (d->K * d->N >= 1 << 20 ? 32 : 16);
  return d->M <= (d->K * d->N >= 1 << 22 ? 16 : 12);
}

FewBackward make_few_backward(const ax_matmul_desc_t* d, bool gated, const void* gy, const void* x, const void* w,
                              const void* w2, const void* z, const void* u, void* ws) {
  FewBackward b{};
  Arena ar(ws);
  const int esz = elem_bytes(d->dtype);
  const bool plain = !gated && d->act == AX_ACT_NONE;
  OuterArgs& o = b.o;
  o.x = x;
  o.gy = gy;
  o.z = plain ? nullptr : z;
  o.u = u;
  o.x_ld = d->x_ld;
  o.gy_ld = d->y_ld;
  o.gw_ld = d->w_ld;
  o.M = (int)d->M;
  o.N = (int)d->N;
  o.K = (int)d->K;
  o.act = d->act;
  o.transposed = d->w_transposed;
  if (!plain) o.gz[0] = ar.take((size_t)d->M * d->N * esz);
  if (gated) o.gz[1] = ar.take((size_t)d->M * d->N * esz);
  GemmArgs& gx = b.gx;
  gx.seg[gx.nseg++] = GemmSeg{plain ? gy : o.gz[0], w, nullptr};
  if (gated) gx.seg[gx.nseg++] = GemmSeg{o.gz[1], w2, nullptr};
  gx.lb = d->w_transposed ? 1 : 0;
  gx.M = (int)d->M;
  gx.N = (int)d->K;
  gx.K = (int)d->N;
  gx.lda = (plain ? d->y_ld : d->N) * esz;
  gx.ldb = d->w_ld * esz;
  gx.odt = d->dtype;
  gx.ldy = d->x_ld;
  b.plan = plan_few(gx, d->dtype);
  b.part = ar.take(b.plan.part_bytes);
  b.bytes = ar.used;
  return b;
}

template <int DT, bool GATED>
void run_outer(const OuterArgs& o, dim3 grid, hipStream_t s) {
  if constexpr (DT == AX_F32) {  // (bf16 does not come with more rows)
    if (o.M > 16) {
      outer_kernel<DT, GATED, 32><<<grid, 256, 0, s>>>(o);
      return;
    }
  }
  outer_kernel<DT, GATED, 16><<<grid, 256, 0, s>>>(o);
}

int run_few_backward(FewBackward& b, int dtype, bool gated, void* gx_out, void* gw_out, void* gw2_out, float* gb_out, hipStream_t s) {
  OuterArgs& o = b.o;
  o.gw[0] = gw_out;
  o.gw[1] = gw2_out;
  o.gb = gb_out;
  if (!gx_out) o.gz[0] = o.gz[1] = nullptr;
  if (gw_out || gb_out || o.gz[0]) {
    // without the weight's gradient, one piece of the other factor
    const int nr = o.transposed ? o.N : o.K, nc = o.transposed ? o.K : o.N;
    const dim3 grid(gw_out || !o.transposed ? (nc + 511) / 512 : 1, gw_out || o.transposed ? (nr + 31) / 32 : 1, gated ? 2 : 1);
    if (dtype == AX_F32) gated ? run_outer<AX_F32, true>(o, grid, s) : run_outer<AX_F32, false>(o, grid, s);
    else gated ? run_outer<AX_BF16, true>(o, grid, s) : run_outer<AX_BF16, false>(o, grid, s);
    if (hipGetLastError() != hipSuccess) return AX_ERR_HIP;
  }
  if (gx_out) {
    b.gx.y = gx_out;
    if (launch_few(b.gx, dtype, b.plan, b.part, s) != hipSuccess) return AX_ERR_HIP;
  }
  return AX_OK;
}

}  // namespace

hipError_t zero_rows(void* p, long long rows, long long cols, long long ld, int esz, hipStream_t s) {
  zero_rows_kernel<<<grid_for(rows * cols * esz / 2), 256, 0, s>>>((uint8_t*)p, rows, cols * esz, ld * esz);
  return hipGetLastError();
}

namespace {

int backward_common(const ax_matmul_desc_t* d, bool gated, const void* gy, const void* x, const void* w, const void* w2,
                    const void* z, const void* u, void* gx_out, void* gw_out, void* gw2_out, float* gb_out, void* ws,
                    size_t ws_bytes, hipStream_t s) {
  const int esz = elem_bytes(d->dtype);
  const long long wr = d->w_transposed ? d->N : d->K, wc = d->w_transposed ? d->K : d->N;
  if (d->M == 0) {
    hipError_t rc = hipSuccess;
    for (void* p : {gw_out, gw2_out})
      if (p && rc == hipSuccess) rc = zero_rows(p, wr, wc, d->w_ld, esz, s);
    if (gb_out && rc == hipSuccess) rc = zero_rows(gb_out, 1, d->N, d->N, 4, s);
    return rc == hipSuccess ? AX_OK : AX_ERR_HIP;
  }
  if (few_backward_fits(d)) {
    FewBackward b = make_few_backward(d, gated, gy, x, w, w2, z, u, ws);
    if (!ws_ok(ws, ws_bytes, b.bytes)) return AX_ERR_WORKSPACE;
    return run_few_backward(b, d->dtype, gated, gx_out, gw_out, gw2_out, gb_out, s);
  }
  Backward b = make_backward(d, gated, gy, x, w, w2, z, u, ws);
  if (!ws_ok(ws, ws_bytes, b.bytes)) return AX_ERR_WORKSPACE;
  const bool products = gx_out || gw_out;
  const bool weights = gx_out && !b.few;
  const bool wanted[3] = {gw_out != nullptr, weights, weights && gated};
  PackBatch copies{};
  const int copy_blocks = fill_pack(&copies, b.jobs, wanted, 3);
  if (gated) {
    if (launch_act_grad(b.ga, true, copies, copy_blocks, d->dtype, s) != hipSuccess) return AX_ERR_HIP;
  } else if ((b.elementwise && products) || gb_out) {
    if (!products) b.ga.gz = nullptr;
    b.ga.part = gb_out ? b.part : nullptr;
    if (launch_act_grad(b.ga, false, copies, copy_blocks, d->dtype, s) != hipSuccess) return AX_ERR_HIP;
    if (gb_out) {
      if (launch_column_sum(b.part, b.row_blocks, (int)d->N, gb_out, s) != hipSuccess) return AX_ERR_HIP;
    }
  } else if (run_pack(copies, copy_blocks, s) != hipSuccess) {
    return AX_ERR_HIP;
  }
  if (gx_out) {
    b.gx.y = gx_out;
    if ((b.few ? launch_few(b.gx, AX_BF16, b.pf, b.partx, s) : launch_gemm(b.gx, b.px, b.partx, s)) != hipSuccess) return AX_ERR_HIP;
  }
  if (gw_out) {
    b.gw.y = gw_out;
    b.gw.y2 = gw2_out;
    if (launch_gemm(b.gw, b.pw, b.partw, s) != hipSuccess) return AX_ERR_HIP;
  }
  return AX_OK;
}

}  // namespace
}  // namespace ax

using namespace ax;

extern "C" size_t ax_matmul_workspace_bytes(const ax_matmul_desc_t* d) {
  if (check_desc(d, false, false, false) != AX_OK || d->M == 0) return 0;
  return make_forward(d, false, false, nullptr, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_matmul(const ax_matmul_desc_t* d, const void* x, const void* w, const void* bias, const void* residual,
                         void* y_out, void* z_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_desc(d, false, false, false)) return rc;
  if (residual && !pitch_ok(d->residual_ld, d->N, elem_bytes(d->out_dtype))) return AX_ERR_SHAPE;
  if (d->M == 0) return AX_OK;
  if (!x || !w || !y_out) return AX_ERR_NULL;
  const int e = elem_bytes(d->dtype), oe = elem_bytes(d->out_dtype);
  if (!operand_aligned(x, e, d->unaligned, d->K, d->x_ld, d->dtype) ||
      !operand_aligned(w, e, d->unaligned, d->w_transposed ? d->K : d->N, d->w_ld, d->dtype))
    return AX_ERR_ALIGN;
  for (const void* p : {bias, residual, (const void*)y_out, (const void*)z_out})
    if (!aligned_to(p, oe)) return AX_ERR_ALIGN;
  Forward f = make_forward(d, false, false, x, w, nullptr, workspace);
  if (!ws_ok(workspace, workspace_bytes, f.bytes)) return AX_ERR_WORKSPACE;
  f.g.y = y_out;
  f.g.z = z_out;
  f.g.bias = bias;
  f.g.res = residual;
  return run_forward(f, (hipStream_t)hip_stream);
}

extern "C" size_t ax_matmul_q8_workspace_bytes(const ax_matmul_desc_t* d) {
  if (check_desc(d, true, false, false) != AX_OK || d->M == 0) return 0;
  return make_forward(d, true, false, nullptr, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_matmul_q8(const ax_matmul_desc_t* d, const int8_t* x, const float* x_scales, const int8_t* w,
                            const float* w_scales, const void* bias, const void* residual, void* y_out, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_desc(d, true, false, false)) return rc;
  if (residual && !pitch_ok(d->residual_ld, d->N, elem_bytes(d->out_dtype))) return AX_ERR_SHAPE;
  if (d->M == 0) return AX_OK;
  if (!x || !x_scales || !w || !w_scales || !y_out) return AX_ERR_NULL;
  const int oe = elem_bytes(d->out_dtype);
  if (!operand_aligned(x, 1, d->unaligned, d->K, d->x_ld, kI8) || !operand_aligned(w, 1, d->unaligned, d->K, d->w_ld, kI8) ||
      !aligned_to(x_scales, 4) || !aligned_to(w_scales, 4))
    return AX_ERR_ALIGN;
  for (const void* p : {bias, residual, (const void*)y_out})
    if (!aligned_to(p, oe)) return AX_ERR_ALIGN;
  Forward f = make_forward(d, true, false, x, w, nullptr, workspace);
  if (!ws_ok(workspace, workspace_bytes, f.bytes)) return AX_ERR_WORKSPACE;
  f.g.y = y_out;
  f.g.bias = bias;
  f.g.res = residual;
  f.g.xs = x_scales;
  f.g.ws = w_scales;
  return run_forward(f, (hipStream_t)hip_stream);
}

extern "C" size_t ax_matmul_backward_workspace_bytes(const ax_matmul_desc_t* d) {
  if (check_desc(d, false, true, false) != AX_OK || d->M == 0) return 0;
  if (few_backward_fits(d)) return make_few_backward(d, false, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr).bytes;
  return make_backward(d, false, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_matmul_backward(const ax_matmul_desc_t* d, const void* gy, const void* x, const void* w, const void* z,
                                  void* gx_out, void* gw_out, float* gb_out, void* workspace, size_t workspace_bytes,
                                  void* hip_stream) {
  if (int rc = check_desc(d, false, true, false)) return rc;
  if (d->M > 0 && !gx_out && !gw_out && !gb_out) return AX_ERR_NULL;  // (a gradient of no rows may be NULL)
  if (d->M > 0 && (!gy || (gw_out && !x) || (gx_out && !w) || (d->act != AX_ACT_NONE && !z))) return AX_ERR_NULL;
  const int e = elem_bytes(d->dtype);
  if (!operand_aligned(x, e, d->unaligned, d->K, d->x_ld, d->dtype) ||
      !operand_aligned(w, e, d->unaligned, d->w_transposed ? d->K : d->N, d->w_ld, d->dtype) ||
      !operand_aligned(gy, e, d->unaligned || d->act != AX_ACT_NONE, d->N, d->y_ld, d->dtype))
    return AX_ERR_ALIGN;
  for (const void* p : {z, (const void*)gx_out, (const void*)gw_out})
    if (!aligned_to(p, e)) return AX_ERR_ALIGN;
  if (!aligned_to(gb_out, 4)) return AX_ERR_ALIGN;
  return backward_common(d, false, gy, x, w, nullptr, z, nullptr, gx_out, gw_out, nullptr, gb_out, workspace, workspace_bytes,
                         (hipStream_t)hip_stream);
}

extern "C" size_t ax_gated_workspace_bytes(const ax_matmul_desc_t* d) {
  if (check_desc(d, false, false, true) != AX_OK || d->M == 0) return 0;
  return make_forward(d, false, true, nullptr, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_gated(const ax_matmul_desc_t* d, const void* x, const void* wg, const void* wu, void* h_out, void* g_out,
                        void* u_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_desc(d, false, false, true)) return rc;
  if (!g_out != !u_out) return AX_ERR_NULL;
  if (d->M == 0) return AX_OK;
  if (!x || !wg || !wu || !h_out) return AX_ERR_NULL;
  const int e = elem_bytes(d->dtype), oe = elem_bytes(d->out_dtype);
  if (!operand_aligned(x, e, d->unaligned, d->K, d->x_ld, d->dtype)) return AX_ERR_ALIGN;
  for (const void* p : {wg, wu})
    if (!operand_aligned(p, e, d->unaligned, d->N, d->w_ld, d->dtype)) return AX_ERR_ALIGN;
  for (const void* p : {(const void*)h_out, (const void*)g_out, (const void*)u_out})
    if (!aligned_to(p, oe)) return AX_ERR_ALIGN;
  Forward f = make_forward(d, false, true, x, wg, wu, workspace);
  if (!ws_ok(workspace, workspace_bytes, f.bytes)) return AX_ERR_WORKSPACE;
  f.g.y = h_out;
  f.g.z = g_out;
  f.g.z2 = u_out;
  return run_forward(f, (hipStream_t)hip_stream);
}

extern "C" size_t ax_gated_q8_workspace_bytes(const ax_matmul_desc_t* d) {
  if (check_desc(d, true, false, true) != AX_OK || d->M == 0) return 0;
  return make_forward(d, true, true, nullptr, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_gated_q8(const ax_matmul_desc_t* d, const int8_t* x, const float* x_scales, const int8_t* wg,
                           const float* wg_scales, const int8_t* wu, const float* wu_scales, void* h_out, void* workspace,
                           size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_desc(d, true, false, true)) return rc;
  if (d->M == 0) return AX_OK;
  if (!x || !x_scales || !wg || !wg_scales || !wu || !wu_scales || !h_out) return AX_ERR_NULL;
  if (!operand_aligned(x, 1, d->unaligned, d->K, d->x_ld, kI8) || !aligned_to(x_scales, 4) || !aligned_to(wg_scales, 4) ||
      !aligned_to(wu_scales, 4) || !aligned_to(h_out, elem_bytes(d->out_dtype)))
    return AX_ERR_ALIGN;
  for (const void* p : {(const void*)wg, (const void*)wu})
    if (!operand_aligned(p, 1, d->unaligned, d->K, d->w_ld, kI8)) return AX_ERR_ALIGN;
  Forward f = make_forward(d, true, true, x, wg, wu, workspace);
  if (!ws_ok(workspace, workspace_bytes, f.bytes)) return AX_ERR_WORKSPACE;
  f.g.y = h_out;
  f.g.xs = x_scales;
  f.g.ws = wg_scales;
  f.g.ws2 = wu_scales;
  return run_forward(f, (hipStream_t)hip_stream);
}

extern "C" size_t ax_gated_backward_workspace_bytes(const ax_matmul_desc_t* d) {
  if (check_desc(d, false, true, true) != AX_OK || d->M == 0) return 0;
  if (few_backward_fits(d)) return make_few_backward(d, true, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr).bytes;
  return make_backward(d, true, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_gated_backward(const ax_matmul_desc_t* d, const void* gh, const void* x, const void* wg, const void* wu,
                                 const void* g, const void* u, void* gx_out, void* gwg_out, void* gwu_out, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_desc(d, false, true, true)) return rc;
  if ((!gwg_out != !gwu_out) || (d->M > 0 && !gx_out && !gwg_out)) return AX_ERR_NULL;
  if (d->M > 0 && (!gh || !g || !u || (gwg_out && !x) || (gx_out && (!wg || !wu)))) return AX_ERR_NULL;
  const int e = elem_bytes(d->dtype);
  if (!operand_aligned(x, e, d->unaligned, d->K, d->x_ld, d->dtype)) return AX_ERR_ALIGN;
  for (const void* p : {wg, wu})
    if (!operand_aligned(p, e, d->unaligned, d->N, d->w_ld, d->dtype)) return AX_ERR_ALIGN;
  for (const void* p : {gh, g, u, (const void*)gx_out, (const void*)gwg_out, (const void*)gwu_out})
    if (!aligned_to(p, e)) return AX_ERR_ALIGN;
  return backward_common(d, true, gh, x, wg, wu, g, u, gx_out, gwg_out, gwu_out, nullptr, workspace, workspace_bytes,
                         (hipStream_t)hip_stream);
}

extern "C" int ax_probe_product_plan(const ax_matmul_desc_t* d, int product, int* kernel, int* rows, int* cols, int* slices) {
  if (product < AX_PRODUCT_MATMUL || product > AX_PRODUCT_GATED_GW) return AX_ERR_OPTION;
  const bool q8 = product == AX_PRODUCT_MATMUL_Q8 || product == AX_PRODUCT_GATED_Q8, back = product >= AX_PRODUCT_MATMUL_GX;
  const bool gated = product == AX_PRODUCT_GATED || product == AX_PRODUCT_GATED_Q8 || product >= AX_PRODUCT_GATED_GX;
  if (int rc = check_desc(d, q8, back, gated)) return rc;
  int k = 0, r = 0, c = 0, n = 1;
  if (d->M > 0 && !back) {
    const Forward f = make_forward(d, q8, gated, nullptr, nullptr, nullptr, nullptr);
    k = f.few;
    n = f.few ? f.few_plan.slices : f.plan.splits;
    if (!f.few) tile_of(f.g, f.plan, &r, &c);
  } else if (d->M > 0) {
    const bool gx = product == AX_PRODUCT_MATMUL_GX || product == AX_PRODUCT_GATED_GX;
    if (few_backward_fits(d)) {
      k = gx ? 1 : 2;
      if (gx) n = make_few_backward(d, gated, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr).plan.slices;
    } else {
      const Backward b = make_backward(d, gated, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr);
      k = gx && b.few;
      n = k ? b.pf.slices : gx ? b.px.splits : b.pw.splits;
      if (!k) gx ? tile_of(b.gx, b.px, &r, &c) : tile_of(b.gw, b.pw, &r, &c);
    }
  }
  if (kernel) *kernel = k;
  if (rows) *rows = r;
  if (cols) *cols = c;
  if (slices) *slices = n;
  return AX_OK;
}
