// Root-mean-square norm of rows with the residual's addition, its output in 8-bit codes, and its gradients.
//
//   t = x + residual,  rstd = 1 / sqrt(mean t^2 + eps),  y = t rstd w
//   codes = round(t w * (127 / max |t w|)),  scale = max |t w| * rstd / 127
//   gx = rstd (gy w - h mean(gy w h)) + gsum,  gw = sum over rows of gy h,  h = t rstd
//
// All kernels are bound by memory.  One pass: a row's values stay in registers between the reduction and the output
// (rows of up to 32768 columns; longer ones are read twice, the second time mostly from the caches).  Few rows get more
// lanes each, since their time is the latency of one row.
//
// Measured: codes, sum and values of 8192 x 4096 bf16 with a residual 75.7 us, 369 MB, 4.9 TB/s (a copy reaches 5.1);
// gradients of 6007 x 1000 float32 with gsum 21 us, 96 MB, 4.6 TB/s, and 4 for the workgroups' sums of gw, which a
// second launch adds so that their order is fixed; one row of 2048: 3.5 us, a launch and two trips to memory.
//
// Codes are reproducible bit for bit: t, t w, the division and the product in front of the rounding are single float32
// operations, the maximum is exact, and rstd, the only quantity that depends on the order of a sum, is in the scale alone.
#include <algorithm>
#include <cmath>

#include "ax_float.h"
#include "ax_internal.h"
#include "ax_norm.h"

#pragma clang fp contract(off)

namespace ax {
namespace {

enum Mode { kValues, kCodes };

struct NormArgs {
  const void* x;
  const void* res;  // may be null
  const void* w;    // may be null (codes)
  void* sum;        // may be null
  void* y;
  int8_t* codes;
  float* scales;
  float* values;  // may be null
  float* rstd;    // may be null
  long long rows, row0;  // row0: first of this launch
  long long x_ld, r_ld, s_ld, y_ld;
  int cols, w_f32, normalize;
  float eps;
};

// Eight consecutive elements of a row a lane and pass.
template <int TPR, bool F32>
__device__ __forceinline__ void load_row(const void* p, long long row, int it, int t, int cols, float (&v)[8]) {
  const int c = (it * TPR + t) * 8;
  load_elems<F32, 8>(p, row + c, cols - c, v);
}
template <int TPR, bool F32>
__device__ __forceinline__ void store_row(void* p, long long row, int it, int t, int cols, const float (&v)[8]) {
  const int c = (it * TPR + t) * 8;
  store_elems<F32, 8>(p, row + c, cols - c, v);
}

// Sum and largest value over the TPR lanes of a row, in a fixed order.  red: 2 * TPR / 64 words of LDS.
template <int TPR>
__device__ __forceinline__ void reduce_row(float& sum, uint32_t& top, float* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    sum += __shfl_xor(sum, off, 64);
    top = max(top, (uint32_t)__shfl_xor((int)top, off, 64));
  }
  if (TPR == 64) return;
  constexpr int W = TPR / 64;
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    red[wave] = sum;
    red[W + wave] = __uint_as_float(top);
  }
  __syncthreads();
  sum = 0.f;
  top = 0;
  for (int i = 0; i < W; ++i) {
    sum += red[i];
    top = max(top, __float_as_uint(red[W + i]));
  }
}

// TPR lanes a row, NV passes of eight elements in registers (0: any number of columns, read twice).
template <int MODE, bool F32, int TPR, int NV>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_kernel(const NormArgs a) {
  constexpr int THREADS = TPR < 256 ? 256 : TPR;
  __shared__ float red[2 * (TPR / 64)];
  const int t = threadIdx.x % TPR;
  const long long row = a.row0 + (long long)blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR;
  if (row >= a.rows) return;  // uniform over a row's lanes (and over the workgroup where it has one row)
  const long long xo = row * a.x_ld, ro = row * a.r_ld, so = row * a.s_ld, yo = row * a.y_ld, co = row * (long long)a.cols;
  const int iters = NV ? NV : (a.cols + TPR * 8 - 1) / (TPR * 8);
  float v[NV ? NV : 1][8], w[NV ? NV : 1][8];

  auto load = [&](int it, float (&tv)[8], float (&wv)[8]) {
    load_row<TPR, F32>(a.x, xo, it, t, a.cols, tv);
    if (a.res) {
      float r[8];
      load_row<TPR, F32>(a.res, ro, it, t, a.cols, r);
      for (int e = 0; e < 8; ++e) tv[e] += r[e];
    }
    if (a.w) {
      if (a.w_f32) load_row<TPR, true>(a.w, 0, it, t, a.cols, wv);
      else load_row<TPR, false>(a.w, 0, it, t, a.cols, wv);
    } else {
      for (int e = 0; e < 8; ++e) wv[e] = 1.f;
    }
  };
  float ss = 0.f;
  uint32_t top = 0;  // bit pattern of the largest |t w|: as integers, NaN is above infinity and both above all numbers
  auto take = [&](int it, float (&tv)[8], float (&wv)[8]) {
    for (int e = 0; e < 8; ++e) {
      ss = __builtin_fmaf(tv[e], tv[e], ss);
      if (MODE == kCodes) {
        tv[e] = tv[e] * wv[e];
        top = max(top, __float_as_uint(tv[e]) & 0x7fffffffu);
      }
    }
  };
  if (NV) {
#pragma unroll
    for (int it = 0; it < iters; ++it) load(it, v[it], w[it]);
#pragma unroll
    for (int it = 0; it < iters; ++it) {
      if (a.sum) store_row<TPR, F32>(a.sum, so, it, t, a.cols, v[it]);
      take(it, v[it], w[it]);
    }
  } else {
    for (int it = 0; it < iters; ++it) {
      load(it, v[0], w[0]);
      take(it, v[0], w[0]);
    }
  }
  reduce_row<TPR>(ss, top, red);
  const float rstd = a.normalize ? 1.f / sqrtf(ss / (float)a.cols + a.eps) : 1.f;
  const float amax = __uint_as_float(top);
  const float inv = amax >= 0x1p-120f && top < 0x7f800000u ? 127.f / amax : 0.f;
  const float scale = top ? amax * rstd / 127.f : 0.f;  // (rstd may be infinite)
  if (t == 0) {
    if (a.rstd) a.rstd[row] = rstd;
    if (MODE == kCodes) a.scales[row] = scale;
  }
  auto put = [&](int it, const float (&tv)[8], const float (&wv)[8]) {
    if (MODE == kValues) {
      float y[8];
      for (int e = 0; e < 8; ++e) y[e] = tv[e] * rstd * wv[e];
      store_row<TPR, F32>(a.y, yo, it, t, a.cols, y);
    } else {
      float c[8];
      for (int e = 0; e < 8; ++e) c[e] = inv > 0.f ? rintf(tv[e] * inv) : 0.f;
      const int col = (it * TPR + t) * 8;
      if (col + 8 <= a.cols) {
        u32x2 q = {0, 0};
        for (int e = 0; e < 8; ++e) q[e >> 2] |= ((uint32_t)(int)c[e] & 0xffu) << (8 * (e & 3));
        store_any(a.codes + co + col, q);
      } else {
        for (int e = 0; e < 8; ++e)
          if (col + e < a.cols) a.codes[co + col + e] = (int8_t)(int)c[e];
      }
      if (a.values) {
        for (int e = 0; e < 8; ++e) c[e] *= scale;
        store_row<TPR, true>(a.values, co, it, t, a.cols, c);
      }
    }
  };
  if (NV) {
#pragma unroll
    for (int it = 0; it < iters; ++it) put(it, v[it], w[it]);
  } else {
    for (int it = 0; it < iters; ++it) {
      load(it, v[0], w[0]);
      // (sum may be x or the residual: written only now, behind this lane's last read of the place)
      if (a.sum) store_row<TPR, F32>(a.sum, so, it, t, a.cols, v[0]);
      if (MODE == kCodes)
        for (int e = 0; e < 8; ++e) v[0][e] = v[0][e] * w[0][e];
      put(it, v[0], w[0]);
    }
  }
}

struct NormGradArgs {
  const void* gy;
  const void* gsum;  // may be null
  const void* t;
  const void* w;
  const float* rstd;
  void* gx;     // may be null
  float* part;  // [workgroups][cols], may be null
  long long rows, row0;
  long long t_ld, gs_ld, gx_ld, gy_ld;
  int cols, w_f32;
};

// A workgroup takes every gridDim.x-th group of THREADS / TPR rows and keeps its share of gw in registers until the end.
template <bool F32, int TPR, int NV>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_grad_kernel(const NormGradArgs a) {
  constexpr int THREADS = TPR < 256 ? 256 : TPR, ROWS = THREADS / TPR;
  __shared__ float red[2 * 2 * (TPR / 64)];
  __shared__ float share[ROWS > 1 ? NV * 8 * THREADS : 1];
  const int t = threadIdx.x % TPR;
  float gw[NV][8], w[NV][8];
#pragma unroll
  for (int it = 0; it < NV; ++it) {
    if (a.w_f32) load_row<TPR, true>(a.w, 0, it, t, a.cols, w[it]);
    else load_row<TPR, false>(a.w, 0, it, t, a.cols, w[it]);
    for (int e = 0; e < 8; ++e) gw[it][e] = 0.f;
  }
  int turn = 0;
  for (long long base = (long long)blockIdx.x * ROWS; base < a.rows; base += (long long)gridDim.x * ROWS) {
    const long long row = base + threadIdx.x / TPR;
    if (ROWS > 1 && row >= a.rows) break;  // uniform over the wave, which has the row to itself
    const float rstd = a.rstd[row];
    float gy[NV][8], h[NV][8];
#pragma unroll
    for (int it = 0; it < NV; ++it) {
      load_row<TPR, F32>(a.gy, row * a.gy_ld, it, t, a.cols, gy[it]);
      load_row<TPR, F32>(a.t, row * a.t_ld, it, t, a.cols, h[it]);
    }
    float dot = 0.f;
#pragma unroll
    for (int it = 0; it < NV; ++it)
      for (int e = 0; e < 8; ++e) {
        h[it][e] = h[it][e] * rstd;
        gw[it][e] = __builtin_fmaf(gy[it][e], h[it][e], gw[it][e]);
        gy[it][e] = gy[it][e] * w[it][e];
        dot = __builtin_fmaf(gy[it][e], h[it][e], dot);
      }
    if (!a.gx) continue;  // uniform
    uint32_t none = 0;
    // two turns' words apart: a wave may write the next row's while another still reads this one's
    reduce_row<TPR>(dot, none, red + turn * 2 * (TPR / 64));
    turn ^= 1;
    const float mean = dot / (float)a.cols;
#pragma unroll
    for (int it = 0; it < NV; ++it) {
      float o[8];
      for (int e = 0; e < 8; ++e) o[e] = rstd * (gy[it][e] - h[it][e] * mean);
      if (a.gsum) {
        float s[8];
        load_row<TPR, F32>(a.gsum, row * a.gs_ld, it, t, a.cols, s);
        for (int e = 0; e < 8; ++e) o[e] += s[e];
      }
      store_row<TPR, F32>(a.gx, row * a.gx_ld, it, t, a.cols, o);
    }
  }
  if (!a.part) return;
  if (ROWS > 1) {  // the waves' shares, in their order
#pragma unroll
    for (int it = 0; it < NV; ++it)
      for (int e = 0; e < 8; ++e) share[(it * 8 + e) * THREADS + threadIdx.x] = gw[it][e];
    __syncthreads();
    if (threadIdx.x >= TPR) return;
#pragma unroll
    for (int it = 0; it < NV; ++it)
      for (int e = 0; e < 8; ++e)
        for (int r = 1; r < ROWS; ++r) gw[it][e] += share[(it * 8 + e) * THREADS + r * TPR + t];
  }
#pragma unroll
  for (int it = 0; it < NV; ++it) {
    store_row<TPR, true>(a.part, (long long)blockIdx.x * a.cols, it, t, a.cols, gw[it]);
  }
}

// Rows of more columns than a workgroup's registers hold: one pass for the row's mean, one for the outputs; gw from a
// kernel of its own.
template <bool F32>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(const NormGradArgs a) {
  constexpr int TPR = 1024;
  __shared__ float red[2 * (TPR / 64)];
  const int t = threadIdx.x;
  const long long row = a.row0 + blockIdx.x;
  const float rstd = a.rstd[row];
  const int iters = (a.cols + TPR * 8 - 1) / (TPR * 8);
  float dot = 0.f;
  for (int pass = 0; pass < 2; ++pass) {
    const float mean = dot / (float)a.cols;
    for (int it = 0; it < iters; ++it) {
      float gy[8], h[8], w[8];
      load_row<TPR, F32>(a.gy, row * a.gy_ld, it, t, a.cols, gy);
      load_row<TPR, F32>(a.t, row * a.t_ld, it, t, a.cols, h);
      if (a.w_f32) load_row<TPR, true>(a.w, 0, it, t, a.cols, w);
      else load_row<TPR, false>(a.w, 0, it, t, a.cols, w);
      for (int e = 0; e < 8; ++e) {
        h[e] = h[e] * rstd;
        gy[e] = gy[e] * w[e];
        if (pass == 0) dot = __builtin_fmaf(gy[e], h[e], dot);
      }
      if (pass == 1) {
        for (int e = 0; e < 8; ++e) gy[e] = rstd * (gy[e] - h[e] * mean);
        if (a.gsum) {
          load_row<TPR, F32>(a.gsum, row * a.gs_ld, it, t, a.cols, w);
          for (int e = 0; e < 8; ++e) gy[e] += w[e];
        }
        store_row<TPR, F32>(a.gx, row * a.gx_ld, it, t, a.cols, gy);
      }
    }
    if (pass == 0) {
      uint32_t none = 0;
      reduce_row<TPR>(dot, none, red);
    }
  }
}
template <bool F32>
__global__ __launch_bounds__(256) void norm_gw_long_kernel(const NormGradArgs a) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.cols) return;
  float s = 0.f;
  for (long long row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const long long g = row * a.gy_ld + c, x = row * a.t_ld + c;
    const float gy = F32 ? ((const float*)a.gy)[g] : bf16_to_f32(((const uint16_t*)a.gy)[g]);
    const float t = F32 ? ((const float*)a.t)[x] : bf16_to_f32(((const uint16_t*)a.t)[x]);
    s = __builtin_fmaf(gy, t * a.rstd[row], s);
  }
  a.part[(long long)blockIdx.y * a.cols + c] = s;
}

// out[c] = sum over the rows of part: 64 lanes a column, 16 columns a workgroup.
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* __restrict__ part, int rows, int cols, float* __restrict__ out) {
  __shared__ float red[64][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
  for (long long c0 = blockIdx.x * 16ll; c0 < cols; c0 += gridDim.x * 16ll) {
    const long long c = c0 + x;
    float s = 0.f;
    if (c < cols) {
      int r = y;
      for (; r + 64 * 7 < rows; r += 64 * 8) {  // eight loads at a time
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = part[(long long)(r + 64 * k) * cols + c];
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[k];
      }
      for (; r < rows; r += 64) s += part[(long long)r * cols + c];
    }
    red[y][x] = s;
    __syncthreads();
    for (int h = 32; h > 0; h >>= 1) {
      if (y < h) red[y][x] += red[y + h][x];
      __syncthreads();
    }
    if (y == 0 && c < cols) out[c] = red[0][x];
    __syncthreads();
  }
}

// ---- dispatch ----------------------------------------------------------------------------------------------------

// Lanes a row and passes of the forward kernels: as few lanes as hold the row in four passes (bandwidth), four times as many
// for few rows, whose time is one row's latency.  Times in us of codes of bf16 rows with a residual, at rows / columns, few
// lanes : many:  1/2048 5.0 : 3.2   1024/2048 7.8 : 6.0   4096/2048 13.4 : 14.9   16/8192 5.8 : 4.2   512/8192 9.4 : 8.7
// 1024/8192 13.5 : 16.0.  (2049 to 4096 columns would leave half of 1024 lanes idle: 512/4096 6.2 : 6.9.)
struct Shape {
  int tpr, nv;
};
Shape shape_of(long long rows, long long cols) {
  if (cols <= (rows <= 1024 ? 512 : 2048)) return {64, (int)((cols + 511) / 512)};
  if (cols <= (rows <= 512 ? 4096 : 8192)) return {256, (int)((cols + 2047) / 2048)};
  if (cols <= 32768) return {1024, (int)((cols + 8191) / 8192)};
  return {1024, 0};
}

// Of the gradient, which keeps four values a column in registers: many lanes at all row counts (float32, 64 lanes a row : 256:
// 6007/1000 21.7 : 21.4, 6007/2048 39.9 : 36.3, 1024/2048 13.0 : 12.6; 256 : 1024: 4096/8192 91 : 84).
Shape grad_shape_of(long long cols) {
  if (cols <= 512) return {64, 1};
  if (cols <= 4096) return {256, (int)((cols + 2047) / 2048)};
  if (cols <= 16384) return {1024, (int)((cols + 8191) / 8192)};
  return {1024, 0};
}

constexpr int kMaxGrid = 1 << 21;  // workgroups of a launch, which counts its threads in 32 bits

template <int MODE, bool F32>
void norm_launch(const NormArgs& all, hipStream_t s) {
  const Shape sh = shape_of(all.rows, all.cols);
  const int per = sh.tpr == 64 ? 4 : 1;
  const int threads = sh.tpr < 256 ? 256 : sh.tpr;
#define AX_NORM(T, V) norm_kernel<MODE, F32, T, V><<<grid, threads, 0, s>>>(a)
#define AX_NORM_T(T)                         \
  switch (sh.nv) {                           \
    case 1: AX_NORM(T, 1); break;            \
    case 2: AX_NORM(T, 2); break;            \
    default: AX_NORM(T, 4); break;           \
  }
  NormArgs a = all;
  for (a.row0 = 0; a.row0 < a.rows; a.row0 += (long long)kMaxGrid * per) {
    const unsigned grid = (unsigned)std::min<long long>((a.rows - a.row0 + per - 1) / per, kMaxGrid);
    if (sh.nv == 0) AX_NORM(1024, 0);
    else if (sh.tpr == 64) AX_NORM_T(64)
    else if (sh.tpr == 256) AX_NORM_T(256)
    else AX_NORM_T(1024)
  }
#undef AX_NORM_T
#undef AX_NORM
}
template <bool F32>
void norm_grad_launch(const NormGradArgs& a, const Shape& sh, int groups, hipStream_t s) {
  if (sh.tpr == 64) norm_grad_kernel<F32, 64, 1><<<groups, 256, 0, s>>>(a);
  else if (sh.tpr == 256) sh.nv == 1 ? norm_grad_kernel<F32, 256, 1><<<groups, 256, 0, s>>>(a) : norm_grad_kernel<F32, 256, 2><<<groups, 256, 0, s>>>(a);
  else sh.nv == 1 ? norm_grad_kernel<F32, 1024, 1><<<groups, 1024, 0, s>>>(a) : norm_grad_kernel<F32, 1024, 2><<<groups, 1024, 0, s>>>(a);
}

// Workgroups of the gradient, each with a row of sums to be added afterwards: four rows each (us with one, two, four and eight,
// 1024/2048: 16.1, 11.9, 12.3, 14.3; 512/8192: 24.1, 18.1, 17.4, 17.2), and no fewer than 128 while there are rows.
int grad_groups(long long rows, long long cols) {
  const Shape sh = grad_shape_of(cols);
  if (sh.nv == 0) return (int)std::min<long long>(rows, 64);
  const long long most = sh.tpr == 1024 ? 512 : 1024;
  const long long least = sh.tpr == 64 ? 1 : std::min<long long>(rows, 128);
  return (int)std::min(most, std::max((rows + 3) / 4, least));
}

int check_norm(const ax_norm_desc_t* d) {
  if (!d) return AX_ERR_NULL;
  if ((d->dtype != AX_F32 && d->dtype != AX_BF16) || (d->w_dtype != AX_F32 && d->w_dtype != AX_BF16)) return AX_ERR_OPTION;
  if (d->normalize & ~1) return AX_ERR_OPTION;
  if (!(d->eps >= 0.f) || !std::isfinite(d->eps)) return AX_ERR_OPTION;
  if (d->rows < 0 || d->cols < 1 || d->rows > 0x7fffffff || d->cols > 0x7fffffff - 32768) return AX_ERR_SHAPE;
  return AX_OK;
}

bool aligned_to(const void* p, int esz) { return (uintptr_t)p % esz == 0; }

int norm_common(const ax_norm_desc_t* d, NormArgs& a, bool codes, hipStream_t s) {
  const int e = d->dtype == AX_F32 ? 4 : 2, we = d->w_dtype == AX_F32 ? 4 : 2;
  if (d->x_ld < d->cols || (a.res && d->residual_ld < d->cols) || (a.sum && d->sum_ld < d->cols) ||
      (a.y && d->y_ld < d->cols))
    return AX_ERR_SHAPE;
  if (d->rows == 0) return AX_OK;
  if (!a.x || (a.sum && !a.res)) return AX_ERR_NULL;
  for (const void* p : {a.x, a.res, (const void*)a.sum, (const void*)a.y})
    if (!aligned_to(p, e)) return AX_ERR_ALIGN;
  for (const void* p : {(const void*)a.scales, (const void*)a.values, (const void*)a.rstd})
    if (!aligned_to(p, 4)) return AX_ERR_ALIGN;
  if (!aligned_to(a.w, we)) return AX_ERR_ALIGN;
  a.rows = d->rows;
  a.cols = (int)d->cols;
  a.x_ld = d->x_ld;
  a.r_ld = d->residual_ld;
  a.s_ld = d->sum_ld;
  a.y_ld = d->y_ld;
  a.w_f32 = d->w_dtype == AX_F32;
  a.normalize = d->normalize;
  a.eps = d->eps;
  const bool f32 = d->dtype == AX_F32;
  if (codes) f32 ? norm_launch<kCodes, true>(a, s) : norm_launch<kCodes, false>(a, s);
  else f32 ? norm_launch<kValues, true>(a, s) : norm_launch<kValues, false>(a, s);
  return hipGetLastError() == hipSuccess ? AX_OK : AX_ERR_HIP;
}

}  // namespace

hipError_t launch_column_sum(const float* part, int rows, int cols, float* out, hipStream_t s) {
  column_sum_kernel<<<std::min((cols + 15ll) / 16, 65536ll), 1024, 0, s>>>(part, rows, cols, out);
  return hipGetLastError();
}

}  // namespace ax

using namespace ax;

extern "C" int ax_rmsnorm(const ax_norm_desc_t* d, const void* x, const void* residual, const void* weight, void* sum_out,
                          void* y_out, float* rstd_out, void* hip_stream) {
  if (int rc = check_norm(d)) return rc;
  if (!d->normalize) return AX_ERR_OPTION;
  if (d->rows > 0 && (!weight || !y_out)) return AX_ERR_NULL;
  NormArgs a{};
  a.x = x;
  a.res = residual;
  a.w = weight;
  a.sum = sum_out;
  a.y = y_out;
  a.rstd = rstd_out;
  return norm_common(d, a, false, (hipStream_t)hip_stream);
}

extern "C" int ax_rmsnorm_q8(const ax_norm_desc_t* d, const void* x, const void* residual, const void* weight, void* sum_out,
                             int8_t* codes_out, float* scales_out, float* values_out, void* hip_stream) {
  if (int rc = check_norm(d)) return rc;
  if (d->rows > 0 && (!codes_out || !scales_out)) return AX_ERR_NULL;
  NormArgs a{};
  a.x = x;
  a.res = residual;
  a.w = weight;
  a.sum = sum_out;
  a.codes = codes_out;
  a.scales = scales_out;
  a.values = values_out;
  return norm_common(d, a, true, (hipStream_t)hip_stream);
}

extern "C" size_t ax_rmsnorm_backward_workspace_bytes(const ax_norm_desc_t* d) {
  if (check_norm(d) != AX_OK || d->rows == 0) return 0;
  return ((size_t)grad_groups(d->rows, d->cols) * d->cols * 4 + 255) / 256 * 256;
}

extern "C" int ax_rmsnorm_backward(const ax_norm_desc_t* d, const void* gy, const void* gsum, const void* t, const void* weight,
                                   const float* rstd, void* gx_out, float* gw_out, void* workspace, size_t workspace_bytes,
                                   void* hip_stream) {
  if (int rc = check_norm(d)) return rc;
  if (!d->normalize) return AX_ERR_OPTION;
  if (d->rows > 0 && !gx_out && !gw_out) return AX_ERR_NULL;  // (a gradient of no rows may be NULL)
  if (d->x_ld < d->cols || d->y_ld < d->cols || (gsum && d->residual_ld < d->cols) || (gx_out && d->sum_ld < d->cols))
    return AX_ERR_SHAPE;
  const int e = d->dtype == AX_F32 ? 4 : 2, we = d->w_dtype == AX_F32 ? 4 : 2;
  for (const void* p : {gy, gsum, t, (const void*)gx_out})
    if (!aligned_to(p, e)) return AX_ERR_ALIGN;
  if (!aligned_to(weight, we) || !aligned_to(rstd, 4) || !aligned_to(gw_out, 4)) return AX_ERR_ALIGN;
  const hipStream_t s = (hipStream_t)hip_stream;
  if (d->rows == 0) {  // no rows: their sum
    if (gw_out && launch_column_sum(gw_out, 0, (int)d->cols, gw_out, s) != hipSuccess) return AX_ERR_HIP;
    return AX_OK;
  }
  if (!gy || !t || !weight || !rstd) return AX_ERR_NULL;
  if (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < ax_rmsnorm_backward_workspace_bytes(d)) return AX_ERR_WORKSPACE;
  NormGradArgs a{};
  a.gy = gy;
  a.gsum = gsum;
  a.t = t;
  a.w = weight;
  a.rstd = rstd;
  a.gx = gx_out;
  a.part = gw_out ? (float*)workspace : nullptr;
  a.rows = d->rows;
  a.t_ld = d->x_ld;
  a.gs_ld = d->residual_ld;
  a.gx_ld = d->sum_ld;
  a.gy_ld = d->y_ld;
  a.cols = (int)d->cols;
  a.w_f32 = d->w_dtype == AX_F32;
  const bool f32 = d->dtype == AX_F32;
  const Shape sh = grad_shape_of(d->cols);
  const int groups = grad_groups(d->rows, d->cols);
  if (sh.nv == 0) {
    if (gx_out) {
      for (a.row0 = 0; a.row0 < a.rows; a.row0 += kMaxGrid) {
        const unsigned grid = (unsigned)std::min<long long>(a.rows - a.row0, kMaxGrid);
        if (f32) norm_grad_long_kernel<true><<<grid, 1024, 0, s>>>(a);
        else norm_grad_long_kernel<false><<<grid, 1024, 0, s>>>(a);
      }
    }
    if (gw_out) {
      const dim3 grid((a.cols + 255) / 256, groups);
      if (f32) norm_gw_long_kernel<true><<<grid, 256, 0, s>>>(a);
      else norm_gw_long_kernel<false><<<grid, 256, 0, s>>>(a);
    }
  } else {
    f32 ? norm_grad_launch<true>(a, sh, groups, s) : norm_grad_launch<false>(a, sh, groups, s);
  }
  if (hipGetLastError() != hipSuccess) return AX_ERR_HIP;
  if (gw_out && launch_column_sum(a.part, groups, a.cols, gw_out, s) != hipSuccess) return AX_ERR_HIP;
  return AX_OK;
}
