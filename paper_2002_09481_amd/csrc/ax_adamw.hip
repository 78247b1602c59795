// AdamW over many tensors in one launch, states in 32 or 8 bits.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g g,  p = p decay - lr m / (sqrt(v) root + eps)
//
// Every line is a float32 operation at a time in the stated order (no contraction into fused multiply-adds, square root
// and division correctly rounded), so that the 8-bit codes, which follow from comparisons of their results, are
// reproducible.  Bound by memory: 28 bytes an element with float32 states, parameters and gradients, 16 with float32
// parameters, bf16 gradients and copies and 8-bit states.  All tensors in one launch, a workgroup for 4096 elements of one
// of them: a step over many small tensors is one launch's latency.
//
// Measured: 302 M elements with 8-bit states 930 to 1055 us (4.8 GB; a copy moves 5.1 TB/s), their states as float32
// values 545 us (5.5 TB/s); 2.3 M elements of 15 tensors with float32 states 12.5 us (5.1 TB/s).
#include <algorithm>
#include <cmath>

#include "ax_float.h"
#include "ax_internal.h"

#pragma clang fp contract(off)

namespace ax {
namespace {

constexpr int kChunk = 4096;  // elements of a workgroup: 16 blocks of 256
constexpr int kThreads = 256;

struct Tensor {
  void* p;
  const void* g;
  void* m;
  void* v;
  float* ms;
  float* vs;
  void* copy;
  long long n;
};
struct Step {
  float b1, nb1, b2, nb2, eps, decay, lr, root;
  const float* grad_scale;
};
// Travels in the kernel arguments: no table in memory, nothing to keep between calls.
struct Batch {
  Tensor t[AX_ADAMW_LAUNCH];
  uint32_t first[AX_ADAMW_LAUNCH];  // first chunk of each tensor (chunks behind the last: 0xffffffff)
  Step s;
};
static_assert(sizeof(Batch) <= 4096, "kernel arguments");

constexpr int kLane = 8;  // consecutive elements of a lane: 32 lanes have a block of the 8-bit states

__device__ __forceinline__ u32x2 get_codes(const uint8_t* p, long long i, int left) {
  if (left >= kLane) return load_any<u32x2>(p + i);
  u32x2 q = {0, 0};
  for (int e = 0; e < kLane; ++e)
    if (e < left) q[e >> 2] |= (uint32_t)p[i + e] << (8 * (e & 3));
  return q;
}
__device__ __forceinline__ void put_codes(uint8_t* p, long long i, int left, u32x2 q) {
  if (left >= kLane) {
    store_any(p + i, q);
    return;
  }
  for (int e = 0; e < kLane; ++e)
    if (e < left) p[i + e] = (uint8_t)(q[e >> 2] >> (8 * (e & 3)));
}

__device__ __forceinline__ float value_m(uint32_t code, float scale) {
  const float r = (float)(int8_t)code * (1.0f / 127.0f);
  return r * fabsf(r) * scale;
}
__device__ __forceinline__ float value_v(uint32_t code, float scale) {
  float r = (float)(code & 0xffu) * (1.0f / 255.0f);
  r = r * r;
  return r * r * scale;
}
// Largest bit pattern over the 32 lanes of a block: of absolute values, so NaN is above infinity and both are above all numbers.
__device__ __forceinline__ uint32_t block_max(uint32_t x) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, off, 64));
  return x;
}
__device__ __forceinline__ float inverse_of(float scale) {
  return scale >= 0x1p-126f && scale < INFINITY ? 1.0f / scale : 0.f;
}

// The tensor that chunk c belongs to: lanes compare the first chunks of all tensors at once.
__device__ __forceinline__ int tensor_of(const uint32_t* first, uint32_t c) {
  const int lane = threadIdx.x & 63;
  const bool below = lane < AX_ADAMW_LAUNCH && first[min(lane, AX_ADAMW_LAUNCH - 1)] <= c;
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(below)) - 1);
}

template <bool PF32, bool GF32, bool Q8>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const Batch b) {
  const int ti = tensor_of(b.first, blockIdx.x);
  const Tensor& T = b.t[ti];
  const Step& s = b.s;
  const long long base = (long long)(blockIdx.x - b.first[ti]) * kChunk;
  const float gs = s.grad_scale ? *s.grad_scale : 1.f;
#pragma unroll
  for (int it = 0; it < kChunk / (kThreads * kLane); ++it) {
    const long long i = base + (it * kThreads + threadIdx.x) * kLane;
    const long long more = T.n - i;
    const int left = more >= kLane ? kLane : more > 0 ? (int)more : 0;
    const long long blk = i / AX_STATE_BLOCK;
    if (T.n <= blk * AX_STATE_BLOCK) break;  // the same for the 32 lanes of a block
    float p[kLane], g[kLane], m[kLane], v[kLane];
    load_elems<PF32>(T.p, i, left, p);
    load_elems<GF32>(T.g, i, left, g);
    if (Q8) {
      const u32x2 qm = get_codes((const uint8_t*)T.m, i, left), qv = get_codes((const uint8_t*)T.v, i, left);
      const float sm = T.ms[blk], sv = T.vs[blk];
#pragma unroll
      for (int e = 0; e < kLane; ++e) {
        m[e] = value_m(qm[e >> 2] >> (8 * (e & 3)), sm);
        v[e] = value_v(qv[e >> 2] >> (8 * (e & 3)), sv);
      }
    } else {
      load_elems<true>(T.m, i, left, m);
      load_elems<true>(T.v, i, left, v);
    }
    uint32_t tm = 0, tv = 0;
#pragma unroll
    for (int e = 0; e < kLane; ++e) {
      const float ge = s.grad_scale ? g[e] * gs : g[e];
      m[e] = s.b1 * m[e] + s.nb1 * ge;
      v[e] = s.b2 * v[e] + s.nb2 * (ge * ge);
      const float u = m[e] / (sqrtf(v[e]) * s.root + s.eps);
      p[e] = p[e] * s.decay - s.lr * u;
      if (Q8 && e < left) {
        tm = max(tm, __float_as_uint(m[e]) & 0x7fffffffu);
        tv = max(tv, __float_as_uint(v[e]) & 0x7fffffffu);
      }
    }
    store_elems<PF32>(T.p, i, left, p);
    if (T.copy) store_elems<false>(T.copy, i, left, p);
    if (Q8) {
      const float sm = __uint_as_float(block_max(tm)), sv = __uint_as_float(block_max(tv));
      const float im = inverse_of(sm), iv = inverse_of(sv);
      u32x2 qm = {0, 0}, qv = {0, 0};
#pragma unroll
      for (int e = 0; e < kLane; ++e) {
        int c = (int)rintf(sqrtf(fabsf(m[e]) * im) * 127.0f);
        if (m[e] < 0.f) c = -c;
        qm[e >> 2] |= ((uint32_t)c & 0xffu) << (8 * (e & 3));
        int k = (int)rintf(sqrtf(sqrtf(v[e] * iv)) * 255.0f);
        if (v[e] > 0.f && iv > 0.f) k = max(k, 1);
        qv[e >> 2] |= ((uint32_t)k & 0xffu) << (8 * (e & 3));
      }
      put_codes((uint8_t*)T.m, i, left, qm);
      put_codes((uint8_t*)T.v, i, left, qv);
      if ((threadIdx.x & 31) == 0) {
        T.ms[blk] = sm;
        T.vs[blk] = sv;
      }
    } else {
      store_elems<true>(T.m, i, left, m);
      store_elems<true>(T.v, i, left, v);
    }
  }
}

// p and copy stand for the two outputs.  Four elements a lane: a wave's stores of 16 bytes are one run of memory (with
// eight, in two halves, 765 us for 302 M elements instead of 565).
__global__ __launch_bounds__(kThreads) void states_kernel(const Batch b) {
  const int ti = tensor_of(b.first, blockIdx.x);
  const Tensor& T = b.t[ti];
  const long long base = (long long)(blockIdx.x - b.first[ti]) * kChunk;
#pragma unroll
  for (int it = 0; it < kChunk / (kThreads * 4); ++it) {
    const long long i = base + (it * kThreads + threadIdx.x) * 4;
    const long long more = T.n - i;
    const int left = more >= 4 ? 4 : more > 0 ? (int)more : 0;
    if (left == 0) break;
    const long long blk = i / AX_STATE_BLOCK;
    const uint8_t *cm = (const uint8_t*)T.m + i, *cv = (const uint8_t*)T.v + i;
    uint32_t qm = 0, qv = 0;
    if (left == 4) {
      qm = load_any<uint32_t>(cm);
      qv = load_any<uint32_t>(cv);
    } else {
      for (int e = 0; e < left; ++e) {
        qm |= (uint32_t)cm[e] << (8 * e);
        qv |= (uint32_t)cv[e] << (8 * e);
      }
    }
    const float sm = T.ms[blk], sv = T.vs[blk];
    float m[4], v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      m[e] = value_m(qm >> (8 * e), sm);
      v[e] = value_v(qv >> (8 * e), sv);
    }
    store_elems<true>(T.p, i, left, m);
    store_elems<true>(T.copy, i, left, v);
  }
}

// Fills a batch with the tensors from *next on; returns its chunks (0: nothing left).
long long fill_batch(Batch* b, const ax_adamw_tensor_t* t, int count, int* next, float* const* m_out, float* const* v_out) {
  long long chunks = 0;
  int k = 0;
  for (int i = 0; i < AX_ADAMW_LAUNCH; ++i) b->first[i] = 0xffffffffu;
  while (*next < count && k < AX_ADAMW_LAUNCH) {
    const ax_adamw_tensor_t& e = t[*next];
    const long long c = (e.n + kChunk - 1) / kChunk;
    if (chunks > 0 && chunks + c >= 1 << 24) break;  // (a launch counts its threads in 32 bits)
    if (e.n > 0) {
      b->t[k] = Tensor{m_out ? (void*)m_out[*next] : e.p, e.g, e.m, e.v, e.m_scale, e.v_scale,
                       v_out ? (void*)v_out[*next] : e.copy, (long long)e.n};
      b->first[k] = (uint32_t)chunks;
      chunks += c;
      ++k;
    }
    ++*next;
  }
  return chunks;
}

}  // namespace
}  // namespace ax

using namespace ax;

extern "C" int ax_adamw(const ax_adamw_desc_t* d, const ax_adamw_tensor_t* tensors, int count, void* hip_stream) {
  if (!d || (count > 0 && !tensors)) return AX_ERR_NULL;
  if (count < 0) return AX_ERR_SHAPE;
  if ((d->p_dtype != AX_F32 && d->p_dtype != AX_BF16) || (d->g_dtype != AX_F32 && d->g_dtype != AX_BF16)) return AX_ERR_OPTION;
  if ((d->state_bits != 32 && d->state_bits != 8) || d->reserved) return AX_ERR_OPTION;
  if (d->step < 1 || !std::isfinite(d->lr) || !std::isfinite(d->weight_decay) || !std::isfinite(d->eps) || d->eps < 0) return AX_ERR_OPTION;
  if (!(d->beta1 >= 0 && d->beta1 < 1) || !(d->beta2 >= 0 && d->beta2 < 1)) return AX_ERR_OPTION;
  if ((uintptr_t)d->grad_scale % 4) return AX_ERR_ALIGN;
  const int pe = d->p_dtype == AX_F32 ? 4 : 2, ge = d->g_dtype == AX_F32 ? 4 : 2;
  const bool q8 = d->state_bits == 8;
  for (int i = 0; i < count; ++i) {
    const ax_adamw_tensor_t& t = tensors[i];
    if (t.n < 0 || t.n >= 1ll << 36) return AX_ERR_SHAPE;
    if (t.n == 0) continue;
    if (!t.p || !t.g || !t.m || !t.v || (q8 && (!t.m_scale || !t.v_scale))) return AX_ERR_NULL;
    if ((uintptr_t)t.p % pe || (uintptr_t)t.g % ge || (uintptr_t)t.copy % 2) return AX_ERR_ALIGN;
    if (q8 ? (uintptr_t)t.m_scale % 4 || (uintptr_t)t.v_scale % 4 : (uintptr_t)t.m % 4 || (uintptr_t)t.v % 4) return AX_ERR_ALIGN;
  }
  Batch b;
  b.s = Step{(float)d->beta1, (float)(1.0 - d->beta1), (float)d->beta2, (float)(1.0 - d->beta2), (float)d->eps,
             (float)(1.0 - d->lr * d->weight_decay), (float)(d->lr / (1.0 - std::pow(d->beta1, (double)d->step))),
             (float)(1.0 / std::sqrt(1.0 - std::pow(d->beta2, (double)d->step))), d->grad_scale};
  int next = 0;
  while (next < count) {
    const long long chunks = fill_batch(&b, tensors, count, &next, nullptr, nullptr);
    if (chunks == 0) break;
    const unsigned grid = (unsigned)chunks;
    const hipStream_t s = (hipStream_t)hip_stream;
    const bool pf = d->p_dtype == AX_F32, gf = d->g_dtype == AX_F32;
    if (q8) {
      if (pf) gf ? adamw_kernel<true, true, true><<<grid, kThreads, 0, s>>>(b) : adamw_kernel<true, false, true><<<grid, kThreads, 0, s>>>(b);
      else gf ? adamw_kernel<false, true, true><<<grid, kThreads, 0, s>>>(b) : adamw_kernel<false, false, true><<<grid, kThreads, 0, s>>>(b);
    } else {
      if (pf) gf ? adamw_kernel<true, true, false><<<grid, kThreads, 0, s>>>(b) : adamw_kernel<true, false, false><<<grid, kThreads, 0, s>>>(b);
      else gf ? adamw_kernel<false, true, false><<<grid, kThreads, 0, s>>>(b) : adamw_kernel<false, false, false><<<grid, kThreads, 0, s>>>(b);
    }
    if (hipGetLastError() != hipSuccess) return AX_ERR_HIP;
  }
  return AX_OK;
}

extern "C" int ax_adamw_states(const ax_adamw_tensor_t* tensors, int count, float* const* m_out, float* const* v_out, void* hip_stream) {
  if (count < 0) return AX_ERR_SHAPE;
  if (count > 0 && (!tensors || !m_out || !v_out)) return AX_ERR_NULL;
  for (int i = 0; i < count; ++i) {
    const ax_adamw_tensor_t& t = tensors[i];
    if (t.n < 0 || t.n >= 1ll << 36) return AX_ERR_SHAPE;
    if (t.n == 0) continue;
    if (!t.m || !t.v || !t.m_scale || !t.v_scale || !m_out[i] || !v_out[i]) return AX_ERR_NULL;
    if ((uintptr_t)t.m_scale % 4 || (uintptr_t)t.v_scale % 4 || (uintptr_t)m_out[i] % 4 || (uintptr_t)v_out[i] % 4) return AX_ERR_ALIGN;
  }
  Batch b{};
  int next = 0;
  while (next < count) {
    const long long chunks = fill_batch(&b, tensors, count, &next, m_out, v_out);
    if (chunks == 0) break;
    states_kernel<<<(unsigned)chunks, kThreads, 0, (hipStream_t)hip_stream>>>(b);
    if (hipGetLastError() != hipSuccess) return AX_ERR_HIP;
  }
  return AX_OK;
}
