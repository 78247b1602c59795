// The router of a block of experts: each token's choice, the order of its rows by expert, and the way back.
//
//   e_1 .. e_k  the k largest logits of a token, ties to the lowest expert;  w_j = exp(l_j - m) / sum of exp(l - m), over the
//               chosen or over all, m the largest
//   rows by (expert, token, choice): a counting sort.  Counts are sums of whole numbers, so the order of their additions does
//   not show, and every rank comes from ballots: the same order every time.
#include <algorithm>
#include <type_traits>

#include "ax_float.h"
#include "ax_group.h"
#include "ax_operand.h"

namespace ax {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMostChoices = AX_MAX_CHOICES;
constexpr int kMostBlocks = 512;  // of tokens: each block of the second launch reads all their counts

// Over the L lanes (16: a row of the DPP network, or all 64) that share a token; every lane gets the result.
template <int CTRL>
__device__ __forceinline__ uint32_t turned(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int L, typename F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, F f) {
  v = f(v, turned<0x128>(v));  // row_ror 8, 4, 2, 1
  v = f(v, turned<0x124>(v));
  v = f(v, turned<0x122>(v));
  v = f(v, turned<0x121>(v));
  if constexpr (L == 64) {
    v = f(v, (uint32_t)__shfl_xor((int)v, 16));
    v = f(v, (uint32_t)__shfl_xor((int)v, 32));
  }
  return v;
}
template <int L>
__device__ __forceinline__ uint32_t max_over(uint32_t v) { return over_lanes<L>(v, [](uint32_t a, uint32_t b) { return max(a, b); }); }
template <int L>
__device__ __forceinline__ uint32_t min_over(uint32_t v) { return over_lanes<L>(v, [](uint32_t a, uint32_t b) { return min(a, b); }); }
// (a + b = b + a: all lanes of a row add the same pairs, whatever their place)
template <int L>
__device__ __forceinline__ float sum_over(float v) {
  return __uint_as_float(over_lanes<L>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// A number whose order as a whole number is that of the floats; the least is 1 (a NaN: taken as minus infinity, kNone).
constexpr uint32_t kNone = 0x007fffffu;  // minus infinity
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v == 0.f ? 0.f : v);  // (the two zeros are one)
  if ((b & 0x7fffffffu) > 0x7f800000u) return kNone;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }

// exp(l - m) for l <= m; where both are the same infinity, one or (minus infinity: a row that is masked altogether) zero.
__device__ __forceinline__ float exp_below(float l, float m) {
  if (l == m) return m == -__builtin_inff() ? 0.f : 1.f;
  const float d = l - m;
  return d < -126.f ? 0.f : exp_near(d, 0.f);  // (exp of less is below float32's normal numbers)
}

struct RouteArgs {
  const void* logits;
  int32_t* experts_out;
  float* weights_out;
  int32_t* offsets_out;
  int32_t* rows_out;
  int32_t* tokens_out;
  int32_t* counts;  // [blocks][experts]
  long long ld;
  int tokens, experts, k, normalize;
  int per;  // tokens of a block
};

// What the search compares: a logit's order, in the upper half of a word for bf16 (nothing is lost), with the expert in the lower one, so that
// one maximum finds both, ties to the lowest.  (route_kernel for 16384 tokens of 128 experts, 8 chosen: 7.9 us with the search for the
// expert behind that for its logit.)
template <bool F32>
__device__ __forceinline__ uint32_t key_of(float v, int expert) {
  return F32 ? ordered(v) : (ordered(v) & 0xffff0000u) | (0xffffu - (uint32_t)expert);
}
template <bool F32>
__device__ __forceinline__ uint32_t order_of(uint32_t key) {
  return F32 ? key : key & 0x80000000u ? key & 0xffff0000u : key | 0xffffu;
}

// The choice of one token by L lanes; lane j < k gets the j-th chosen expert and its weight (-1 and 0 where only logits of minus
// infinity are left).  Lane l holds experts V l .. V l + V - 1.
template <bool F32, int L, int V>
__device__ __forceinline__ void choose(const RouteArgs& a, int token, int lane, int& expert, float& weight) {
  constexpr int E = V < 8 ? 4 : 8;
  uint32_t o[V];  // (0: none)
  bool nan = false;
  const int first = lane * V;
#pragma unroll
  for (int h = 0; h < V / E; ++h) {
    float v[E];
    load_elems<F32, E>(a.logits, token * a.ld + first + h * E, a.experts - first - h * E, v);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int e = first + h * E + i;
      nan |= e < a.experts && v[i] != v[i];
      o[h * E + i] = e < a.experts ? key_of<F32>(v[i], e) : 0u;
    }
  }
  auto largest = [&]() __attribute__((always_inline)) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) top = max(top, o[i]);
    return max_over<L>(top);
  };
  uint32_t top = largest();
  const float m = unordered(order_of<F32>(top));
  float sum = 0.f;
  if (!a.normalize) {
#pragma unroll
    for (int i = 0; i < V; ++i) sum += o[i] ? exp_below(unordered(order_of<F32>(o[i])), m) : 0.f;
    sum = sum_over<L>(sum);
  }
  expert = -1;
  uint32_t mine = 0;
  for (int j = 0; j < a.k; ++j) {
    if (j) top = largest();
    uint32_t at = 0xffffu - (top & 0xffffu);
    if constexpr (F32) {
      at = 0xffffffffu;
#pragma unroll
      for (int i = V - 1; i >= 0; --i) at = o[i] == top ? (uint32_t)(first + i) : at;
      at = min_over<L>(at);
    }
    if (lane == j) {
      mine = top;
      expert = (int)at;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = (F32 ? (uint32_t)(first + i) == at : o[i] == top) ? 0u : o[i];
  }
  mine = order_of<F32>(mine);
  if (lane >= a.k || mine <= kNone) expert = -1;
  const float e = expert >= 0 ? exp_below(unordered(mine), m) : 0.f;
  if (a.normalize) sum = sum_over<L>(e);
  if (max_over<L>(nan)) sum = __builtin_nanf("");
  weight = expert >= 0 ? e / sum : 0.f;
}

// Inclusive sum over the threads of a workgroup, in their order.
__device__ __forceinline__ int sum_upto(int v, int* waves) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(v, d);
    if (lane >= d) v += u;
  }
  if (lane == 63) waves[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += waves[w];
  __syncthreads();
  return v;
}

struct Shared {
  int32_t next[kMaxExperts];            // the row that an expert's next choice gets
  int32_t count[kMaxExperts];
  int32_t of_wave[kWaves][kMaxExperts];  // an expert's choices in each wave's 64, then in those of the waves before
  int32_t waves[kWaves];
};

// Rows of the choices of tokens t0 .. t1 - 1, 1024 at a time; s.next[e] is the first of expert e's.
__device__ __forceinline__ void place(const RouteArgs& a, int t0, int t1, Shared& s) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const long long end = (long long)t1 * a.k;
  int bits = 1;
  while ((1 << bits) < a.experts) ++bits;
  for (long long i0 = (long long)t0 * a.k; i0 < end; i0 += kThreads) {
    const long long i = i0 + t;
    const int e = i < end ? a.experts_out[i] : -1;
    if (t < a.experts)
#pragma unroll
      for (int w = 0; w < kWaves; ++w) s.of_wave[w][t] = 0;
    __syncthreads();
    unsigned long long same = __ballot(e >= 0);
    for (int b = 0; b < bits; ++b) {
      const unsigned long long set = __ballot((e >> b) & 1);
      same &= (e >> b) & 1 ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (e >= 0 && rank == 0) s.of_wave[wave][e] = __popcll(same);
    __syncthreads();
    int all = 0;
    if (t < a.experts) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const int c = s.of_wave[w][t];
        s.of_wave[w][t] = all;
        all += c;
      }
    }
    __syncthreads();
    if (i < end) {
      int row = -1;
      if (e >= 0) {
        row = s.next[e] + s.of_wave[wave][e] + rank;
        a.tokens_out[row] = (int)(i / a.k);
      }
      a.rows_out[i] = row;
    }
    __syncthreads();
    if (t < a.experts) s.next[t] += all;
    __syncthreads();
  }
}

// s.next[e] from the experts' counts (a thread each): the first row of each expert; writes the offsets where asked to, and
// the token -1 behind the last row.
__device__ __forceinline__ void lay_out(const RouteArgs& a, int count, bool write, Shared& s) {
  const int t = threadIdx.x;
  const int upto = sum_upto(t < a.experts ? count : 0, s.waves);
  if (t < a.experts) s.next[t] = upto - count;
  if (!write) return;
  if (t < a.experts) a.offsets_out[t] = upto - count;
  if (t == kThreads - 1) {
    a.offsets_out[a.experts] = upto;
    s.waves[0] = upto;
  }
  __syncthreads();
  for (long long i = (long long)s.waves[0] + t; i < (long long)a.tokens * a.k; i += kThreads) a.tokens_out[i] = -1;
  __syncthreads();
}

// Choices of a block of tokens, and how many each expert gets of them; one block finishes the order as well (a few tokens
// decoded together: one launch).  16 lanes a token, four tokens a wave: bound by instructions, mostly the k searches.  16384 tokens of
// 128 bf16 logits, 8 chosen: 6.0 us; one token of 64, 6 chosen, 4.7 us.
template <bool F32, int L, int V>
__global__ __launch_bounds__(kThreads) void route_kernel(const RouteArgs a) {
  __shared__ Shared s;
  const int t = threadIdx.x, lane = t % L;
  const int t0 = blockIdx.x * a.per, t1 = min(a.tokens, t0 + a.per);
  s.count[t] = 0;
  __syncthreads();
  for (int token = t0 + t / L; token < t1; token += kThreads / L) {
    int e;
    float w;
    choose<F32, L, V>(a, token, lane, e, w);
    if (lane < a.k) {
      const long long i = (long long)token * a.k + lane;
      a.experts_out[i] = e;
      a.weights_out[i] = w;
      if (e >= 0) atomicAdd(&s.count[e], 1);
    }
  }
  __syncthreads();  // (and what this workgroup has written of experts_out is there for it)
  if (gridDim.x > 1) {
    for (int e = t; e < a.experts; e += kThreads) a.counts[(long long)blockIdx.x * a.experts + e] = s.count[e];
    return;
  }
  lay_out(a, s.count[t], true, s);
  place(a, t0, t1, s);
}

// Rows of a block's choices: the counts of all blocks say where its own begin.  16384 tokens of 128 experts, 8 chosen: 7.9 us, a chain
// of latencies (256 counts of each expert, two sums over the workgroup, the places).
__global__ __launch_bounds__(kThreads) void place_kernel(const RouteArgs a) {
  __shared__ Shared s;
  const int t = threadIdx.x, blocks = gridDim.x, mine = blockIdx.x;
  // thread (part, expert): parts take blocks in turn
  const int parts = max(1, kThreads / a.experts), e = t % a.experts, part = t / a.experts;
  int before = 0, all = 0;
  if (part < parts) {
    // (sixteen loads under way: one after the other, their latencies are most of the launch)
    for (int b0 = part; b0 < blocks; b0 += 16 * parts) {
      int c[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) c[i] = b0 + i * parts < blocks ? a.counts[(long long)(b0 + i * parts) * a.experts + e] : 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        all += c[i];
        before += b0 + i * parts < mine ? c[i] : 0;
      }
    }
  }
  int32_t* sums = &s.of_wave[0][0];  // (not in use yet)
  sums[t] = all;
  sums[kThreads + t] = before;
  __syncthreads();
  all = before = 0;
  if (t < a.experts)
    for (int p = 0; p < parts; ++p) {
      all += sums[p * a.experts + t];
      before += sums[kThreads + p * a.experts + t];
    }
  __syncthreads();
  lay_out(a, all, mine == 0, s);
  if (t < a.experts) s.next[t] += before;
  __syncthreads();
  const int t0 = mine * a.per;
  place(a, t0, min(a.tokens, t0 + a.per), s);
}

// ---- gradient of the logits --------------------------------------------------------------------
//
// inner = sum over j of gw_j w_j.  Over the chosen: gl[e_j] = w_j (gw_j - inner), zero elsewhere.  Over all, with p the softmax:
// gl = p (g - inner), g the gradient of a chosen expert's weight and zero elsewhere.  Bound by memory (6007 tokens of 60 float32
// logits: 3.9 us, mostly the launch).
struct RouteGradArgs {
  const float* gw;
  const void* logits;
  const int32_t* experts;
  const float* weights;
  void* out;
  long long ld, out_ld;
  int tokens, count, k, normalize;
};
template <bool F32, int L, int V>
__global__ __launch_bounds__(256) void route_grad_kernel(const RouteGradArgs a) {
  constexpr int E = V < 8 ? 4 : 8;
  const int lane = threadIdx.x % L, first = lane * V;
  const long long token = (long long)blockIdx.x * (256 / L) + threadIdx.x / L;
  if (token >= a.tokens) return;
  int e = -1;
  float w = 0.f, g = 0.f;
  if (lane < a.k) {
    const long long i = token * a.k + lane;
    e = a.experts[i];
    w = a.weights[i];
    g = a.gw[i];
    if (e < 0) g = w = 0.f;
  }
  const float inner = sum_over<L>(w * g);
  float v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = 0.f;
  const float mine = a.normalize ? w * (g - inner) : g;
  for (int j = 0; j < a.k; ++j) {
    const int ej = __shfl(e, j, L);
    const float gj = __shfl(mine, j, L);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = first + i == ej ? gj : v[i];
  }
  if (!a.normalize) {
    float l[V], sum = 0.f;
    uint32_t top = 0;
#pragma unroll
    for (int h = 0; h < V / E; ++h) {
      float t[E];
      load_elems<F32, E>(a.logits, token * a.ld + first + h * E, a.count - first - h * E, t);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int x = h * E + i;
        l[x] = t[i];
        if (first + x < a.count) top = max(top, ordered(l[x]));
      }
    }
    const float m = unordered(max_over<L>(top));
#pragma unroll
    for (int i = 0; i < V; ++i) {
      l[i] = first + i < a.count ? exp_below(l[i], m) : 0.f;
      sum += l[i];
    }
    sum = sum_over<L>(sum);
    const float each = sum > 0.f ? 1.f / sum : sum;  // (masked altogether: zeros; NaN stays)
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = l[i] * each * (v[i] - inner);
  }
#pragma unroll
  for (int h = 0; h < V / E; ++h) {
    float t[E];
#pragma unroll
    for (int i = 0; i < E; ++i) t[i] = v[h * E + i];
    const int left = a.count - first - h * E;
    if (left > 0) store_elems<F32, E>(a.out, token * a.out_ld + first + h * E, left, t);
  }
}

// ---- the way back ------------------------------------------------------------------------------
//
// y_t = residual_t + sum over j of w_tj h[row_tj], in float32 in the order of the choices; a row outside h (a choice that
// was dropped) counts nothing.  Eight columns a thread, all rows asked for before the first is used.  Bound by memory: two rows and a residual of 8192 x 4096 bf16 48 us, 5.6 TB/s.
struct CombineArgs {
  const void* h;
  const int32_t* rows;
  const float* weights;
  const void* residual;
  void* y;
  const void* gy;
  void* gh;
  float* gw;
  long long h_ld, r_ld, y_ld, gh_ld;
  int tokens, h_rows, cols, k;
  int wide, lanes;  // workgroups along the columns, threads of a workgroup along them
};
constexpr int kAtOnce = 4;  // rows under way

template <bool F32>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a) {
  const int by = blockIdx.x / a.wide, bx = blockIdx.x - by * a.wide;
  const int lane = threadIdx.x & (a.lanes - 1);
  const long long token = (long long)by * (256 / a.lanes) + threadIdx.x / a.lanes;
  const long long c = ((long long)bx * a.lanes + lane) * 8;
  const int left = (int)min(8ll, a.cols - c);
  if (token >= a.tokens || left <= 0) return;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (a.residual) load_elems<F32, 8>(a.residual, token * a.r_ld + c, left, sum);
  const int32_t* rows = a.rows + token * a.k;
  for (int j0 = 0; j0 < a.k; j0 += kAtOnce) {
    float v[kAtOnce][8], w[kAtOnce];
    bool in[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int row = j0 + j < a.k ? rows[j0 + j] : -1;
      in[j] = row >= 0 && row < a.h_rows;
      w[j] = a.weights && in[j] ? a.weights[token * a.k + j0 + j] : 1.f;
      if (in[j]) load_elems<F32, 8>(a.h, row * a.h_ld + c, left, v[j]);
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (in[j]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = __builtin_fmaf(w[j], v[j][e], sum[e]);
      }
  }
  store_elems<F32, 8>(a.y, token * a.y_ld + c, left, sum);
}

// gh[row_tj] = w_tj gy_t, gw_tj = the product of gy_t and h[row_tj] over the columns, summed in a fixed order.  T threads a
// token, four choices at a time.  Bound by memory: four rows of 3001 x 1000 bf16 12.4 us, 4.4 TB/s.
template <bool F32, int T>
__global__ __launch_bounds__(256) void combine_grad_kernel(const CombineArgs a) {
  __shared__ float part[kAtOnce][4];
  const int lane = threadIdx.x % T;
  const long long token = (long long)blockIdx.x * (256 / T) + threadIdx.x / T;
  if (T < 256 && token >= a.tokens) return;  // (whole waves; a token each in the larger form)
  const int32_t* rows = a.rows + token * a.k;
  for (int j0 = 0; j0 < a.k; j0 += kAtOnce) {
    int row[kAtOnce];
    bool in[kAtOnce];
    float w[kAtOnce], dot[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      row[j] = j0 + j < a.k ? rows[j0 + j] : -1;
      in[j] = row[j] >= 0 && row[j] < a.h_rows;
      w[j] = a.weights && in[j] ? a.weights[token * a.k + j0 + j] : 1.f;
      dot[j] = 0.f;
    }
    for (long long c = lane * 8; c < a.cols; c += T * 8) {
      const int left = (int)min(8ll, a.cols - c);
      float gy[8], v[kAtOnce][8];
      load_elems<F32, 8>(a.gy, token * a.y_ld + c, left, gy);
      if (a.gw) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
          if (in[j]) load_elems<F32, 8>(a.h, row[j] * a.h_ld + c, left, v[j]);
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
        if (in[j]) {
          if (a.gw) {
#pragma unroll
            for (int e = 0; e < 8; ++e) dot[j] = __builtin_fmaf(gy[e], v[j][e], dot[j]);
          }
          if (a.gh) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = w[j] * gy[e];
            store_elems<F32, 8>(a.gh, row[j] * a.gh_ld + c, left, v[j]);
          }
        }
    }
    if (!a.gw) continue;
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      dot[j] = sum_over<64>(dot[j]);
      if (T == 256 && (lane & 63) == 0) part[j][lane >> 6] = dot[j];
    }
    if constexpr (T == 256) {
      __syncthreads();
      if (lane < kAtOnce && j0 + lane < a.k)
        a.gw[token * a.k + j0 + lane] = part[lane][0] + part[lane][1] + part[lane][2] + part[lane][3];
      __syncthreads();
    } else {
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
        if (lane == j && j0 + j < a.k) a.gw[token * a.k + j0 + j] = dot[j];
    }
  }
}

// ---- launches and checks -----------------------------------------------------------------------

// 16 lanes a token with 4, 8 or 16 experts each, or a wave with 16 each.
template <typename F>
void by_experts(int experts, F f) {
  if (experts <= 64) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 4>{});
  else if (experts <= 128) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 8>{});
  else if (experts <= 256) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 16>{});
  else f(std::integral_constant<int, 64>{}, std::integral_constant<int, 16>{});
}

// Tokens of a block: what its threads take at a time, more where there would be too many blocks.
int tokens_a_block(long long tokens, int experts) {
  const long long once = kThreads / (experts <= 256 ? 16 : 64);
  const long long blocks = std::min<long long>(kMostBlocks, std::max(1ll, (tokens + once - 1) / once));
  return (int)std::max(1ll, ((tokens + blocks - 1) / blocks + once - 1) / once * once);
}

int check_route(const ax_route_desc_t* d) {
  if (!d) return AX_ERR_NULL;
  if (!dtype_ok(d->dtype) || (d->normalize & ~1)) return AX_ERR_OPTION;
  if (d->tokens < 0 || d->experts < 1 || d->experts > kMaxExperts || d->k < 1 || d->k > kMostChoices || d->k > d->experts ||
      d->tokens > kMaxDim / d->k || !pitch_ok(d->ld, d->experts, elem_bytes(d->dtype)))
    return AX_ERR_SHAPE;
  return AX_OK;
}

size_t route_workspace(const ax_route_desc_t* d) {
  const int per = tokens_a_block(d->tokens, d->experts);
  const long long blocks = (d->tokens + per - 1) / per;
  return blocks > 1 ? (size_t)blocks * d->experts * 4 : 0;
}

int check_combine(const ax_combine_desc_t* d, bool backward, bool residual) {
  if (!d) return AX_ERR_NULL;
  if (!dtype_ok(d->dtype)) return AX_ERR_OPTION;
  const int e = elem_bytes(d->dtype);
  if (d->tokens < 0 || d->h_rows < 0 || d->k < 1 || d->k > kMostChoices || d->tokens > kMaxDim / d->k || d->h_rows > kMaxDim ||
      d->cols < 1 || d->cols > kMaxDim || !pitch_ok(d->h_ld, d->cols, e) || !pitch_ok(d->y_ld, d->cols, e) ||
      (residual && !pitch_ok(d->residual_ld, d->cols, e)) || (backward && !pitch_ok(d->gh_ld, d->cols, e)))
    return AX_ERR_SHAPE;
  return AX_OK;
}

CombineArgs combine_args(const ax_combine_desc_t* d, const void* h, const int32_t* rows, const float* weights) {
  CombineArgs a{};
  a.h = h;
  a.rows = rows;
  a.weights = weights;
  a.h_ld = d->h_ld;
  a.r_ld = d->residual_ld;
  a.y_ld = d->y_ld;
  a.gh_ld = d->gh_ld;
  a.tokens = (int)d->tokens;
  a.h_rows = (int)d->h_rows;
  a.cols = (int)d->cols;
  a.k = d->k;
  return a;
}

}  // namespace
}  // namespace ax

using namespace ax;

extern "C" size_t ax_route_workspace_bytes(const ax_route_desc_t* d) { return check_route(d) == AX_OK ? route_workspace(d) : 0; }

extern "C" int ax_route(const ax_route_desc_t* d, const void* logits, int32_t* experts_out, float* weights_out, int32_t* offsets_out,
                        int32_t* rows_out, int32_t* tokens_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_route(d)) return rc;
  if (!offsets_out || (d->tokens > 0 && (!logits || !experts_out || !weights_out || !rows_out || !tokens_out))) return AX_ERR_NULL;
  if (!aligned_to(logits, elem_bytes(d->dtype))) return AX_ERR_ALIGN;
  for (const void* p : {(const void*)experts_out, (const void*)weights_out, (const void*)offsets_out, (const void*)rows_out, (const void*)tokens_out})
    if (!aligned_to(p, 4)) return AX_ERR_ALIGN;
  if (!ws_ok(workspace, workspace_bytes, route_workspace(d))) return AX_ERR_WORKSPACE;
  RouteArgs a{logits, experts_out, weights_out, offsets_out, rows_out, tokens_out, (int32_t*)workspace, d->ld, (int)d->tokens,
              d->experts, d->k, d->normalize, tokens_a_block(d->tokens, d->experts)};
  const int blocks = (int)std::max(1ll, (long long)(d->tokens + a.per - 1) / a.per);
  const hipStream_t s = (hipStream_t)hip_stream;
  by_experts(d->experts, [&](auto l, auto v) {
    constexpr int L = decltype(l)::value, V = decltype(v)::value;
    if (d->dtype == AX_F32) route_kernel<true, L, V><<<blocks, kThreads, 0, s>>>(a);
    else route_kernel<false, L, V><<<blocks, kThreads, 0, s>>>(a);
  });
  if (hipGetLastError() != hipSuccess) return AX_ERR_HIP;
  if (blocks > 1) place_kernel<<<blocks, kThreads, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? AX_OK : AX_ERR_HIP;
}

extern "C" int ax_route_backward(const ax_route_desc_t* d, const float* gweights, const void* logits, const int32_t* experts,
                                 const float* weights, void* glogits_out, int64_t glogits_ld, void* hip_stream) {
  if (int rc = check_route(d)) return rc;
  if (!pitch_ok(glogits_ld, d->experts, elem_bytes(d->dtype))) return AX_ERR_SHAPE;
  if (d->tokens == 0) return AX_OK;
  if (!gweights || !experts || !weights || !glogits_out || (!d->normalize && !logits)) return AX_ERR_NULL;
  if (!aligned_to(logits, elem_bytes(d->dtype)) || !aligned_to(glogits_out, elem_bytes(d->dtype))) return AX_ERR_ALIGN;
  for (const void* p : {(const void*)gweights, (const void*)experts, (const void*)weights})
    if (!aligned_to(p, 4)) return AX_ERR_ALIGN;
  const hipStream_t s = (hipStream_t)hip_stream;
  const int e = elem_bytes(d->dtype);
  const int64_t most = 1 << 24;  // (a launch counts its threads in 32 bits)
  for (int64_t t0 = 0; t0 < d->tokens; t0 += most) {
    const int n = (int)std::min(most, d->tokens - t0);
    const RouteGradArgs a{gweights + t0 * d->k, logits ? (const char*)logits + t0 * d->ld * e : nullptr, experts + t0 * d->k,
                          weights + t0 * d->k, (char*)glogits_out + t0 * glogits_ld * e, d->ld, glogits_ld, n, d->experts, d->k, d->normalize};
    by_experts(d->experts, [&](auto l, auto v) {
      constexpr int L = decltype(l)::value, V = decltype(v)::value;
      const int grid = (n + 256 / L - 1) / (256 / L);
      if (d->dtype == AX_F32) route_grad_kernel<true, L, V><<<grid, 256, 0, s>>>(a);
      else route_grad_kernel<false, L, V><<<grid, 256, 0, s>>>(a);
    });
    if (hipGetLastError() != hipSuccess) return AX_ERR_HIP;
  }
  return AX_OK;
}

extern "C" int ax_combine(const ax_combine_desc_t* d, const void* h, const int32_t* rows, const float* weights, const void* residual,
                          void* y_out, void* hip_stream) {
  if (int rc = check_combine(d, false, residual != nullptr)) return rc;
  if (d->tokens == 0) return AX_OK;
  if ((d->h_rows > 0 && !h) || !rows || !y_out) return AX_ERR_NULL;
  const int e = elem_bytes(d->dtype);
  if (!aligned_to(h, e) || !aligned_to(residual, e) || !aligned_to(y_out, e) || !aligned_to(rows, 4) || !aligned_to(weights, 4)) return AX_ERR_ALIGN;
  CombineArgs a = combine_args(d, h, rows, weights);
  a.residual = residual;
  a.y = y_out;
  const long long groups = (d->cols + 7) / 8;
  a.lanes = 8;
  while (a.lanes < 256 && a.lanes < groups) a.lanes *= 2;
  a.wide = (int)((groups + a.lanes - 1) / a.lanes);
  const long long grid = (d->tokens + 256 / a.lanes - 1) / (256 / a.lanes) * a.wide;
  if (grid >= 1 << 23) {  // (a launch counts its threads in 32 bits: fewer, by halves of the tokens)
    ax_combine_desc_t half = *d;
    half.tokens = d->tokens / 2;
    if (int rc = ax_combine(&half, h, rows, weights, residual, y_out, hip_stream)) return rc;
    half.tokens = d->tokens - d->tokens / 2;
    const long long at = d->tokens / 2;
    return ax_combine(&half, h, rows + at * d->k, weights ? weights + at * d->k : nullptr,
                      residual ? (const char*)residual + at * d->residual_ld * e : nullptr, (char*)y_out + at * d->y_ld * e, hip_stream);
  }
  const hipStream_t s = (hipStream_t)hip_stream;
  if (d->dtype == AX_F32) combine_kernel<true><<<(int)grid, 256, 0, s>>>(a);
  else combine_kernel<false><<<(int)grid, 256, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? AX_OK : AX_ERR_HIP;
}

extern "C" int ax_combine_backward(const ax_combine_desc_t* d, const void* gy, const void* h, const int32_t* rows, const float* weights,
                                   void* gh_out, float* gweights_out, void* hip_stream) {
  if (int rc = check_combine(d, true, false)) return rc;
  if (d->tokens == 0) return AX_OK;
  if (!gh_out && !gweights_out) return AX_ERR_NULL;
  if (!gy || !rows || (gweights_out && d->h_rows > 0 && !h)) return AX_ERR_NULL;
  const int e = elem_bytes(d->dtype);
  if (!aligned_to(gy, e) || !aligned_to(h, e) || !aligned_to(gh_out, e) || !aligned_to(rows, 4) || !aligned_to(weights, 4) ||
      !aligned_to(gweights_out, 4))
    return AX_ERR_ALIGN;
  const bool large = d->cols > 2048;
  const long long per = large ? 1 : 4, most = 1 << 22;
  for (long long t0 = 0; t0 < d->tokens; t0 += most * per) {  // (a launch counts its threads in 32 bits)
    const long long n = std::min<long long>(d->tokens - t0, most * per);
    CombineArgs a = combine_args(d, h, rows + t0 * d->k, weights ? weights + t0 * d->k : nullptr);
    a.gy = (const char*)gy + t0 * d->y_ld * e;
    a.gh = gh_out;
    a.gw = gweights_out ? gweights_out + t0 * d->k : nullptr;
    a.tokens = (int)n;
    const int grid = (int)((n + per - 1) / per);
    const hipStream_t s = (hipStream_t)hip_stream;
    if (d->dtype == AX_F32) large ? combine_grad_kernel<true, 256><<<grid, 256, 0, s>>>(a) : combine_grad_kernel<true, 64><<<grid, 256, 0, s>>>(a);
    else large ? combine_grad_kernel<false, 256><<<grid, 256, 0, s>>>(a) : combine_grad_kernel<false, 64><<<grid, 256, 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return AX_ERR_HIP;
  }
  return AX_OK;
}
