// Feed-forward products of rows grouped by expert and their gradients: validation, operand copies and launches.
//
//   row r of the products is row index[r] of x (r itself without an index) and belongs to the expert e with
//   offsets[e] <= r < offsets[e + 1]:
//   z = x w_e,  y = act(z)                gz = gy act'(z),  gx = gz w_e^T,  gw_e = sum over the rows of e of x^T gz
//   h = act(x wg_e) (x wu_e)              gg = gh u act'(g),  gu = gh act(g),  gx = gg wg_e^T + gu wu_e^T, ...
//
// Two forms: few rows an expert (launch_few_experts: weights read once, straight into registers, rows found through the index)
// and tiles (launch_gemm_experts), which find rows that they can read in place through the index as well; others, and those of
// the weights' gradients, where rows are the contraction, are copied first.
#include <algorithm>

#include "ax_float.h"
#include "ax_group.h"
#include "ax_operand.h"
#include "axconv_probe.h"

namespace ax {
namespace {

// Whether the tiles find indexed rows themselves (forward): where they could read x in place, and count its bytes in 31 bits.  us at
// experts / rows / inputs / outputs of a gated pair, found : copied first: 8/16384/2048/8192 904 : 929, 32/8192/1024/1416 63 : 69,
// 16/1024/2048/1408 31 : 35.
bool found_in_place(const ax_experts_desc_t* d) {
  return d->indexed && d->x_rows > 0 && d->dtype == AX_BF16 && !d->unaligned && d->K % 8 == 0 && d->x_ld % 8 == 0 &&
         d->x_rows * d->x_ld * 2 < 1ll << 31;
}
// x as the tiles read it: in place, or copied, in the order of the products where it is indexed and not found.
Operand make_rows(const ax_experts_desc_t* d, bool found, const void* x, const int32_t* index, Arena& ar, PackJob* job) {
  const Operand o = make_operand(x, found ? d->x_rows : d->rows, d->K, d->x_ld, d->dtype, d->unaligned || (d->indexed && !found), ar, job);
  if (!found) {
    job->index = index;
    job->src_rows = (int)d->x_rows;
  }
  return o;
}

int check_experts(const ax_experts_desc_t* d, bool backward, bool gated) {
  if (!d) return AX_ERR_NULL;
  if (!dtype_ok(d->dtype) || d->act < AX_ACT_NONE || d->act > AX_ACT_GELU) return AX_ERR_OPTION;
  if ((d->w_transposed & ~1) || (d->indexed & ~1) || (d->unaligned & ~1) || (gated && d->w_transposed)) return AX_ERR_OPTION;
  if (d->rows < 0 || d->x_rows < 0 || d->N < 1 || d->K < 1 || d->rows > kMaxDim || d->x_rows > kMaxDim || d->N > kMaxDim || d->K > kMaxDim)
    return AX_ERR_SHAPE;
  if (d->experts < 1 || d->experts > kMaxExperts || (long long)d->experts * std::max(d->N, d->K) >= 1ll << 31) return AX_ERR_SHAPE;
  if (!d->indexed && d->x_rows != d->rows) return AX_ERR_SHAPE;
  const int e = elem_bytes(d->dtype);
  if (!pitch_ok(d->x_ld, d->K, e) || !pitch_ok(d->w_ld, d->w_transposed ? d->K : d->N, e) || !pitch_ok(d->y_ld, d->N, e) ||
      (backward && !pitch_ok(d->gx_ld, d->K, e)))
    return AX_ERR_SHAPE;
  return AX_OK;
}
long long weight_rows(const ax_experts_desc_t* d) { return d->w_transposed ? d->N : d->K; }
long long weight_cols(const ax_experts_desc_t* d) { return d->w_transposed ? d->K : d->N; }

// ---- forward -----------------------------------------------------------------------------------

struct Forward {
  bool few, found;
  PackJob jobs[3];  // x, w, wu
  GemmArgs g;
  Groups e;
  int tile;
  size_t bytes;
};

// Whether the experts' rows are so few that launch_few_experts, which reads the weights as they lie, is worth it.  us at experts /
// inputs / outputs (rows of each expert), few : tiles.
//   bf16, in place: while its workgroups (32 columns of an expert each) are few as well, since it reads all x in each of them
//     64/1024/1024 (1) 30 : 22, (14) 35 : 23   8/2048/4096 (one row of two) 9 : 14, (8) 27 : 22   4/4096/2048 (8) 16 : 23, (20) 17 : 23
//   bf16, weights that the tiles copy first: 16/1001/777 gated (4) 30 : 29, (14) 32 : 29   [N, K] (8) 17 : 23, (20) 29 : 23
//   float32, weights that the tiles take in copied pieces: 64/1024/1024 (30) 96 : 212, (60) 174 : 220   [N, K] (20) 140 : 214, (60) 295 : 230
//     8/2048/4096 (60) 146 : 213   [N, K] (30) 127 : 213, (60) 245 : 219   32/256/512 [N, K] (20) 21 : 27, (30) 23 : 27
bool few_fits(const ax_experts_desc_t* d) {
  if (d->x_rows == 0) return false;  // (it reads some row of x for an index outside)
  const long long used = std::min<long long>(d->experts, d->rows), tiles = (d->N + 31) / 32;
  if ((d->rows / 16 + used) * 2 * tiles >= 1 << 21) return false;  // (a launch counts its threads in 32 bits)
  if (d->dtype == AX_F32) return d->rows <= (d->w_transposed ? 40 : 64) * used;
  const bool in_place = !d->unaligned && weight_cols(d) % 8 == 0 && d->w_ld % 8 == 0;
  return d->rows <= (!in_place ? 12 : used * tiles <= 256 ? 20 : used * tiles <= 512 ? 8 : 0) * used;
}

Forward make_forward(const ax_experts_desc_t* d, bool gated, const void* x, const int32_t* index, const int32_t* offsets, const void* w,
                     const void* w2, void* ws) {
  Forward f{};
  Arena ar(ws);
  GemmArgs& g = f.g;
  const long long wr = weight_rows(d), wc = weight_cols(d);
  f.e = Groups{offsets, d->experts, (int)d->rows, nullptr, 0};
  f.few = few_fits(d);
  if (f.few) {
    const int esz = elem_bytes(d->dtype);
    g.seg[g.nseg++] = GemmSeg{x, w, w2};
    g.K = (int)d->K;
    g.lda = d->x_ld * esz;
    g.ldb = d->w_ld * esz;
  } else {
    f.found = found_in_place(d);
    const Operand a = make_rows(d, f.found, x, index, ar, &f.jobs[0]);
    const Operand b = make_operand(w, d->experts * wr, wc, d->w_ld, d->dtype, d->unaligned, ar, &f.jobs[1]);
    Operand b2{};
    if (gated) b2 = make_operand(w2, d->experts * wr, wc, d->w_ld, d->dtype, d->unaligned, ar, &f.jobs[2]);
    add_segment(&g, a, b, gated ? &b2 : nullptr);
    g.K = (int)(d->w_transposed ? a.cols : d->K);  // (whole chunks where both operands have the contraction contiguous)
  }
  g.lb = d->w_transposed ? 0 : 1;
  g.M = (int)d->rows;
  g.N = (int)d->N;
  g.gated = gated;
  g.odt = d->dtype;
  g.act = d->act;
  g.ldy = d->y_ld;
  if (!f.few) f.tile = plan_experts(g, f.e, false);
  f.bytes = ar.used;
  return f;
}

int run_forward(Forward& f, const ax_experts_desc_t* d, const int32_t* index, hipStream_t s) {
  if (f.few) return launch_few_experts(f.g, d->dtype, f.e, index, (int)d->x_rows, s) == hipSuccess ? AX_OK : AX_ERR_HIP;
  if (f.found) {
    f.e.index = index;
    f.e.x_rows = (int)d->x_rows;
  }
  const bool wanted[3] = {true, true, f.g.gated != 0};
  PackBatch copies{};
  const int blocks = fill_pack(&copies, f.jobs, wanted, 3);
  if (run_pack(copies, blocks, s) != hipSuccess) return AX_ERR_HIP;
  return launch_gemm_experts(f.g, f.e, false, f.tile, s) == hipSuccess ? AX_OK : AX_ERR_HIP;
}

// ---- backward ----------------------------------------------------------------------------------

struct Backward {
  PackJob jobs[3];  // x, w, wu
  GradArgs ga;
  bool elementwise;
  GemmArgs gx, gw;
  Groups e;
  int tile_x, tile_w;
  size_t bytes;
};

Backward make_backward(const ax_experts_desc_t* d, bool gated, const void* gy, const void* x, const int32_t* index, const int32_t* offsets,
                       const void* w, const void* w2, const void* z, const void* u, void* ws) {
  Backward b{};
  Arena ar(ws);
  const int dt = d->dtype;
  const long long wr = weight_rows(d), wc = weight_cols(d);
  b.e = Groups{offsets, d->experts, (int)d->rows, nullptr, 0};
  const Operand ox = make_rows(d, false, x, index, ar, &b.jobs[0]);
  const Operand ow = make_operand(w, d->experts * wr, wc, d->w_ld, dt, d->unaligned, ar, &b.jobs[1]);
  Operand ow2{}, oz{}, ou{};
  if (gated) ow2 = make_operand(w2, d->experts * wr, wc, d->w_ld, dt, d->unaligned, ar, &b.jobs[2]);
  // gz as an operand: gy itself where nothing is multiplied to it and it can be read in place
  PackJob unused;
  const bool plain = !gated && d->act == AX_ACT_NONE;
  const bool in_place = plain && dt == AX_BF16 && !d->unaligned && d->N % 8 == 0 && d->y_ld % 8 == 0;
  const long long pcols = (d->N + 7) / 8 * 8;
  oz = make_operand(gy, d->rows, d->N, d->y_ld, dt, !in_place, ar, &unused);
  GradArgs& ga = b.ga;
  if (!in_place) {
    ga.gz = unused.dst;
    if (gated) {
      ou = make_operand(gy, d->rows, d->N, d->y_ld, dt, true, ar, &unused);
      ga.gu = unused.dst;
    }
  }
  b.elementwise = !in_place;
  ga.gy = gy;
  ga.z = plain ? nullptr : z;
  ga.u = u;
  ga.ldy = d->y_ld;
  ga.pcols = pcols;
  ga.pitch = oz.ld / 2;
  ga.M = (int)d->rows;
  ga.N = (int)d->N;
  ga.act = d->act;
  ga.rows_per = rows_per_block((int)d->rows, (int)d->N);
  ga.wide = (int)((pcols + 255) / 256);
  ga.blocks = ga.wide * (int)((d->rows + ga.rows_per - 1) / ga.rows_per);

  GemmArgs& gx = b.gx;  // gx [rows, K] = gz [rows, N] w_e^T
  add_segment(&gx, oz, ow, nullptr);
  if (gated) add_segment(&gx, ou, ow2, nullptr);
  gx.lb = d->w_transposed ? 1 : 0;
  gx.M = (int)d->rows;
  gx.N = (int)d->K;
  gx.K = (int)(d->w_transposed ? d->N : pcols);
  gx.odt = dt;
  gx.ldy = d->gx_ld;
  b.tile_x = plan_experts(gx, b.e, false);

  GemmArgs& gw = b.gw;  // gw_e [K, N] = x^T gz over the rows of e, or [N, K] = gz^T x
  if (d->w_transposed) add_segment(&gw, oz, ox, nullptr);
  else add_segment(&gw, ox, oz, gated ? &ou : nullptr);
  gw.la = gw.lb = 1;
  gw.M = (int)wr;
  gw.N = (int)wc;
  gw.K = (int)d->rows;
  gw.dual = gated;
  gw.odt = dt;
  gw.ldy = d->w_ld;
  b.tile_w = plan_experts(gw, b.e, true);
  b.bytes = ar.used;
  return b;
}

int backward_common(const ax_experts_desc_t* d, bool gated, const void* gy, const void* x, const int32_t* index, const int32_t* offsets,
                    const void* w, const void* w2, const void* z, const void* u, void* gx_out, void* gw_out, void* gw2_out, void* ws,
                    size_t ws_bytes, hipStream_t s) {
  const int esz = elem_bytes(d->dtype);
  if (d->rows == 0) {
    hipError_t rc = hipSuccess;
    for (void* p : {gw_out, gw2_out})
      if (p && rc == hipSuccess) rc = zero_rows(p, d->experts * weight_rows(d), weight_cols(d), d->w_ld, esz, s);
    return rc == hipSuccess ? AX_OK : AX_ERR_HIP;
  }
  Backward b = make_backward(d, gated, gy, x, index, offsets, w, w2, z, u, ws);
  if ((gx_out && !experts_fit(b.gx, b.e, false, b.tile_x)) || (gw_out && !experts_fit(b.gw, b.e, true, b.tile_w))) return AX_ERR_SHAPE;
  if (!ws_ok(ws, ws_bytes, b.bytes)) return AX_ERR_WORKSPACE;
  const bool wanted[3] = {gw_out != nullptr, gx_out != nullptr, gx_out && gated};
  PackBatch copies{};
  const int blocks = fill_pack(&copies, b.jobs, wanted, 3);
  if (b.elementwise) {
    if (launch_act_grad(b.ga, gated, copies, blocks, d->dtype, s) != hipSuccess) return AX_ERR_HIP;
  } else if (run_pack(copies, blocks, s) != hipSuccess) {
    return AX_ERR_HIP;
  }
  if (gx_out) {
    b.gx.y = gx_out;
    if (launch_gemm_experts(b.gx, b.e, false, b.tile_x, s) != hipSuccess) return AX_ERR_HIP;
  }
  if (gw_out) {
    b.gw.y = gw_out;
    b.gw.y2 = gw2_out;
    if (launch_gemm_experts(b.gw, b.e, true, b.tile_w, s) != hipSuccess) return AX_ERR_HIP;
  }
  return AX_OK;
}

// Pointers that all calls share.  AX_OK, or what is wrong with them.
int check_rows(const ax_experts_desc_t* d, const void* x, bool need_x, const int32_t* index, const int32_t* offsets) {
  if (!offsets || (d->indexed != 0) != (index != nullptr) || (need_x && !x && d->x_rows > 0)) return AX_ERR_NULL;
  if (!aligned_to(offsets, 4) || !aligned_to(index, 4)) return AX_ERR_ALIGN;
  return operand_aligned(x, elem_bytes(d->dtype), d->unaligned, d->K, d->x_ld, d->dtype) ? AX_OK : AX_ERR_ALIGN;
}
int check_weight(const ax_experts_desc_t* d, const void* w) {
  return operand_aligned(w, elem_bytes(d->dtype), d->unaligned, weight_cols(d), d->w_ld, d->dtype) ? AX_OK : AX_ERR_ALIGN;
}

}  // namespace
}  // namespace ax

using namespace ax;

extern "C" size_t ax_matmul_experts_workspace_bytes(const ax_experts_desc_t* d) {
  if (check_experts(d, false, false) != AX_OK || d->rows == 0) return 0;
  return make_forward(d, false, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_matmul_experts(const ax_experts_desc_t* d, const void* x, const int32_t* index, const int32_t* offsets, const void* w,
                                 void* y_out, void* z_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_experts(d, false, false)) return rc;
  if (d->rows == 0) return AX_OK;
  if (int rc = check_rows(d, x, true, index, offsets)) return rc;
  if (!w || !y_out) return AX_ERR_NULL;
  if (int rc = check_weight(d, w)) return rc;
  for (const void* p : {(const void*)y_out, (const void*)z_out})
    if (!aligned_to(p, elem_bytes(d->dtype))) return AX_ERR_ALIGN;
  Forward f = make_forward(d, false, x, index, offsets, w, nullptr, workspace);
  if (!f.few && !experts_fit(f.g, f.e, false, f.tile)) return AX_ERR_SHAPE;
  if (!ws_ok(workspace, workspace_bytes, f.bytes)) return AX_ERR_WORKSPACE;
  f.g.y = y_out;
  f.g.z = z_out;
  return run_forward(f, d, index, (hipStream_t)hip_stream);
}

extern "C" size_t ax_gated_experts_workspace_bytes(const ax_experts_desc_t* d) {
  if (check_experts(d, false, true) != AX_OK || d->rows == 0) return 0;
  return make_forward(d, true, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_gated_experts(const ax_experts_desc_t* d, const void* x, const int32_t* index, const int32_t* offsets, const void* wg,
                                const void* wu, void* h_out, void* g_out, void* u_out, void* workspace, size_t workspace_bytes,
                                void* hip_stream) {
  if (int rc = check_experts(d, false, true)) return rc;
  if (!g_out != !u_out) return AX_ERR_NULL;
  if (d->rows == 0) return AX_OK;
  if (int rc = check_rows(d, x, true, index, offsets)) return rc;
  if (!wg || !wu || !h_out) return AX_ERR_NULL;
  for (const void* p : {wg, wu})
    if (int rc = check_weight(d, p)) return rc;
  for (const void* p : {(const void*)h_out, (const void*)g_out, (const void*)u_out})
    if (!aligned_to(p, elem_bytes(d->dtype))) return AX_ERR_ALIGN;
  Forward f = make_forward(d, true, x, index, offsets, wg, wu, workspace);
  if (!f.few && !experts_fit(f.g, f.e, false, f.tile)) return AX_ERR_SHAPE;
  if (!ws_ok(workspace, workspace_bytes, f.bytes)) return AX_ERR_WORKSPACE;
  f.g.y = h_out;
  f.g.z = g_out;
  f.g.z2 = u_out;
  return run_forward(f, d, index, (hipStream_t)hip_stream);
}

extern "C" size_t ax_matmul_experts_backward_workspace_bytes(const ax_experts_desc_t* d) {
  if (check_experts(d, true, false) != AX_OK || d->rows == 0) return 0;
  return make_backward(d, false, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_matmul_experts_backward(const ax_experts_desc_t* d, const void* gy, const void* x, const int32_t* index,
                                          const int32_t* offsets, const void* w, const void* z, void* gx_out, void* gw_out,
                                          void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_experts(d, true, false)) return rc;
  if (d->rows > 0 && !gx_out && !gw_out) return AX_ERR_NULL;  // (a gradient of no rows may be NULL)
  const int e = elem_bytes(d->dtype);
  if (d->rows > 0) {
    if (int rc = check_rows(d, x, gw_out != nullptr, index, offsets)) return rc;
    if (!gy || (gx_out && !w) || (d->act != AX_ACT_NONE && !z)) return AX_ERR_NULL;
    if (int rc = check_weight(d, w)) return rc;
    if (!operand_aligned(gy, e, d->unaligned || d->act != AX_ACT_NONE, d->N, d->y_ld, d->dtype)) return AX_ERR_ALIGN;
  }
  for (const void* p : {z, (const void*)gx_out, (const void*)gw_out})
    if (!aligned_to(p, e)) return AX_ERR_ALIGN;
  return backward_common(d, false, gy, x, index, offsets, w, nullptr, z, nullptr, gx_out, gw_out, nullptr, workspace, workspace_bytes,
                         (hipStream_t)hip_stream);
}

extern "C" size_t ax_gated_experts_backward_workspace_bytes(const ax_experts_desc_t* d) {
  if (check_experts(d, true, true) != AX_OK || d->rows == 0) return 0;
  return make_backward(d, true, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr).bytes;
}

extern "C" int ax_gated_experts_backward(const ax_experts_desc_t* d, const void* gh, const void* x, const int32_t* index,
                                         const int32_t* offsets, const void* wg, const void* wu, const void* g, const void* u,
                                         void* gx_out, void* gwg_out, void* gwu_out, void* workspace, size_t workspace_bytes,
                                         void* hip_stream) {
  if (int rc = check_experts(d, true, true)) return rc;
  if ((!gwg_out != !gwu_out) || (d->rows > 0 && !gx_out && !gwg_out)) return AX_ERR_NULL;
  const int e = elem_bytes(d->dtype);
  if (d->rows > 0) {
    if (int rc = check_rows(d, x, gwg_out != nullptr, index, offsets)) return rc;
    if (!gh || !g || !u || (gx_out && (!wg || !wu))) return AX_ERR_NULL;
    for (const void* p : {wg, wu})
      if (int rc = check_weight(d, p)) return rc;
  }
  for (const void* p : {gh, g, u, (const void*)gx_out, (const void*)gwg_out, (const void*)gwu_out})
    if (!aligned_to(p, e)) return AX_ERR_ALIGN;
  return backward_common(d, true, gh, x, index, offsets, wg, wu, g, u, gx_out, gwg_out, gwu_out, workspace, workspace_bytes,
                         (hipStream_t)hip_stream);
}

extern "C" int ax_probe_experts_plan(const ax_experts_desc_t* d, int product, int* kernel, int* rows, int* cols, int* per_cu,
                                     int* found) {
  const bool gated = product == AX_PRODUCT_GATED || product == AX_PRODUCT_GATED_GX || product == AX_PRODUCT_GATED_GW;
  const bool gx = product == AX_PRODUCT_MATMUL_GX || product == AX_PRODUCT_GATED_GX;
  const bool gw = product == AX_PRODUCT_MATMUL_GW || product == AX_PRODUCT_GATED_GW;
  if (!gx && !gw && product != AX_PRODUCT_MATMUL && product != AX_PRODUCT_GATED) return AX_ERR_OPTION;
  if (int rc = check_experts(d, gx || gw, gated)) return rc;
  int k = 0, r = 0, c = 0, n = 0, at = 0;
  if (d->rows > 0 && (gx || gw)) {
    const Backward b = make_backward(d, gated, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr);
    gx ? tile_of_experts(b.gx, false, b.tile_x, &r, &c, &n) : tile_of_experts(b.gw, true, b.tile_w, &r, &c, &n);
  } else if (d->rows > 0) {
    const Forward f = make_forward(d, gated, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr);
    k = f.few;
    at = f.found;
    if (!f.few) tile_of_experts(f.g, false, f.tile, &r, &c, &n);
  }
  if (kernel) *kernel = k;
  if (rows) *rows = r;
  if (cols) *cols = c;
  if (per_cu) *per_cu = n;
  if (found) *found = at;
  return AX_OK;
}
