// Operands of the matrix products as the kernels read them, workspaces, and the checks that the entry points share.
#pragma once

#include <algorithm>

#include "ax_gemm.h"

namespace ax {

constexpr size_t kAlign = 256;

// Hands out pieces of the workspace; with base 0 it only counts.
struct Arena {
  uintptr_t base;
  size_t used = 0;
  explicit Arena(void* p) : base((uintptr_t)p) {}
  void* take(size_t bytes) {
    void* p = (void*)(base + used);
    used += (bytes + kAlign - 1) / kAlign * kAlign;
    return p;
  }
};

inline int elem_bytes(int dtype) { return dtype == AX_F32 ? 4 : 2; }

// A matrix as the products read it: planes of bf16 (or int8) rows whose length is a multiple of 16 bytes.
struct Operand {
  const void* p;
  int planes;       // 3 for float32
  long long plane;  // bytes from one to the next
  long long ld;     // bytes
  long long cols;  // row length, rounded up to whole 16-byte chunks (zeros behind the given columns)
};

struct PackJob {
  const void* src;
  void* dst;  // planes back to back; null: read in place
  long long rows, cols, ld;  // of the source, elements
  long long pcols;  // cols in whole chunks, zeros behind cols
  long long pitch;  // of the copy, elements
  int dtype;  // AX_F32, AX_BF16, or kI8
  const int32_t* index;  // row of the source for each row (null: the same); one outside its src_rows stands for zeros
  int src_rows;
};
constexpr int kI8 = 2;

struct PackBatch {
  PackJob job[3];
  int first[3];  // workgroup that each job starts at
  int blocks[3];
};
// fill_pack: the jobs of an operation that have something to copy (wanted[i]: whether job i is needed by this call); returns
// the workgroups that they take.
int fill_pack(PackBatch* b, const PackJob* jobs, const bool* wanted, int n);
hipError_t run_pack(const PackBatch& b, int grid, hipStream_t s);

inline int grid_for(long long items) { return (int)std::max<long long>(1, std::min<long long>((items + 255) / 256, 8192)); }

// Row pitch of a copy: whole lines of 128 bytes, and not a multiple of 2 KB, at which the pieces of one stage of a tile
// fall on few channels (bf16 8192^3, both operands contiguous along the sum: 956 us at 16 KB, 863 us at 16 KB + 128).
inline long long copy_pitch(long long cols, int esz) {
  const long long line = 128 / esz, pitch = (cols + line - 1) / line * line;
  return pitch * esz % 2048 ? pitch : pitch + line;
}

// Whether the matrix is read in place or copied is decided by its description alone, so that the workspace query knows.
inline Operand make_operand(const void* p, long long rows, long long cols, long long ld, int dtype, bool unaligned, Arena& ar, PackJob* job) {
  Operand o{};
  const int chunk = dtype == kI8 ? 16 : 8, esz = dtype == kI8 ? 1 : 2;
  const long long pcols = (cols + chunk - 1) / chunk * chunk;
  const long long pitch = copy_pitch(cols, esz);
  *job = PackJob{p, nullptr, rows, cols, ld, pcols, pitch, dtype, nullptr, 0};
  o.cols = pcols;
  if (dtype != AX_F32 && !unaligned && pcols == cols && ld % chunk == 0) {
    o.planes = 1;
    o.p = p;
    o.ld = ld * esz;
    return o;
  }
  o.planes = dtype == AX_F32 ? 3 : 1;
  o.ld = pitch * esz;
  const size_t plane = (size_t)rows * pitch * esz;
  job->dst = ar.take(plane * o.planes);
  o.p = job->dst;
  o.plane = (long long)plane;
  return o;
}

// A factor pair of a product (all pairs of a product have the same pitches).
inline void add_segment(GemmArgs* g, const Operand& a, const Operand& b, const Operand* b2) {
  g->seg[g->nseg++] = GemmSeg{a.p, b.p, b2 ? b2->p : nullptr};
  g->pieces = a.planes;
  g->lda = a.ld;
  g->ldb = b.ld;
  g->a_plane = a.plane;
  g->b_plane = b.plane;
}

// The elementwise part of the gradients (act_grad_kernel): gz = gy act'(z), or gg and gu of a gated pair.
struct GradArgs {
  const void* gy;  // [M, N], pitch ldy (GATED: gh)
  const void* z;   // [M, N], pitch N (may be NULL; GATED: the gate projection)
  const void* u;   // GATED
  void* gz;        // planes [M, pcols] (may be NULL: gy itself is read by the products)
  void* gu;        // GATED
  float* part;     // [row blocks][N] (may be NULL)
  long long ldy, pcols, pitch;  // pcols, pitch: of gz and gu
  int M, N, act, rows_per;
  int wide, blocks;  // workgroups along the columns, in all
};

inline int rows_per_block(int M, int N) {  // about eight workgroups per compute unit, at least eight rows each
  const long long cols = (N + 255) / 256;
  const long long want = std::max(1ll, 2048 / cols);
  return (int)std::max(8ll, ((M + want - 1) / want + 7) / 8 * 8);
}

// The elementwise part, with the copies of `copies` (copy_blocks workgroups) in the same launch.
hipError_t launch_act_grad(const GradArgs& a, bool gated, const PackBatch& copies, int copy_blocks, int dtype, hipStream_t s);
// rows x cols elements of esz bytes at pitch ld set to zero.
hipError_t zero_rows(void* p, long long rows, long long cols, long long ld, int esz, hipStream_t s);

constexpr long long kMaxDim = 1 << 30, kMaxPitch = 1 << 22;

inline bool dtype_ok(int d) { return d == AX_F32 || d == AX_BF16; }
inline bool pitch_ok(long long ld, long long cols, int esz) { return ld >= cols && ld * esz < kMaxPitch; }

// 16-byte operands where the description promises them, element alignment otherwise.
inline bool operand_aligned(const void* p, int esz, bool unaligned, long long cols, long long ld, int dtype) {
  if ((uintptr_t)p % esz) return false;
  const int chunk = 16 / esz;
  const bool in_place = dtype != AX_F32 && !unaligned && cols % chunk == 0 && ld % chunk == 0;
  return !in_place || (uintptr_t)p % 16 == 0;
}
inline bool aligned_to(const void* p, int esz) { return (uintptr_t)p % esz == 0; }
inline bool ws_ok(const void* ws, size_t have, size_t need) {
  return need == 0 || (ws && (uintptr_t)ws % kAlign == 0 && have >= need);
}

}  // namespace ax
