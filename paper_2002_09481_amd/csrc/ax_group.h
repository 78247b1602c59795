// Rows grouped by expert: where the tile of a workgroup lies.
//
// The experts' sizes are known on the device alone (the router has just counted them), so a launch has as many workgroups as
// there can be tiles, and each looks its own up in the offsets: 64 experts at a time, a lane each, summed over the wave.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "axconv.h"

namespace ax {

constexpr int kMaxExperts = AX_MAX_EXPERTS;

// Rows of an expert, within the rows that there are whatever the offsets hold.
struct Span {
  int first, count;
};
__device__ __forceinline__ Span span_of(const int32_t* offsets, int e, int rows) {
  const int lo = min(max(offsets[e], 0), rows), hi = min(max(offsets[e + 1], lo), rows);
  return Span{lo, hi - lo};
}

// Workgroups b, b + 8, ... share an XCD and its L2: item b of n in an order in which they take neighbouring ones.
__device__ __forceinline__ int xcd_run(int b, int n) {
  const int x = b & 7, i = b >> 3;
  return x * (n >> 3) + min(x, n & 7) + i;
}

struct GroupTile {
  int expert, first, count;  // its rows
  int tile, tiles;           // of the expert's tiles
};

// Tile of workgroup b among all experts' tiles, `per` for every (begun) `height` rows; false where there are not as many.  Without
// offsets all rows are those of one expert.  height and per are above zero.  The tiles of all experts are dealt out in runs
// (xcd_run), so that an XCD has few experts, whose rows and weights it fetches once (the runs of each expert's own tiles: 5 to 25 %
// slower from 16 experts on, the same with fewer).
__device__ __forceinline__ bool find_tile(const int32_t* offsets, int experts, int rows, int height, int per, int b, GroupTile& g) {
  if (!offsets) {
    g = GroupTile{0, 0, rows, b, (rows + height - 1) / height * per};
    if (b >= g.tiles) return false;
    g.tile = xcd_run(b, g.tiles);
    return true;
  }
  const int lane = threadIdx.x & 63;
  Span s;
  int mine, upto;
  auto look = [&](int base) __attribute__((always_inline)) {  // 64 experts from base on; returns their tiles
    s = Span{0, 0};
    if (base + lane < experts) s = span_of(offsets, base + lane, rows);
    mine = (s.count + height - 1) / height * per;
    upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(upto, d);
      if (lane >= d) upto += v;
    }
    return __builtin_amdgcn_readlane(upto, 63);
  };
  auto take = [&](int base, int want) __attribute__((always_inline)) {  // the want-th of those
    const unsigned long long behind = __ballot(want < upto);
    if (!behind) return false;
    const int l = __builtin_ctzll(behind);
    g.expert = base + l;
    g.first = __builtin_amdgcn_readlane(s.first, l);
    g.count = __builtin_amdgcn_readlane(s.count, l);
    g.tiles = __builtin_amdgcn_readlane(mine, l);
    g.tile = want - (__builtin_amdgcn_readlane(upto, l) - g.tiles);
    return g.tile >= 0 && g.tile < g.tiles;  // (sums that leave 32 bits: only with offsets that do not ascend)
  };
  g = GroupTile{};
  int all = look(0);
  if (experts <= 64) return b < all && take(0, xcd_run(b, all));
  int total = all;
  for (int base = 64; base < experts; base += 64) total += look(base);
  if (b >= total) return false;
  int want = xcd_run(b, total), base = 0;
  all = look(0);
  while (want >= all && base + 64 < experts) {
    want -= all;
    base += 64;
    all = look(base);
  }
  return want < all && take(base, want);
}

// The i-th expert by size, the larger ones first, and its rows.  By powers of two, those of one power in their order; up to 64
// experts (a lane each), more in their order.
__device__ __forceinline__ int by_size(const int32_t* offsets, int experts, int rows, int i, Span& s) {
  if (experts > 64) {
    s = span_of(offsets, i, rows);
    return i;
  }
  const int lane = threadIdx.x & 63;
  Span mine{0, 0};
  int power = -1;
  if (lane < experts) {
    mine = span_of(offsets, lane, rows);
    power = 32 - __clz(mine.count);  // (no rows: 0)
  }
  int before = 0, e = i;
  for (int p = 32 - __clz(rows); p >= 0; --p) {
    const unsigned long long all = __ballot(power == p);
    const int n = __popcll(all);
    if (i < before + n) {
      const int rank = __popcll(all & ((1ull << lane) - 1));
      e = __builtin_ctzll(__ballot(power == p && rank == i - before));
      break;
    }
    before += n;
  }
  s = Span{__builtin_amdgcn_readlane(mine.first, e), __builtin_amdgcn_readlane(mine.count, e)};
  return e;
}

}  // namespace ax
