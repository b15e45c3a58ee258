// What the cross attention kernels share: two sets of ranges, query heads side by side.
//
// The query heads that share a key head are rows of one tile: with G of them, tile row r of
// a sample is its query r / G, head hk G + r % G.  A block then reads its keys once for all
// of them, and a single query of G heads is a tile of G rows.
#pragma once

#include "attn.h"

namespace scn {

// Tiles of `rows` tile rows over all samples, numbered as attn.h's with `many` tile rows a row.
struct Place {
  int64_t base;  // first row of the sample
  int m;         // its tile rows
  int first;     // first tile row of the tile, counted in the sample (m: no such tile)
  int sample;
};
__device__ inline int64_t first_tile(const int32_t* ranges, int b, int64_t n, int rows, int many) {
  return range_at(ranges, b, n) * many / rows + b;
}
// Every lane of the wave takes part.
__device__ inline Place find_place(const int32_t* ranges, int batch, int64_t n, int64_t tile,
                                   int rows, int many) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = batch;
  while (len > 1) {
    const int stride = (len + 63) >> 6, b = lo + lane * stride;
    const bool below = lane * stride < len && first_tile(ranges, b, n, rows, many) <= tile;
    const int c = __popcll(__ballot(below));
    const int step = max(c - 1, 0) * stride;
    lo += step;
    len = min(stride, len - step);
  }
  Place s;
  s.sample = __builtin_amdgcn_readfirstlane(lo);
  const int base = __builtin_amdgcn_readfirstlane((int)range_at(ranges, s.sample, n));
  const int end = __builtin_amdgcn_readfirstlane((int)range_at(ranges, s.sample + 1, n));
  s.base = base;
  s.m = max(0, end - base) * many;
  const int64_t local = tile - ((int64_t)base * many / rows + s.sample);
  s.first = local < 0 || local * rows >= s.m ? s.m : (int)(local * rows);
  return s;
}
// The sample of a row; false if it has none.  Every lane of the wave takes part.
__device__ inline bool find_row(const int32_t* ranges, int batch, int64_t n, int row, int& sample) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = batch;
  while (len > 1) {
    const int stride = (len + 63) >> 6, b = lo + lane * stride;
    const bool below = lane * stride < len && range_at(ranges, b, n) <= row;
    const int c = __popcll(__ballot(below));
    const int step = max(c - 1, 0) * stride;
    lo += step;
    len = min(stride, len - step);
  }
  sample = __builtin_amdgcn_readfirstlane(lo);
  return range_at(ranges, sample, n) <= row && row < range_at(ranges, sample + 1, n);
}
// a sample's rows of the other side
__device__ inline void find_rows(const int32_t* ranges, int sample, int64_t n, int64_t& base,
                                 int& m) {
  const int lo = __builtin_amdgcn_readfirstlane((int)range_at(ranges, sample, n));
  const int hi = __builtin_amdgcn_readfirstlane((int)range_at(ranges, sample + 1, n));
  base = lo;
  m = max(0, hi - lo);
}

constexpr int MAX_PARTS = 256;  // of a split axis

// Parts of an axis of about `len` steps: `want` blocks in all, at least `least` steps each.
inline int parts(int64_t blocks, int64_t want, int64_t len, int64_t least) {
  return (int)std::max<int64_t>(
      1, std::min({ceil_div(want, std::max<int64_t>(1, blocks)), len / least, (int64_t)MAX_PARTS}));
}

// host checks of both directions
scn_status check_cross(const char* who, int32_t type, int64_t nq, int64_t nk, int32_t batch,
                       const int32_t* q_ranges, const int32_t* k_ranges, int32_t D, int32_t Hq,
                       int32_t Hk, float scale);

}  // namespace scn
