// What the cross attention kernels share: two sets of ranges, query heads side by side.
//
// The query heads that share a key head are rows of one tile: with G of them, tile row r of
// a sample is its query r / G, head hk G + r % G.  A block then reads its keys once for all
// of them, and a single query of G heads is a tile of G rows.
#pragma once

#include "attn.h"

namespace scn {

// One side of a call: rows of samples, and how many tile rows each is.
struct Side {
  const int32_t* ranges;
  int64_t n;
  int many;
  // first row of sample b
  __device__ inline int at(int b) const { return (int)range_at(ranges, b, n); }
};

// An axis that is split over blocks: a sample of m steps has of(m) parts, at most `most`, of at
// least `least` steps each but for a sample's last.  Samples differ in length, so the longer
// have more parts and no block has much more to do than another.
constexpr int MAX_PARTS = 256;

struct Parts {
  int most, least;
  __host__ __device__ inline int of(int64_t m) const {
    const int64_t n = (m + least - 1) / least;
    return n < 1 ? 1 : n > most ? most : (int)n;
  }
};

// What a block does: a tile of one side's rows, for a key head, with a part of the other
// side's steps.
struct Work {
  int64_t base, other;  // first rows of the sample on both sides
  int m, mo;            // its tile rows on the tiles' side, its rows on the other
  int first;            // first tile row of the tile, counted in the sample (m: no tile)
  int hk, part, parts;
};

// The work of a launch, one a block.  Unsplit, tiles of `rows` tile rows are numbered as
// attn.h's, tile t of sample b being ranges[b] many / rows + b + t, and no block has to know more
// than its own sample.  Split, each block counts the samples' tiles and parts, 64 samples at a
// time, so that the blocks without work are the last ones: each costs 2 us of a place on the
// card.  Work-groups go to the XCDs in turn, which spreads the key heads of a tile over them;
// `near` has them follow each other on one XCD, for few rows of heads that share cache lines
// (one row over 262,144 states, 4 heads of 32 bf16 channels: 32 us a call, 54 otherwise; 20 rows of
// 16 samples over 8,192 each, 25 and 36; many tiles of rows with whole lines to each head lose 2%,
// for an XCD then reads all heads' states).
struct Deal {
  Side tiles, steps;
  int batch, rows, Hk;
  Parts parts;
  bool near;

  // blocks of a launch
  int64_t blocks() const {
    const int64_t n = (tiles.n * tiles.many / rows + batch) * parts.most;
    return (near ? ceil_div(n, 8) * 8 : n) * Hk;
  }
  __device__ inline int count(int b) const {
    if (b >= batch) return 0;
    const int m = tiles.at(b + 1) - tiles.at(b), o = steps.at(b + 1) - steps.at(b);
    if (m <= 0) return 0;
    return (int)(((int64_t)m * tiles.many + rows - 1) / rows) *
           parts.of(max(o, 0) * (int64_t)steps.many) * Hk;
  }
  // Every lane of the wave takes part.
  __device__ inline Work find(int block) const {
    const int lane = threadIdx.x & 63;
    const int item = near ? (block / (8 * Hk) * 8 + block % 8) * Hk + block / 8 % Hk : block;
    int sample = 0, local = 0;
    bool none = false;  // past the last work
    Work w;
    if (parts.most == 1) {
      const int tile = item / Hk;
      w.hk = item % Hk;
      int len = batch;
      while (len > 1) {
        const int stride = (len + 63) >> 6, b = sample + lane * stride;
        const bool below = lane * stride < len &&
                           tiles.at(b) * (int64_t)tiles.many / rows + b <= tile;
        // (a signed count: a tile of rows in front of all samples has none below it)
        const int c = __popcll(__ballot(below));
        const int step = max(c - 1, 0) * stride;
        sample += step;
        len = min(stride, len - step);
      }
      sample = __builtin_amdgcn_readfirstlane(sample);
      local = tile - (int)(tiles.at(sample) * (int64_t)tiles.many / rows + sample);
    } else {
      local = item;
      for (int b = 0; b < batch; b += 64) {
        const int c = count(b + lane);
        int s = c;  // .. of the samples up to this one
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int x = __shfl_up(s, d);
          s += lane >= d ? x : 0;
        }
        const int here = __popcll(__ballot(s <= local));
        none = here == 64;
        sample = min(b + here, batch - 1);
        local -= __shfl(none ? s : s - c, none ? 63 : here);
        if (!none) break;
      }
    }
    const int base = __builtin_amdgcn_readfirstlane(tiles.at(sample));
    const int end = __builtin_amdgcn_readfirstlane(tiles.at(sample + 1));
    const int other = __builtin_amdgcn_readfirstlane(steps.at(sample));
    const int oend = __builtin_amdgcn_readfirstlane(steps.at(sample + 1));
    w.base = base;
    w.m = max(0, end - base) * tiles.many;
    w.other = other;
    w.mo = max(0, oend - other);
    w.parts = parts.of(w.mo * (int64_t)steps.many);
    w.part = 0;
    if (parts.most > 1) {
      const int n = (w.m + rows - 1) / rows * Hk;
      w.part = n ? __builtin_amdgcn_readfirstlane(local / n) : 0;
      local -= w.part * n;
      w.hk = __builtin_amdgcn_readfirstlane(local % Hk);
      local /= Hk;
    }
    local = __builtin_amdgcn_readfirstlane(local);
    w.first = none || local < 0 || (int64_t)local * rows >= w.m ? w.m : local * rows;
    return w;
  }
};

// Blocks that works of several tiles leave at least (up to 8 tiles to one: 120,011 rows of 4 fp32
// heads on 2 of 32 over 40 states each, forward 53 us in works of 4 tiles, 56 of 2, 70 of 7).
constexpr int FEW_BLOCKS = 768;

// `blocks` blocks over samples of about `mean` steps, cut for `want` blocks in all where there
// are fewer, in parts of `least` steps or more; a sample of twice the mean has all parts that it
// would have by its length.
inline Parts cut(int64_t blocks, int64_t want, int64_t mean, int64_t least, int samples) {
  blocks = std::max<int64_t>(1, blocks);
  least = std::max(least, ceil_div(blocks * mean, want));
  if (blocks >= want || mean <= least) return Parts{1, INT32_MAX};
  const int64_t most = ceil_div(mean, least) * (samples > 1 ? 2 : 1);
  return Parts{(int)std::min<int64_t>(most, MAX_PARTS), (int)std::min<int64_t>(least, INT32_MAX)};
}

// What eight floats' rounding to bf16 left.  Weights and dS are rounded for their products,
// which leaves a sum 1.4 times as far off as its own rounding, and more where one term holds
// it; sums of few terms, which memory bounds, take them in two parts.
__device__ inline Frag<1> low_part(const float (&v)[8], const Frag<1>& hi) {
  Frag<1> f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    f.s[0][j] = cvt2_bf16(v[2 * j] - __uint_as_float(hi.s[0][j] << 16),
                          v[2 * j + 1] - __uint_as_float(hi.s[0][j] & 0xffff0000u));
  return f;
}

// A lane's row of an operand on its way from memory (load_frag in two steps).
template <int NS, int DP>
struct Ahead {
  static constexpr int N = NS == 1 ? 1 : 2;
  v4u r[DP / 16][N];
  __device__ inline void load(const typename Elem<NS>::T* row, int D, int lane) {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      const int c = 16 * s + 8 * (lane >> 5);
#pragma unroll
      for (int i = 0; i < N; ++i)
        r[s][i] = c < D ? *reinterpret_cast<const v4u*>(row + c + 4 * i) : v4u{0, 0, 0, 0};
    }
  }
  __device__ inline void floats(int s, float (&v)[8]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (NS == 1) {
        v[2 * j] = __uint_as_float(r[s][0][j] << 16);
        v[2 * j + 1] = __uint_as_float(r[s][0][j] & 0xffff0000u);
      } else {
        v[j] = __uint_as_float(r[s][0][j]);
        v[4 + j] = __uint_as_float(r[s][N - 1][j]);
      }
    }
  }
  __device__ inline Frag<NS> frag(int s) const {
    if constexpr (NS == 1) {
      Frag<NS> f;
      f.s[0] = r[s][0];
      return f;
    } else {
      float v[8];
      floats(s, v);
      return to_frag<NS>(v);
    }
  }
};

// host check of both directions
scn_status check_cross(const char* who, int32_t type, int64_t nq, int64_t nk, int32_t batch,
                       const int32_t* q_ranges, const int32_t* k_ranges, int32_t D, int32_t Hq,
                       int32_t Hk, float scale);

}  // namespace scn
