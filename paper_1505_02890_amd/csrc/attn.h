// What the attention kernels share: element types, the samples' ranges and the
// visible sites, and operand tiles in LDS.
//
// Products run on v_mfma_f32_32x32x16_bf16.  Lane (n, h), n = lane % 32,
// h = lane / 32, holds row n of A (column n of B) at the eight reduction steps
// 8 h + j, and of the result column n, rows 8 (r / 4) + 4 h + r % 4 in register r.
// A result with keys along its rows is therefore an operand of the next product
// (eight registers are one of its operands) as it stands, if the other operand
// takes its reduction in the same order: step j of half h is row
// 8 (j / 4) + 4 h + j % 4.  Transposed LDS reads (ds_read_b64_tr_b16: four lanes
// by four give a lane one column of four rows) deliver that order.
// bf16 operands are multiplied as they are (NS = 1); floats are split into three
// bf16 planes whose six products stand for one (NS = 3, split.h).
#pragma once

#include <type_traits>

#include "scn_internal.h"
#include "split.h"

namespace scn {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

template <int NS>
struct Elem;
template <>
struct Elem<1> {
  typedef uint16_t T;
  static constexpr int BYTES = 2;
  static __device__ inline float get(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ inline uint16_t put(float v) { return (uint16_t)cvt2_bf16(v, v); }
};
template <>
struct Elem<3> {
  typedef float T;
  static constexpr int BYTES = 4;
  static __device__ inline float get(float v) { return v; }
  static __device__ inline float put(float v) { return v; }
};

// channel c of head h of row t at p[t * row + h * head + c]
template <class T>
struct Heads {
  T* p;
  int64_t row, head;
};

// The rows of one tile of a sample.  Tiles of `rows` rows are numbered over all samples
// with tile_start(b) = ranges[b] / rows + b, which leaves room for each sample's
// tiles whatever the lengths, so a grid of n / rows + B blocks covers them and no
// length has to be known on the host (blocks past a sample's rows leave at once).
// Bounds are clamped to [0, n], so that a bad range reads no row outside the arrays.
// Where only samples of more than `cut` rows have tiles, min(b, ranges[b] / cut) stands for
// b: it grows by one at each such sample, but the tiles are n / rows + min(B, n / cut).
struct Span {
  int64_t base;  // first row of the sample
  int m;         // its rows
  int first;     // first row of the tile, counted in the sample
  int sample;
};
__device__ inline int64_t range_at(const int32_t* ranges, int b, int64_t n) {
  const int64_t v = ranges[b];
  return v < 0 ? 0 : v > n ? n : v;
}
__device__ inline int tile_start(int base, int b, int rows, int cut) {
  return base / rows + (cut ? min(b, base / cut) : b);
}
// Every lane of the wave takes part.  The sample is the last b with
// tile_start(b) <= tile, found 64 ways at a time.
__device__ inline Span find_span(const int32_t* ranges, int batch, int64_t n, int tile, int rows,
                                 int cut = 0) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = batch;
  while (len > 1) {
    const int stride = (len + 63) >> 6, b = lo + lane * stride;
    const bool below = lane * stride < len &&
                       tile_start((int)range_at(ranges, b, n), b, rows, cut) <= tile;
    const int c = __popcll(__ballot(below));
    const int step = max(c - 1, 0) * stride;
    lo += step;
    len = min(stride, len - step);
  }
  Span s;
  s.sample = __builtin_amdgcn_readfirstlane(lo);
  const int base = __builtin_amdgcn_readfirstlane((int)range_at(ranges, s.sample, n));
  const int end = __builtin_amdgcn_readfirstlane((int)range_at(ranges, s.sample + 1, n));
  s.base = base;
  s.m = max(0, end - base);
  const int64_t local = tile - tile_start(base, s.sample, rows, cut);
  s.first = local < 0 || local * rows >= s.m ? s.m : (int)(local * rows);
  return s;
}

// Which sites see which: i sees j if j <= i + right and (j >= i - left or
// j < sinks); left and right are clamped to n by the host (unbounded: n).
struct Window {
  int left, right, sinks;
  __device__ inline int lo(int i) const { return max(0, i - left); }
  __device__ inline int hi(int i, int m) const { return min(m - 1, i + right); }
};

template <int NS>
struct Frag {
  v4u s[NS];
};

template <int NS>
__device__ inline v16f mma(const Frag<NS>& a, const Frag<NS>& b, v16f c) {
  if constexpr (NS == 1) {
    return mfma_bf16(a.s[0], b.s[0], c);
  } else {
#pragma unroll
    for (int p = 0; p < SPLIT_PROD; ++p) c = mfma_bf16(a.s[split_a(p)], b.s[split_b(p)], c);
    return c;
  }
}

// eight floats along the reduction to an operand
template <int NS>
__device__ inline Frag<NS> to_frag(const float (&v)[8]) {
  Frag<NS> f;
  if constexpr (NS == 1) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f.s[0][j] = cvt2_bf16(v[2 * j], v[2 * j + 1]);
  } else {
    const Frag3 t = split8(v);
#pragma unroll
    for (int p = 0; p < 3; ++p) f.s[p] = t.s[p];
  }
  return f;
}

__device__ inline v16f zero16() {
  v16f z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}

// maximum, NaN if either is (v_maximum3_f32 takes two at a time; fmaxf would quiet each
// operand first)
__device__ inline float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// sum and maximum of the lanes n of both halves, in both
__device__ inline float both_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline float both_larger(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return larger(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A tile of ROWS rows by DP channels in LDS: NS planes of bf16, rows of DP, in pieces
// of 16 bytes.  Piece c of row r lies at c ^ twist(r), so that eight rows' pieces of
// one column (ds_read_b128) and four rows' 64 bytes (the transposed reads) each fall
// on all 64 banks once.
template <int NS, int DP, int ROWS>
struct Tile {
  static constexpr int PLANE = ROWS * DP * 2;
  static constexpr int BYTES = NS * PLANE;
  static __device__ inline int twist(int r) {
    if constexpr (DP == 64) return ((r >> 1) & 1) << 2 | ((r >> 2) & 1) << 1 | ((r >> 3) & 1);
    if constexpr (DP == 128) return (r & 3) << 2 | ((r >> 2) & 3);
    return (r >> 2) & 3;
  }
  static __device__ inline int at(int row, int piece) {
    return row * (DP * 2) + ((piece ^ twist(row)) << 4);
  }
  // A lane's places in the tile, kept in registers: r[s] of rows n, channels
  // 16 s + 8 h + 0..7; c[d] and c[d] + 8 rows of the transposed reads.
  struct Lane {
    int r[DP / 16], c[DP / 32][2];
    __device__ inline Lane(int lane) {
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) r[s] = at(lane & 31, 2 * s + (lane >> 5));
      const int row = ((lane >> 5) << 2) + ((lane & 15) >> 2);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        const int ch = d * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
        c[d][0] = at(row, ch >> 3) + (ch & 7) * 2;
        c[d][1] = at(row + 8, ch >> 3) + (ch & 7) * 2;
      }
    }
  };
  // rows r0 + n, channels 16 s + 8 h + 0..7 (r0 a multiple of 32)
  static __device__ inline Frag<NS> rows(const char* t, const Lane& l, int r0, int s) {
    Frag<NS> f;
#pragma unroll
    for (int p = 0; p < NS; ++p)
      f.s[p] = *reinterpret_cast<const v4u*>(t + l.r[s] + r0 * (DP * 2) + p * PLANE);
    return f;
  }
  // channels 32 d + n along the operand's rows; its reduction over the tile's rows
  // r0 + 8 (j / 4) + 4 h + j % 4 (r0 a multiple of 16)
  static __device__ inline Frag<NS> cols(char* t, const Lane& l, int r0, int d) {
    Frag<NS> f;
    typedef __attribute__((address_space(3))) v4s lds4;
#pragma unroll
    for (int p = 0; p < NS; ++p) {
      char* const o = t + r0 * (DP * 2) + p * PLANE;
      const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(o + l.c[d][0]));
      const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(o + l.c[d][1]));
      const v2u x = __builtin_bit_cast(v2u, a), y = __builtin_bit_cast(v2u, b);
      f.s[p] = v4u{x[0], x[1], y[0], y[1]};
    }
    return f;
  }
};

// A tile on its way from memory to LDS, through registers of THREADS threads.  Rows past
// those that there are read as zero (the buffer's bounds), and pieces past channel D are
// the row's first again: what they put into the tile is multiplied with the other
// operand's zeros, or becomes channels past D of a result.
template <int NS, int DP, int ROWS, int THREADS>
struct Stage {
  typedef typename Elem<NS>::T T;
  static constexpr int EPP = 16 / Elem<NS>::BYTES;  // elements of a 16-byte piece
  static constexpr int PIECES = DP / EPP;
  static constexpr int N = (ROWS * PIECES + THREADS - 1) / THREADS;
  static constexpr bool EVEN = ROWS * PIECES % THREADS == 0;
  v4u r[N];
  // `off`: where the thread's pieces lie, bytes from the tile's first row (rows lie at
  // most 2^24 bytes apart)
  static __device__ inline void places(uint32_t (&off)[N], int64_t stride, int D, int tid) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int y = tid + u * THREADS, c = y % PIECES * EPP;
      off[u] = ((uint32_t)(y / PIECES % ROWS) * (uint32_t)stride + (c < D ? c : 0)) * sizeof(T);
    }
  }
  // up to `rows` >= 1 rows from row j of p (p, j and rows uniform)
  __device__ inline void load(const T* p, int64_t stride, const uint32_t (&off)[N], int j, int rows,
                              int D) {
    T* const q = const_cast<T*>(p) + (uint64_t)(uint32_t)j * (uint32_t)stride;
    const uint32_t bytes = ((uint32_t)(min(rows, ROWS) - 1) * (uint32_t)stride + D) * sizeof(T);
    const __amdgpu_buffer_rsrc_t b = __builtin_amdgcn_make_buffer_rsrc(q, 0, (int)bytes, 0x00020000);
#pragma unroll
    for (int u = 0; u < N; ++u)
      r[u] = __builtin_amdgcn_raw_buffer_load_b128(b, (int)off[u], 0, 0);
  }
  __device__ inline void store(char* t, int tid) const {
    typedef Tile<NS, DP, ROWS> L;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int y = tid + u * THREADS, row = y / PIECES, c = y % PIECES;
      if (!EVEN && y >= ROWS * PIECES) continue;
      if constexpr (NS == 1) {
        *reinterpret_cast<v4u*>(t + L::at(row, c)) = r[u];
      } else {
        uint32_t h[2], m[2], l[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
          split2(__uint_as_float(r[u][2 * j]), __uint_as_float(r[u][2 * j + 1]), h[j], m[j], l[j]);
        char* const o = t + L::at(row, c >> 1) + (c & 1) * 8;
        *reinterpret_cast<v2u*>(o) = v2u{h[0], h[1]};
        *reinterpret_cast<v2u*>(o + L::PLANE) = v2u{m[0], m[1]};
        *reinterpret_cast<v2u*>(o + 2 * L::PLANE) = v2u{l[0], l[1]};
      }
    }
  }
};

// one lane's row of an operand, channels 16 s + 8 h + 0..7 (zero past D)
template <int NS>
__device__ inline Frag<NS> load_frag(const typename Elem<NS>::T* row, int s, int D, int lane) {
  const int c = 16 * s + 8 * (lane >> 5);
  Frag<NS> f;
#pragma unroll
  for (int p = 0; p < NS; ++p) f.s[p] = v4u{0, 0, 0, 0};
  if (c < D) {
    if constexpr (NS == 1) {
      f.s[0] = *reinterpret_cast<const v4u*>(row + c);
    } else {
      float v[8];
      const v4f a = *reinterpret_cast<const v4f*>(row + c);
      const v4f b = *reinterpret_cast<const v4f*>(row + c + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = a[j];
        v[4 + j] = b[j];
      }
      f = to_frag<NS>(v);
    }
  }
  return f;
}

// A result column's channels 32 db + 8 (r / 4) + 4 h + r % 4, times f, to a row
template <int NS>
__device__ inline void store_cols(typename Elem<NS>::T* row, const v16f& v, float f, int db, int D,
                                  int lane) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int c = 32 * db + 8 * g + 4 * (lane >> 5);
    if (c >= D) continue;
    if constexpr (NS == 1) {
      *reinterpret_cast<v2u*>(row + c) = v2u{cvt2_bf16(v[4 * g] * f, v[4 * g + 1] * f),
                                             cvt2_bf16(v[4 * g + 2] * f, v[4 * g + 3] * f)};
    } else {
      *reinterpret_cast<v4f*>(row + c) =
          v4f{v[4 * g] * f, v[4 * g + 1] * f, v[4 * g + 2] * f, v[4 * g + 3] * f};
    }
  }
}

// eight channels of a row
template <int NS>
__device__ inline void load8(const typename Elem<NS>::T* p, float (&v)[8]) {
  if constexpr (NS == 1) {
    const v4u a = *reinterpret_cast<const v4u*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(a[j] << 16);
      v[2 * j + 1] = __uint_as_float(a[j] & 0xffff0000u);
    }
  } else {
    const v4f a = *reinterpret_cast<const v4f*>(p), b = *reinterpret_cast<const v4f*>(p + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = a[j];
      v[4 + j] = b[j];
    }
  }
}
// (past: not to be kept in the caches)
template <int NS>
__device__ inline void store8(typename Elem<NS>::T* p, const float (&v)[8], bool past) {
  auto put = [&](auto x, auto* q) {
    if (past)
      __builtin_nontemporal_store(x, q);
    else
      *q = x;
  };
  if constexpr (NS == 1) {
    v4u a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = cvt2_bf16(v[2 * j], v[2 * j + 1]);
    put(a, reinterpret_cast<v4u*>(p));
  } else {
    put(v4f{v[0], v[1], v[2], v[3]}, reinterpret_cast<v4f*>(p));
    put(v4f{v[4], v[5], v[6], v[7]}, reinterpret_cast<v4f*>(p + 4));
  }
}

// sum over aligned groups of LP <= 16 lanes, in all of them
template <int LP>
__device__ inline float group_sum(float v) {
  auto add = [&](auto perm) {
    v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), decltype(perm)::value, 0xf,
                                                  0xf, true));
  };
  if constexpr (LP >= 2) add(std::integral_constant<int, 0xb1>());   // lanes 1, 0, 3, 2
  if constexpr (LP >= 4) add(std::integral_constant<int, 0x4e>());   // 2, 3, 0, 1
  if constexpr (LP >= 8) add(std::integral_constant<int, 0x141>());  // mirrored in eights
  if constexpr (LP >= 16) add(std::integral_constant<int, 0x140>()); // in sixteens
  return v;
}

__device__ inline bool finite16(const v16f& v) {
  float s = 0.f;  // 0 * x is NaN for infinities and NaN
#pragma unroll
  for (int r = 0; r < 16; ++r) s = fmaf(v[r], 0.f, s);
  return s == 0.f;
}

// Whether the row's results (v times f, f positive; both halves hold some) are so small that their
// fp32 operands may have lost low parts (split.h): nothing of 2^-95 or more, and not zero.
// A larger one says that what was lost is below 2^-38 of it, as scores say of theirs:
// they are off by what is below 2^-133 of a query, times its keys.
template <int N>
__device__ inline bool tiny(const v16f (&v)[N], float f) {
  float m = 0.f;
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) m = larger(m, fabsf(v[d][r]));
  m = both_larger(m);
  return m > 0.f && m * f < 0x1p-95f;
}

__device__ inline float wave_max(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ inline float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// dot product of two rows of D channels, in order (redone rows)
template <int NS>
__device__ inline float row_dot(const typename Elem<NS>::T* a, const typename Elem<NS>::T* b,
                                int D) {
  float s = 0.f;
  for (int c = 0; c < D; c += 8) {
    float x[8], y[8];
    load8<NS>(a + c, x);
    load8<NS>(b + c, y);
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(x[j], y[j], s);
  }
  return s;
}

// The softmax of one row that a wave forms again: the largest score and the sum of the
// weights, a share of the keys per lane.  (A score of NaN makes the sum NaN, and so the
// weights.)
struct RowSum {
  float top = -INFINITY, sum = 0.f;
  __device__ inline void add(float s) {
    if (s > top) {
      sum *= expf(top - s);
      top = s;
    }
    sum += s == -INFINITY ? 0.f : expf(s - top);
  }
  // all lanes' shares, in all of them
  __device__ inline void join() {
    const float t = wave_max(top);
    sum = wave_sum(top == -INFINITY ? sum : sum * expf(top - t));
    top = t;
  }
  __device__ inline float weight(float s) const { return expf(s - top) / sum; }
};

// A sum of weights is at least 1, and below 2^8 times the keys, but for the rounding of
// the maximum: the weights are exp2(s c - m) with m rounded and s c not, so all of a row's
// are off by the same factor, which leaves o and lse as they are.  From scores of 2^31 on
// that factor passes 2^64, and weights end at 0 or infinity; sums outside these bounds say
// so (what is lost within them is below 2^-86 of the sum).
constexpr float SUM_LEAST = 0x1p-40f, SUM_MOST = 0x1p60f;
// A sum that is NaN, and not for scores' size: a score is NaN, and so is all that the
// row gives.  (Of fp32 operands, and beside zeros that fill a head's last tile, an
// infinite operand may be the reason.)
__device__ inline bool nan_score(float top, float sum) {
  return sum != sum && (fabsf(top) < 0x1p30f || top == -INFINITY);
}
// The backward passes form weights from log sums in fp32, each off by up to some 2^-23 of its
// log sum relatively.  Rows past this bound (2^-10 so) are formed again, from their own
// scores' maximum and sum.
constexpr float LSE_MOST = 8192.f;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr int ATTN_D = 128;                     // most channels of a head
constexpr int64_t ATTN_ROWS = int64_t(1) << 30; // most rows of a call

// host checks shared by the entry points; messages name the call
scn_status check_heads(const char* who, const char* name, const scn_heads* h, int type);
scn_status check_attn(const char* who, int32_t type, int64_t n, int32_t batch,
                      const int32_t* ranges, int32_t D, int32_t Hq, int32_t Hk, float scale);
template <class T>
Heads<T> view(const scn_heads* h) {
  return h ? Heads<T>{static_cast<T*>(h->p), h->row, h->head} : Heads<T>{nullptr, 0, 0};
}
inline int bound(int64_t w, int64_t n) { return (int)(w < 0 || w > n ? n : w); }

}  // namespace scn
