// Attention within samples, forward: one pass over the keys that a tile of queries
// sees, with the running maximum and sum of the softmax.
//
// A block holds 32 QW consecutive queries of one sample and head, 32 a wave, and takes
// their keys in tiles through two LDS buffers, one tile ahead in registers: first the
// sinks below the window, then the window from its first key.  Per 32 keys and wave
// S^T = K Q^T has a query in each lane (its keys along the registers), so the maximum and
// the sum stay in the lane but for one exchange with the other half, and P^T goes on into
// O^T += V^T P^T as it is.  bf16: P is rounded to bf16 for that product, which leaves o at
// most 1.4 times as far off as its own rounding; the sum has the unrounded terms.  fp32:
// each operand in three bf16 parts, six products.
//
// 32 x 32 scores of 64 channels cost some 74 vector instructions, 400 cycles, beside 256 on
// the matrix cores.  All pairs of 16,384 rows, 4 heads of 64 channels, bf16: 330 us, 834
// TFLOP/s; the vector unit issues in 55% of the cycles, the matrix cores are busy in 36%, the
// waves wait to issue for 34% of theirs, and neither a third wave, wave priorities nor another
// order of the instructions gain.  Windows of 1025 rows (60,007 rows, 4 heads): 110 us, 570
// TFLOP/s, vector unit 44%, matrix cores 23%; the waves wait for loads and barriers for 28%
// of their cycles, to issue for 27%.  Causal samples (32,001 rows of 16 samples): 74 us, 33% and
// 19%, one wave a SIMD in the mean where two fit, for a sample's last tiles see the most keys
// and come last.
#include <cmath>

#include "attn.h"

namespace scn {
namespace {

template <int NS>
struct FwdArgs {
  typedef typename Elem<NS>::T T;
  int64_t n;
  int batch, D, Hq, group;
  const int32_t* ranges;
  Heads<const T> q, k, v;
  Heads<T> o;
  float* lse;
  float scale;  // positive
  Window w;
};

// One row once more in fp32, over the keys that it sees and no others: the maximum and
// the sum first, a key per lane, then the values by weights that are divided already
// (terms before the division may pass fp32's range where the result does not), channels
// along the lanes.
template <int NS>
__device__ inline void fwd_row(const FwdArgs<NS>& a, const Span& sp, int h, int i) {
  typedef Elem<NS> E;
  const int lane = threadIdx.x & 63;
  const auto* const q = a.q.p + (sp.base + i) * a.q.row + h * a.q.head;
  const auto* const k = a.k.p + sp.base * a.k.row + (h / a.group) * a.k.head;
  const auto* const v = a.v.p + sp.base * a.v.row + (h / a.group) * a.v.head;
  const int lo = a.w.lo(i), hi = a.w.hi(i, sp.m), ns = min(a.w.sinks, lo);
  const int cnt = ns + hi - lo + 1;  // the keys: [0, ns), then [lo, hi]
  auto key = [&](int x) { return x < ns ? x : lo + x - ns; };
  auto score = [&](int x) { return row_dot<NS>(q, k + key(x) * a.k.row, a.D) * a.scale; };
  RowSum r;
  for (int x = lane; x < cnt; x += 64) r.add(score(x));
  r.join();
  float o0 = 0.f, o1 = 0.f;
  for (int x0 = 0; x0 < cnt; x0 += 64) {
    const float p = x0 + lane < cnt ? r.weight(score(x0 + lane)) : 0.f;
    for (int y = 0; y < min(64, cnt - x0); ++y) {
      const auto* const vj = v + key(x0 + y) * a.v.row;
      const float py = __shfl(p, y);
      if (lane < a.D) o0 = fmaf(py, E::get(vj[lane]), o0);
      if (64 + lane < a.D) o1 = fmaf(py, E::get(vj[64 + lane]), o1);
    }
  }
  auto* const o = a.o.p + (sp.base + i) * a.o.row + h * a.o.head;
  if (lane < a.D) o[lane] = E::put(o0);
  if (64 + lane < a.D) o[64 + lane] = E::put(o1);
  if (a.lse && lane == 0) a.lse[h * a.n + sp.base + i] = r.top + logf(r.sum);
}

// QW waves of 32 queries by KW groups that share out the keys of a tile, 32 NB each
template <int NS, int DP, int QW_, int KW_, int NB_>
struct Shape {
  static constexpr int QW = QW_, KW = KW_, NB = NB_, QB = 32 * QW, NT = 64 * QW * KW;
  static constexpr int KT = 32 * NB * KW;
  typedef Tile<NS, DP, KT> L;
  static constexpr int BUF = 2 * L::BYTES;       // keys and values
  static constexpr int JOIN = DP / 32 * 16 + 2;  // floats a lane hands over
  static constexpr size_t SMEM = std::max<size_t>(2 * BUF, (size_t)QW * (KW - 1) * JOIN * 256);
};

// Two waves a SIMD leave each 256 registers, which all but fp32 heads of more than 96
// channels do with.  (With 512 the compiler put fp32 sums of 96 channels into accumulation
// registers, copied them out at the loop's head, and read the last product's too early there.)
template <int NS, int DP, int QW, int KW, int NB>
__global__ void __launch_bounds__(64 * QW * KW, NS == 3 && DP > 96 ? 1 : 2)
    attn_fwd_kernel(FwdArgs<NS> a) {
  typedef Shape<NS, DP, QW, KW, NB> X;
  typedef typename X::L L;
  constexpr int QB = X::QB, KT = X::KT, NT = X::NT;
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kw = KW == 1 ? 0 : wave / QW;
  const int h = blockIdx.x % a.Hq;
  const Span sp = find_span(a.ranges, a.batch, a.n, blockIdx.x / a.Hq, QB);
  if (sp.first >= sp.m) return;
  // the wave's queries (i1 < i0 past the sample's rows) and the lane's
  const int i0 = sp.first + (wave - kw * QW) * 32, i1 = min(i0 + 31, sp.m - 1);
  const int i = min(i0 + n32, sp.m - 1);
  const float c2 = a.scale * LOG2E;

  Frag<NS> Q[DP / 16];
  {
    const auto* const q = a.q.p + (sp.base + i) * a.q.row + h * a.q.head;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) Q[s] = load_frag<NS>(q, s, a.D, lane);
  }
  v16f O[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) O[d] = zero16();
  // The maximum of the scores (log 2) and the sum, of this half's keys.  The maximum
  // moves only when a score passes it by 2^8 (`limit`, unscaled): until then the terms
  // stay below 2^8 and the sums far from fp32's range.
  float top = -INFINITY, base = 0.f, limit = -INFINITY, sum = 0.f;

  // The block's keys: the sinks [0, ns), then the window [lo, hi], in tiles of KT; and
  // what some query of the wave and all of them see of the window
  const int lo = a.w.lo(sp.first), hi = a.w.hi(min(sp.first + QB, sp.m) - 1, sp.m);
  const int ns = min(a.w.sinks, lo), nst = (ns + KT - 1) / KT, nt = nst + (hi - lo + KT) / KT;
  const int wl = lo < a.w.sinks ? lo : a.w.lo(i0), wh = a.w.hi(i1, sp.m);
  const int al = a.w.lo(i0 + 31), ah = a.w.hi(i0, sp.m);
  const auto* const kp = a.k.p + sp.base * a.k.row + (h / a.group) * a.k.head;
  const auto* const vp = a.v.p + sp.base * a.v.row + (h / a.group) * a.v.head;
  typedef Stage<NS, DP, KT, NT> St;
  St sk, sv;
  uint32_t ko[St::N], vo[St::N];
  St::places(ko, a.k.row, a.D, tid);
  St::places(vo, a.v.row, a.D, tid);
  const typename L::Lane at(lane);
  auto first_key = [&](int t) { return t < nst ? t * KT : lo + (t - nst) * KT; };
  auto fetch = [&](int t) {
    const int j = first_key(t), rows = (t < nst ? ns : hi + 1) - j;
    sk.load(kp, a.k.row, ko, j, rows, a.D);
    sv.load(vp, a.v.row, vo, j, rows, a.D);
  };
  auto put = [&](int t) {
    sk.store(smem + (t & 1) * X::BUF, tid);
    sv.store(smem + (t & 1) * X::BUF + L::BYTES, tid);
  };
  // the wave's keys of tile t
  auto take = [&](int t) {
    constexpr int M = NB;
    const int j0 = first_key(t) + kw * 32 * NB;
    const bool sink = t < nst;
    char* const kt = smem + (t & 1) * X::BUF + kw * 32 * NB * DP * 2;
    char* const vt = kt + L::BYTES;
    constexpr bool EARLY = NS == 1 || DP == 32;  // values read before they are needed
    Frag<NS> V[M][2][DP / 32];
    v16f S[M];
    {
      Frag<NS> K[M][DP / 16];
#pragma unroll
      for (int b = 0; b < M; ++b)
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) K[b][s] = L::rows(kt, at, 32 * b, s);
      if constexpr (EARLY) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int d = 0; d < DP / 32; ++d) V[0][s][d] = L::cols(vt, at, 16 * s, d);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int b = 0; b < M; ++b) {
        S[b] = zero16();
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) S[b] = mma<NS>(K[b][s], Q[s], S[b]);
      }
    }
    if (sink ? j0 + 32 * M > ns : j0 < al || j0 + 32 * M - 1 > ah) {
      const int l = (sink ? 0 : a.w.lo(i)) - j0 - 4 * half;
      const int u = (sink ? ns - 1 : a.w.hi(i, sp.m)) - j0 - 4 * half;
      const int z = a.w.sinks - j0 - 4 * half;
      if (sink || j0 >= a.w.sinks) {
#pragma unroll
        for (int b = 0; b < M; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int e = 32 * b + 8 * (r / 4) + r % 4;
            S[b][r] = ((e >= l) & (e <= u)) ? S[b][r] : -INFINITY;
          }
      } else {
#pragma unroll
        for (int b = 0; b < M; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int e = 32 * b + 8 * (r / 4) + r % 4;
            S[b][r] = ((e <= u) & ((e >= l) | (e < z))) ? S[b][r] : -INFINITY;
          }
      }
    }
    float mx[M];
#pragma unroll
    for (int b = 0; b < M; ++b) {
      mx[b] = larger(S[b][0], S[b][1]);
#pragma unroll
      for (int r = 2; r < 16; ++r) mx[b] = larger(mx[b], S[b][r]);
    }
    const float m = both_larger(M == 2 ? larger(mx[0], mx[M - 1]) : mx[0]);
    if (__ballot(m > limit)) {
      const float now = fmaxf(top, m * c2);
      const float f = now == top ? 1.f : __builtin_amdgcn_exp2f(top - now);
      top = now;
      base = now == -INFINITY ? 0.f : now;
      limit = (now + 8.f) / c2;
      sum *= f;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[d][r] *= f;
    }
#pragma unroll
    for (int b = 0; b < M; ++b) {
      if constexpr (EARLY && M == 2)
        if (b == 1) {
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) V[1][s][d] = L::cols(vt, at, 32 + 16 * s, d);
        }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        S[b][r] = __builtin_amdgcn_exp2f(fmaf(S[b][r], c2, -base));
        sum += S[b][r];
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = S[b][8 * s + j];
        const Frag<NS> P = to_frag<NS>(p);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
          O[d] = mma<NS>(EARLY ? V[b][s][d] : L::cols(vt, at, 32 * b + 16 * s, d), P, O[d]);
      }
    }
  };
  // While a tile is taken, the next one goes from registers to the other buffer and the
  // one after that is loaded.
  auto pass = [&](int t) {
    if (t + 1 < nt) put(t + 1);
    if (t + 2 < nt) fetch(t + 2);
  };
  // The wave takes the tiles [0, e0) of sinks and [s1, e1) of its window, and passes the
  // others on.  (A branch round `take` would have the sums copied at its end.)
  auto place = [&](int x) { return nst + max(0, x - kw * 32 * NB) / KT; };
  const int some = i0 <= i1 && wh - lo >= kw * 32 * NB;  // if it sees any of its window's keys
  const int e0 = i0 <= i1 ? nst : 0;
  const int s1 = some ? place(wl - lo) : nt, e1 = some ? place(wh - lo) + 1 : nt;
  fetch(0);
  put(0);
  if (nt > 1) fetch(1);
  __syncthreads();
  int t = 0;
  for (int seg = 0; seg < 2; ++seg) {
    const int s = seg ? s1 : 0, e = seg ? e1 : e0;
    for (; t < s; ++t) {
      pass(t);
      __syncthreads();
    }
    for (; t < e; ++t) {
      pass(t);
      take(t);
      __syncthreads();
    }
  }
  for (; t < nt; ++t) {
    pass(t);
    __syncthreads();
  }
  sum = both_sum(sum);
  if constexpr (KW > 1) {
    // the groups' shares of the keys, joined in order
    float* const x = reinterpret_cast<float*>(smem) + lane;
    if (kw > 0) {
      float* const o = x + (wave - QW) * X::JOIN * 64;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[(d * 16 + r) * 64] = O[d][r];
      o[(X::JOIN - 2) * 64] = top;
      o[(X::JOIN - 1) * 64] = sum;
    }
    __syncthreads();
    if (kw > 0) return;
    for (int g = 1; g < KW; ++g) {
      const float* const o = x + ((g - 1) * QW + wave) * X::JOIN * 64;
      const float top2 = o[(X::JOIN - 2) * 64], now = fmaxf(top, top2);
      const float base = now == -INFINITY ? 0.f : now;
      const float f = __builtin_amdgcn_exp2f(top - base), f2 = __builtin_amdgcn_exp2f(top2 - base);
      top = now;
      sum = sum * f + o[(X::JOIN - 1) * 64] * f2;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[d][r] = O[d][r] * f + o[(d * 16 + r) * 64] * f2;
    }
  }
  const float inv = 1.f / sum;
  bool fine = fabsf(top) < INFINITY && sum > SUM_LEAST && sum < SUM_MOST;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) fine &= finite16(O[d]);
  if constexpr (NS == 3) fine &= !tiny(O, inv);
  if constexpr (NS == 1) fine |= a.D == DP && nan_score(top, sum);  // NaN, as it stands
  const bool mine = i0 + n32 < sp.m;
  if (mine) {
    auto* const o = a.o.p + (sp.base + i) * a.o.row + h * a.o.head;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) store_cols<NS>(o, O[d], inv, d, a.D, lane);
    if (a.lse && half == 0) a.lse[h * a.n + sp.base + i] = (top + log2f(sum)) * LN2;
  }
  // A term that is infinite or NaN spoils sums it does not enter (0 times it is NaN), and
  // scores past 2^31 lose theirs
  const uint64_t bad = __ballot(mine && !fine);
  uint32_t rows = (uint32_t)bad | (uint32_t)(bad >> 32);
  while (rows) {
    const int r = __builtin_ctz(rows);
    rows &= rows - 1;
    fwd_row<NS>(a, sp, h, i0 + r);
  }
}

template <int NS, int DP, int QW, int KW, int NB>
scn_status launch(const FwdArgs<NS>& a, hipStream_t st) {
  typedef Shape<NS, DP, QW, KW, NB> X;
  static LdsLimit limit;
  auto fn = attn_fwd_kernel<NS, DP, QW, KW, NB>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, X::SMEM)) return rc;
  const int64_t blocks = (a.n / X::QB + a.batch) * a.Hq;
  if (blocks > INT32_MAX) {
    set_error("scn_attn_fwd: more than 2^31 blocks of rows and heads");
    return SCN_ERR_OVERFLOW;
  }
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(X::NT), X::SMEM, st, a);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}

// The shapes (waves of queries, groups of keys, blocks of 32 keys), by measurement (us):
//  - Few blocks of 128 queries leave compute units idle: groups share out the keys (4 x
//    4000 rows, 4 heads of 64, bf16: 19 against 22; 16,384 rows, 2 heads of 128: 297
//    against 361).  Many do better without (60,007 rows, 4 heads of 64: 110 against 149;
//    32,001 rows, 2 heads of 128: 79 against 94; fp32, 34,567 rows, 4 heads of 32: 51
//    against 72), but for fp32 heads of 64, whose operands leave a SIMD one wave (20,000
//    rows of 4 heads: 224 against 302).
//  - bf16 up to 64 channels has the registers for 64 keys at a time (32,001 rows of 4
//    heads: 76 against 83).  Narrower heads do better in small blocks, two waves and 32
//    keys (160,003 rows of 8 heads of 32, windows of 257 rows: 144 against 169).
template <int NS, int DP>
scn_status launch(const FwdArgs<NS>& a, hipStream_t st) {
  const int64_t blocks = (a.n / 128 + a.batch) * a.Hq;
  if constexpr (NS == 1 && DP <= 64) {
    if (blocks < 512) return launch<NS, DP, 2, 2, 2>(a, st);
    if constexpr (DP <= 32) return launch<NS, DP, 2, 1, 1>(a, st);
    return launch<NS, DP, 4, 1, 2>(a, st);
  } else {
    if constexpr (NS == 1 || DP <= 64)
      if (blocks < 512 || (NS == 3 && DP == 64)) return launch<NS, DP, 4, 2, 1>(a, st);
    return launch<NS, DP, 4, 1, 1>(a, st);
  }
}

template <int NS>
scn_status run(const FwdArgs<NS>& a, hipStream_t st) {
  if (a.D <= 32) return launch<NS, 32>(a, st);
  if (a.D <= 64) return launch<NS, 64>(a, st);
  if (a.D <= 96) return launch<NS, 96>(a, st);
  return launch<NS, 128>(a, st);
}

}  // namespace

scn_status check_attn(const char* who, int32_t type, int64_t n, int32_t batch,
                      const int32_t* ranges, int32_t D, int32_t Hq, int32_t Hk, float scale) {
  if (type != SCN_F32 && type != SCN_BF16) {
    set_error("%s: unknown type %d", who, type);
    return SCN_ERR_INVALID;
  }
  if (n < 0 || batch < 1 || !ranges || D < 1 || Hk < 1 || Hq < 1 || Hq % Hk != 0) {
    set_error("%s: bad size, no ranges, or Hq not a multiple of Hk", who);
    return SCN_ERR_INVALID;
  }
  if (!(scale > 0.f) || !std::isfinite(scale)) {
    set_error("%s: scale must be positive and finite", who);
    return SCN_ERR_INVALID;
  }
  if (D % 8 != 0 || D > ATTN_D) {
    set_error("%s: heads of %d channels (multiples of 8 up to %d are supported)", who, D, ATTN_D);
    return SCN_ERR_UNSUPPORTED;
  }
  if (n > ATTN_ROWS) {
    set_error("%s: more than 2^30 rows", who);
    return SCN_ERR_OVERFLOW;
  }
  return SCN_OK;
}

}  // namespace scn

using namespace scn;

extern "C" scn_status scn_attn_fwd(int32_t type, int64_t n, int32_t batch, const int32_t* ranges,
                                   int32_t D, int32_t Hq, int32_t Hk, const scn_heads* q,
                                   const scn_heads* k, const scn_heads* v, float scale,
                                   int64_t left, int64_t right, int64_t sinks, const scn_heads* o,
                                   float* lse, hipStream_t st) {
  clear_error();
  const char* const who = "scn_attn_fwd";
  if (scn_status rc = check_attn(who, type, n, batch, ranges, D, Hq, Hk, scale)) return rc;
  if (sinks < 0) {
    set_error("%s: negative number of sinks", who);
    return SCN_ERR_INVALID;
  }
  if (n == 0) return SCN_OK;
  if (scn_status rc = check_heads(who, "q", q, type)) return rc;
  if (scn_status rc = check_heads(who, "k", k, type)) return rc;
  if (scn_status rc = check_heads(who, "v", v, type)) return rc;
  if (scn_status rc = check_heads(who, "o", o, type)) return rc;
  const Window w{bound(left, n), bound(right, n), bound(sinks, n)};
  if (type == SCN_BF16) {
    typedef uint16_t T;
    return run<1>(FwdArgs<1>{n, batch, D, Hq, Hq / Hk, ranges, view<const T>(q), view<const T>(k),
                             view<const T>(v), view<T>(o), lse, scale, w}, st);
  }
  typedef float T;
  return run<3>(FwdArgs<3>{n, batch, D, Hq, Hq / Hk, ranges, view<const T>(q), view<const T>(k),
                           view<const T>(v), view<T>(o), lse, scale, w}, st);
}
