// Cross attention, forward: a sample's queries over the states of the same sample, which are
// rows of other arrays and of another number.
//
// As attn_fwd.hip's without a window: one pass over the keys with the running maximum and
// sum of the softmax, S^T = K Q^T and O^T += V^T P^T, 32 tile rows a wave (cross.h).  Where
// there are few queries the keys are split over blocks, whose outputs, maxima and sums a
// second kernel joins in order.
//
// Long samples wait in turn to issue and for data (one sample of 16,384 rows and states, 2 bf16
// heads of 128: 302 us, 910 TFLOP/s, and 16 for the join), few rows for memory: 128 streams of
// 2,000 states, 35 us and 7 for the join; one row over 262,144 states, 4 heads of 32 bf16, 30 and
// 6.
#include <cmath>

#include "cross.h"

namespace scn {
namespace {

template <int NS>
struct CrossArgs {
  typedef typename Elem<NS>::T T;
  Deal deal;  // tiles of queries, parts of their keys
  int D, group;
  int repeat;  // tiles of queries that a work is, where the keys are few
  Heads<const T> q, k, v;
  Heads<T> o;
  float* lse;   // [Hq][nq] or null
  float scale;  // positive
  float* part;  // [Hq][nq][parts][D], then [Hq][nq][parts][2]: maximum, sum
  __device__ inline int64_t at(int64_t row, int h) const { return h * deal.tiles.n + row; }
  __device__ inline float* out(int64_t at, int s) const {
    return part + (at * deal.parts.most + s) * D;
  }
  __device__ inline float* sums(int64_t at, int s) const {
    return part + deal.tiles.n * deal.Hk * group * deal.parts.most * D +
           (at * deal.parts.most + s) * 2;
  }
};

// One row once more in fp32, term by term, as attn_fwd.hip's fwd_row: over the `cnt` >= 1 keys
// from k0 on.
template <int NS>
__device__ inline void cross_row(const CrossArgs<NS>& a, int64_t row, int h, int64_t k0, int cnt) {
  typedef Elem<NS> E;
  const int lane = threadIdx.x & 63;
  const auto* const q = a.q.p + row * a.q.row + h * a.q.head;
  const auto* const k = a.k.p + k0 * a.k.row + (h / a.group) * a.k.head;
  const auto* const v = a.v.p + k0 * a.v.row + (h / a.group) * a.v.head;
  auto score = [&](int x) { return row_dot<NS>(q, k + x * a.k.row, a.D) * a.scale; };
  RowSum r;
  for (int x = lane; x < cnt; x += 64) r.add(score(x));
  r.join();
  float o0 = 0.f, o1 = 0.f;
  for (int x0 = 0; x0 < cnt; x0 += 64) {
    const float p = x0 + lane < cnt ? r.weight(score(x0 + lane)) : 0.f;
    for (int y = 0; y < min(64, cnt - x0); ++y) {
      const auto* const vj = v + (x0 + y) * a.v.row;
      const float py = __shfl(p, y);
      if (lane < a.D) o0 = fmaf(py, E::get(vj[lane]), o0);
      if (64 + lane < a.D) o1 = fmaf(py, E::get(vj[64 + lane]), o1);
    }
  }
  auto* const o = a.o.p + row * a.o.row + h * a.o.head;
  if (lane < a.D) o[lane] = E::put(o0);
  if (64 + lane < a.D) o[64 + lane] = E::put(o1);
  if (a.lse && lane == 0) a.lse[a.at(row, h)] = r.top + logf(r.sum);
}

// m, l: maximum (log 2) and sum of the terms that an output holds; f, f2: what both outputs are
// taken times.  A side without terms has m = -inf and l = 0.
__device__ inline void join(float& m, float& l, float m2, float l2, float& f, float& f2) {
  const float t = fmaxf(m, m2), b = t == -INFINITY ? 0.f : t;
  f = __builtin_amdgcn_exp2f(m - b);
  f2 = __builtin_amdgcn_exp2f(m2 - b);
  l = l * f + l2 * f2;
  m = t;
}
// A wave's 32 tile rows from `first` on: out, or to the workspace where the keys are split, and
// those that attn.h's bounds do not serve once more.
template <int NS, int DP>
__device__ __forceinline__ void finish(const CrossArgs<NS>& a, const Work& w, const v16f (&O)[DP / 32],
                              float top, float sum, int first, bool mine, int64_t row, int h) {
  const int lane = threadIdx.x & 63, half = lane >> 5;
  if (w.parts > 1) {
    if (mine) {
      const int64_t to = a.at(row, h);
      float* const o = a.out(to, w.part);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) store_cols<3>(o, O[d], 1.f, d, a.D, lane);
      if (half == 0) {
        float* const s = a.sums(to, w.part);
        s[0] = top;
        s[1] = sum;
      }
    }
    return;
  }
  // (no key seen: nothing, and a log sum of -inf)
  const float inv = w.mo > 0 ? 1.f / sum : 0.f;
  bool fine = fabsf(top) < INFINITY && sum > SUM_LEAST && sum < SUM_MOST;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) fine &= finite16(O[d]);
  if constexpr (NS == 3) fine &= !tiny(O, inv);
  if constexpr (NS == 1) fine |= a.D == DP && nan_score(top, sum);  // NaN, as it stands
  if (mine) {
    auto* const o = a.o.p + row * a.o.row + h * a.o.head;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) store_cols<NS>(o, O[d], inv, d, a.D, lane);
    if (a.lse && half == 0) a.lse[a.at(row, h)] = (top + log2f(sum)) * LN2;
  }
  // rows that attn.h's bounds do not serve (SUM_LEAST, tiny)
  const uint64_t bad = __ballot(mine && !fine && w.mo > 0);
  uint32_t rows = (uint32_t)bad | (uint32_t)(bad >> 32);
  for (; rows; rows &= rows - 1) {
    const int x = first + __builtin_ctz(rows);
    cross_row<NS>(a, w.base + x / a.group, w.hk * a.group + x % a.group, w.other, w.mo);
  }
}

// QW waves of 32 tile rows by KW groups that share out the keys of a tile, 32 NB each
template <int NS, int DP, int QW_, int KW_, int NB_>
struct Shape {
  static constexpr int QW = QW_, KW = KW_, NB = NB_, QB = 32 * QW, NT = 64 * QW * KW;
  static constexpr int KT = 32 * NB * KW;
  typedef Tile<NS, DP, KT> L;
  static constexpr int BUF = 2 * L::BYTES;       // keys and values
  static constexpr int JOIN = DP / 32 * 16 + 2;  // floats a lane hands over
  static constexpr size_t SMEM = std::max<size_t>(2 * BUF, (size_t)QW * (KW - 1) * JOIN * 256);
  static_assert(SMEM <= 160 * 1024, "LDS of a compute unit");
};

// FEW: a work is several tiles of queries in turn
template <int NS, int DP, int QW, int KW, int NB, bool FEW>
__global__ void __launch_bounds__(64 * QW * KW, NS == 3 && DP > 96 ? 1 : 2)
    cross_fwd_kernel(CrossArgs<NS> a) {
  typedef Shape<NS, DP, QW, KW, NB> X;
  typedef typename X::L L;
  constexpr int QB = X::QB, KT = X::KT, NT = X::NT;
  constexpr bool TWO = NS == 1 && FEW;  // few keys: low_part
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kw = KW == 1 ? 0 : wave / QW;
  const float c2 = a.scale * LOG2E;
  typedef Stage<NS, DP, KT, NT> St;
  uint32_t ko[St::N], vo[St::N];
  St::places(ko, a.k.row, a.D, tid);
  St::places(vo, a.v.row, a.D, tid);
  const typename L::Lane at(lane);

  const Work w = a.deal.find(blockIdx.x);
  if (w.first >= w.m) return;
  const int mk = w.mo, hk = w.hk;
  const int64_t k0 = w.other;
  Frag<NS> Q[DP / 16];
  v16f O[DP / 32];
  // the running maximum (log 2) and sum of this half's keys, as in attn_fwd.hip
  float top, base, limit, sum;

  // the block's tiles of the sample's keys
  const int nt = (mk + KT - 1) / KT, per = (nt + w.parts - 1) / w.parts;
  const int t0 = min(nt, w.part * per), t1 = min(nt, t0 + per);
  const auto* const kp = a.k.p + k0 * a.k.row + hk * a.k.head;
  const auto* const vp = a.v.p + k0 * a.v.row + hk * a.v.head;
  St sk, sv;
  auto fetch = [&](int t) {
    sk.load(kp, a.k.row, ko, t * KT, mk - t * KT, a.D);
    sv.load(vp, a.v.row, vo, t * KT, mk - t * KT, a.D);
  };
  auto put = [&](int t) {
    char* const b = smem + ((t - t0) & 1) * X::BUF;
    sk.store(b, tid);
    sv.store(b + L::BYTES, tid);
  };
  auto take = [&](int t) {
    constexpr int M = NB;
    const int left = mk - t * KT - kw * 32 * NB;  // keys from the wave's first on
    char* const kt = smem + ((t - t0) & 1) * X::BUF + kw * 32 * NB * DP * 2;
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
    if (left < 32 * M) {
#pragma unroll
      for (int b = 0; b < M; ++b)
#pragma unroll
        for (int x = 0; x < 16; ++x)
          S[b][x] = 32 * b + 8 * (x / 4) + 4 * half + x % 4 < left ? S[b][x] : -INFINITY;
    }
    float mx[M];
#pragma unroll
    for (int b = 0; b < M; ++b) {
      mx[b] = larger(S[b][0], S[b][1]);
#pragma unroll
      for (int x = 2; x < 16; ++x) mx[b] = larger(mx[b], S[b][x]);
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
        for (int x = 0; x < 16; ++x) O[d][x] *= f;
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
      for (int x = 0; x < 16; ++x) {
        S[b][x] = __builtin_amdgcn_exp2f(fmaf(S[b][x], c2, -base));
        sum += S[b][x];
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = S[b][8 * s + j];
        const Frag<NS> P = to_frag<NS>(p);
        Frag<NS> low;
        if constexpr (TWO) low = low_part(p, P);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
          const Frag<NS> W = EARLY ? V[b][s][d] : L::cols(vt, at, 32 * b + 16 * s, d);
          if constexpr (TWO) O[d] = mma<NS>(W, low, O[d]);
          O[d] = mma<NS>(W, P, O[d]);
        }
      }
    }
  };
  // Works of several tiles load the next one's queries while they take one.
  constexpr bool PRE = FEW && DP <= 64;
  Ahead<NS, PRE ? DP : 16> next;
  auto ahead = [&](int first) {
    const int r = min(first + (wave - kw * QW) * 32 + n32, w.m - 1);
    next.load(a.q.p + (w.base + r / a.group) * a.q.row + (hk * a.group + r % a.group) * a.q.head, a.D,
              lane);
  };
  auto sweep = [&](int first, bool stage) {
    const int r = first + (wave - kw * QW) * 32 + n32;  // the lane's tile row
    const bool mine = r < w.m;
    const int rr = min(r, w.m - 1);
    const int64_t row = w.base + rr / a.group;
    const int h = hk * a.group + rr % a.group;
    if constexpr (PRE) {
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) Q[s] = next.frag(s);
      ahead(first + QB);
    } else {
      const auto* const q = a.q.p + row * a.q.row + h * a.q.head;
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) Q[s] = load_frag<NS>(q, s, a.D, lane);
    }
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) O[d] = zero16();
    top = limit = -INFINITY;
    base = sum = 0.f;
    // While a tile is taken, the next one goes from registers to the other buffer and the
    // one after that is loaded.  Two tiles or fewer stay for the block's next queries.
    if (stage && t0 < t1) {
      fetch(t0);
      put(t0);
      if (t0 + 1 < t1) fetch(t0 + 1);
      __syncthreads();
    }
    for (int t = t0; t < t1; ++t) {
      if (stage) {
        if (t + 1 < t1) put(t + 1);
        if (t + 2 < t1) fetch(t + 2);
      }
      take(t);
      if (stage) __syncthreads();
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
          for (int e = 0; e < 16; ++e) o[(d * 16 + e) * 64] = O[d][e];
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
          for (int e = 0; e < 16; ++e) O[d][e] = O[d][e] * f + o[(d * 16 + e) * 64] * f2;
      }
    }
    finish<NS, DP>(a, w, O, top, sum, first + wave * 32, mine, row, h);
  };
  if constexpr (!FEW) {
    sweep(w.first, true);
  } else {
    const int end = min(w.m, w.first + QB * a.repeat);
    if constexpr (PRE) ahead(w.first);
    for (int first = w.first; first < end; first += QB)
      sweep(first, first == w.first || t1 - t0 > 2);
  }
}

// Few bf16 rows: one tile of 32 a block, whose waves take 32 keys at a time each, through its own
// part of LDS and without a barrier (attn_step.hip), up to AHEAD tiles ahead in registers.  The
// weights keep 16 bits (low_part): the matrix cores wait for memory here.
template <int DP>
struct Thin {
  static constexpr int WAVES = 4, NT = 64 * WAVES, AHEAD = DP <= 64 ? 2 : 1;
  typedef Tile<1, DP, 32> L;
  static constexpr int JOIN = DP / 32 * 16 + 2;
  static constexpr int SMEM = std::max(WAVES * 2 * L::BYTES, (WAVES - 1) * JOIN * 256);
};
template <int DP>
__global__ void __launch_bounds__(Thin<DP>::NT, 2) cross_thin_kernel(CrossArgs<1> a) {
  typedef Thin<DP> X;
  typedef typename X::L L;
  typedef Stage<1, DP, 32, 64> St;
  constexpr int WAVES = X::WAVES, AHEAD = X::AHEAD;
  __shared__ __align__(16) char smem[X::SMEM];
  const Work w = a.deal.find(blockIdx.x);
  if (w.first >= w.m) return;
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool mine = w.first + n32 < w.m;
  const int rr = min(w.first + n32, w.m - 1), h = w.hk * a.group + rr % a.group;
  const int64_t row = w.base + rr / a.group;
  const float c2 = a.scale * LOG2E;
  Frag<1> Q[DP / 16];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s)
    Q[s] = load_frag<1>(a.q.p + row * a.q.row + h * a.q.head, s, a.D, lane);
  v16f O[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) O[d] = zero16();
  float top = -INFINITY, base = 0.f, sum = 0.f;

  const int nt = (w.mo + 31) / 32, per = (nt + w.parts - 1) / w.parts;
  const int t1 = min(nt, (w.part + 1) * per);
  const uint16_t* const kp = a.k.p + w.other * a.k.row + w.hk * a.k.head;
  const uint16_t* const vp = a.v.p + w.other * a.v.row + w.hk * a.v.head;
  St sk[AHEAD], sv[AHEAD];
  uint32_t ko[St::N], vo[St::N];
  St::places(ko, a.k.row, a.D, lane);
  St::places(vo, a.v.row, a.D, lane);
  const typename L::Lane at(lane);
  char* const kt = smem + wave * 2 * L::BYTES;
  char* const vt = kt + L::BYTES;
  auto fetch = [&](int u, int t) {
    if (t < t1) {
      sk[u].load(kp, a.k.row, ko, t * 32, w.mo - t * 32, a.D);
      sv[u].load(vp, a.v.row, vo, t * 32, w.mo - t * 32, a.D);
    }
  };
  auto take = [&](int u, int t) {
    sk[u].store(kt, lane);
    sv[u].store(vt, lane);
    fetch(u, t + AHEAD * WAVES);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    v16f S = zero16();
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) S = mma<1>(L::rows(kt, at, 0, c), Q[c], S);
    const int left = w.mo - t * 32;
    if (left < 32)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        S[r] = 8 * (r / 4) + 4 * half + r % 4 < left ? S[r] : -INFINITY;
    float m = larger(S[0], S[1]);
#pragma unroll
    for (int r = 2; r < 16; ++r) m = larger(m, S[r]);
    m = both_larger(m) * c2;
    if (__ballot(m > top + 8.f)) {
      const float next = fmaxf(top, m);
      const float f = next == top ? 1.f : __builtin_amdgcn_exp2f(top - next);
      top = next;
      base = next == -INFINITY ? 0.f : next;
      sum *= f;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[d][r] *= f;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      S[r] = __builtin_amdgcn_exp2f(fmaf(S[r], c2, -base));
      sum += S[r];
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = S[8 * e + j];
      const Frag<1> P = to_frag<1>(p), low = low_part(p, P);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        const Frag<1> V = L::cols(vt, at, 16 * e, d);
        O[d] = mma<1>(V, low, O[d]);
        O[d] = mma<1>(V, P, O[d]);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  const int t0 = w.part * per + wave;
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) fetch(u, t0 + u * WAVES);
  for (int t = t0; t < t1; t += AHEAD * WAVES) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (t + u * WAVES < t1) take(u, t + u * WAVES);
  }
  sum = both_sum(sum);
  // the waves, joined in order
  float* const x = reinterpret_cast<float*>(smem) + lane;
  __syncthreads();
  if (wave > 0) {
    float* const o = x + (wave - 1) * X::JOIN * 64;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[(d * 16 + r) * 64] = O[d][r];
    o[(X::JOIN - 2) * 64] = top;
    o[(X::JOIN - 1) * 64] = sum;
  }
  __syncthreads();
  if (wave > 0) return;
  for (int g = 0; g < WAVES - 1; ++g) {
    const float* const o = x + g * X::JOIN * 64;
    float f, f2;
    join(top, sum, o[(X::JOIN - 2) * 64], o[(X::JOIN - 1) * 64], f, f2);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) O[d][r] = O[d][r] * f + o[(d * 16 + r) * 64] * f2;
  }
  finish<1, DP>(a, w, O, top, sum, w.first, mine, row, h);
}

// Few fp32 rows, on the vector unit (attn_step.hip): LP lanes hold a key's channels, eight a lane,
// straight from memory, and take GC tile rows while its row is in registers.  Each group of
// LP lanes keeps a running maximum, sum and output of its own, which join within the wave
// and the block.
constexpr int FEW_NT = 256;
template <int LP, int GC>
__global__ void __launch_bounds__(FEW_NT) cross_few_kernel(CrossArgs<3> a) {
  constexpr int U = 4;                    // keys of a lane group in flight
  constexpr int KW = 64 / LP;             // keys of a wave at once
  constexpr int KB = KW * (FEW_NT / 64);  // ... of the block
  __shared__ float red[FEW_NT / 64][GC][LP * 8 + 2];
  __shared__ bool bad[GC];
  const Work w = a.deal.find(blockIdx.x);
  if (w.first >= w.m) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = lane % LP * 8;
  const bool on = c < a.D;
  const int nh = min(GC, w.m - w.first);
  const int per = (w.mo + w.parts - 1) / w.parts;
  const int x0 = min(w.mo, w.part * per), x1 = min(w.mo, x0 + per);
  const float* const k = a.k.p + w.other * a.k.row + w.hk * a.k.head + c;
  const float* const v = a.v.p + w.other * a.v.row + w.hk * a.v.head + c;
  auto row = [&](int g) { return w.base + (w.first + g) / a.group; };
  auto head = [&](int g) { return w.hk * a.group + (w.first + g) % a.group; };

  // (maxima of unscaled scores: equal scores have equal weights, however large)
  const float c2 = a.scale * LOG2E;
  float q[GC][8], o[GC][8], m[GC], l[GC];
#pragma unroll
  for (int g = 0; g < GC; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) q[g][j] = o[g][j] = 0.f;
    if (on && g < nh) load8<3>(a.q.p + row(g) * a.q.row + head(g) * a.q.head + c, q[g]);
  }
  for (int x = x0 + wave * KW + lane / LP; x - lane / LP < x1; x += KB * U) {
    float kk[U][8], vv[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int y = x + u * KB;
#pragma unroll
      for (int j = 0; j < 8; ++j) kk[u][j] = vv[u][j] = 0.f;
      if (on && y < x1) {
        load8<3>(k + y * a.k.row, kk[u]);
        load8<3>(v + y * a.v.row, vv[u]);
      }
    }
#pragma unroll
    for (int g = 0; g < GC; ++g) {
      float sc[U], top = m[g];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float d = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) d = fmaf(q[g][j], kk[u][j], d);
        d = group_sum<LP>(d);
        sc[u] = x + u * KB < x1 ? d : -INFINITY;
        top = fmaxf(top, sc[u]);
      }
      const float b = top == -INFINITY ? 0.f : top;
      const float f = __builtin_amdgcn_exp2f((m[g] - b) * c2);
      m[g] = top;
      l[g] *= f;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[g][j] *= f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float e = __builtin_amdgcn_exp2f((sc[u] - b) * c2);
        l[g] += e;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[g][j] = fmaf(e, vv[u][j], o[g][j]);
      }
    }
  }
  // the lane groups of the wave, then the waves
#pragma unroll
  for (int g = 0; g < GC; ++g) {
    m[g] *= c2;
#pragma unroll
    for (int d = LP; d < 64; d <<= 1) {
      float f, f2;
      join(m[g], l[g], __shfl_xor(m[g], d), __shfl_xor(l[g], d), f, f2);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[g][j] = o[g][j] * f + __shfl_xor(o[g][j], d) * f2;
    }
    if (lane < LP) {
#pragma unroll
      for (int j = 0; j < 8; ++j) red[wave][g][c + j] = o[g][j];
      red[wave][g][LP * 8] = m[g];
      red[wave][g][LP * 8 + 1] = l[g];
    }
  }
  if (tid < GC) bad[tid] = false;
  __syncthreads();
  for (int i = tid; i < nh * a.D; i += FEW_NT) {
    const int g = i / a.D, ch = i % a.D;
    float mm = red[0][g][LP * 8], ll = red[0][g][LP * 8 + 1], y = red[0][g][ch], f, f2;
#pragma unroll
    for (int u = 1; u < FEW_NT / 64; ++u) {
      join(mm, ll, red[u][g][LP * 8], red[u][g][LP * 8 + 1], f, f2);
      y = y * f + red[u][g][ch] * f2;
    }
    const int64_t at = a.at(row(g), head(g));
    if (w.parts > 1) {
      a.out(at, w.part)[ch] = y;
      if (ch == 0) {
        a.sums(at, w.part)[0] = mm;
        a.sums(at, w.part)[1] = ll;
      }
    } else {
      y = w.mo > 0 ? y / ll : 0.f;
      a.o.p[row(g) * a.o.row + head(g) * a.o.head + ch] = y;
      if (a.lse && ch == 0) a.lse[at] = (mm + log2f(ll)) * LN2;
      if (w.mo > 0 && !(fabsf(y) < INFINITY)) bad[g] = true;
    }
  }
  if (w.parts > 1) return;
  __syncthreads();
  for (int g = wave; g < nh; g += FEW_NT / 64)
    if (bad[g]) cross_row<3>(a, row(g), head(g), w.other, w.mo);
}

// The parts of the rows' outputs, joined in order: `deal.rows` tile rows a block, four channels
// a thread, and what threads are left share out the parts.
template <int NS>
__global__ void __launch_bounds__(256) cross_join_kernel(CrossArgs<NS> a, Parts parts) {
  __shared__ float x[256][6];
  __shared__ bool bad[128];
  // (the works of unsplit tiles, and the parts beside them)
  const Work w = a.deal.find(blockIdx.x);
  const int n = parts.of(w.mo);
  if (w.first >= w.m || n == 1) return;
  const int lanes = a.D >> 2, tid = threadIdx.x;
  const int rows = a.deal.rows, slices = 256 / (lanes * rows);
  const int c = tid % lanes * 4, r = tid / lanes % rows, sl = tid / (lanes * rows);
  const bool on = sl < slices && w.first + r < w.m;
  const int rr = min(w.first + r, w.m - 1), h = w.hk * a.group + rr % a.group;
  const int64_t row = w.base + rr / a.group, at = h * a.deal.tiles.n + row;
  const float* const out = a.part + at * parts.most * a.D + c;
  const float* const sums =
      a.part + a.deal.tiles.n * a.deal.Hk * a.group * parts.most * a.D + at * parts.most * 2;
  float top = -INFINITY, sum = 0.f;
  v4f v = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](float t, float s, v4f o) {
    const float now = fmaxf(top, t), base = now == -INFINITY ? 0.f : now;
    const float f = __builtin_amdgcn_exp2f(top - base), g = __builtin_amdgcn_exp2f(t - base);
    top = now;
    sum = sum * f + s * g;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = v[j] * f + o[j] * g;
  };
  if (on) {
    const int per = (n + slices - 1) / slices, s1 = min(n, (sl + 1) * per);
    for (int s0 = sl * per; s0 < s1; s0 += 4) {
      float t[4], u[4];
      v4f o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int s = min(s0 + j, s1 - 1);
        t[j] = sums[2 * s];
        u[j] = sums[2 * s + 1];
        o[j] = *reinterpret_cast<const v4f*>(out + (int64_t)s * a.D);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (s0 + j < s1) add(t[j], u[j], o[j]);
    }
  }
  if (tid < 128) bad[tid] = false;
  if (slices > 1) {
    if (on && sl > 0) {
      x[tid][0] = top;
      x[tid][1] = sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[tid][2 + j] = v[j];
    }
    __syncthreads();
    if (on && sl == 0)
      for (int s = 1; s < slices; ++s) {
        const float* const y = x[s * lanes * rows + tid];
        add(y[0], y[1], v4f{y[2], y[3], y[4], y[5]});
      }
  } else {
    __syncthreads();
  }
  if (on && sl == 0) {
    const float inv = 1.f / sum;
    bool fine = fabsf(top) < INFINITY && sum > SUM_LEAST && sum < SUM_MOST;
    bool large = false, any = false;  // (fp32: attn.h's tiny, of these channels)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] *= inv;
      fine &= fabsf(v[j]) < INFINITY;
      large |= fabsf(v[j]) >= 0x1p-95f;
      any |= v[j] != 0.f;
    }
    if constexpr (NS == 3) fine &= large || !any;
    if constexpr (NS == 1) fine |= a.D % 32 == 0 && nan_score(top, sum);
    auto* const o = a.o.p + row * a.o.row + h * a.o.head + c;
    if constexpr (NS == 1)
      *reinterpret_cast<v2u*>(o) = v2u{cvt2_bf16(v[0], v[1]), cvt2_bf16(v[2], v[3])};
    else
      *reinterpret_cast<v4f*>(o) = v;
    if (a.lse && c == 0) a.lse[at] = (top + log2f(sum)) * LN2;
    if (!fine) bad[r] = true;
  }
  __syncthreads();
  for (int i = tid >> 6; i < min(rows, w.m - w.first); i += 4)
    if (bad[i]) {
      const int y = w.first + i;
      cross_row<NS>(a, w.base + y / a.group, w.hk * a.group + y % a.group, w.other, w.mo);
    }
}

// The kernel's shape, the parts of the keys and the tiles of queries that a block takes, by rules
// on sizes alone (the lengths lie on the device): tile rows and keys of a mean sample, blocks.
// Both sides of each rule, as whole calls in us, the rule's first:
//  - Few fp32 rows, on the vector unit: 64 samples of 4,096 states, 2 key heads of 64, 1 tile row
//    a sample 57 and 94 in tiles, 8 rows 70 and 92, 16 rows 93 in tiles and 97.
//  - Few bf16 rows, waves that take tiles alone: 16 samples of 4,096 states, 2 heads of 32, 16
//    rows 16 and 18 in the general kernel, 32 rows 16.5 and 18.5, 64 rows 17.8 and 18.6.
//  - bf16 to 64 channels, two waves of queries by two of keys below 512 blocks: 8 samples of 2,000
//    states, 4 heads of 64, 4,000 rows 88 (four waves) and 108; around the border the other side
//    wins, 1,000 rows 47 and 42, 2,000 rows 66 and 56.
//  - fp32 to 64 channels, two by two for 64 rows or fewer: 64 rows on 4,000 states, 4 heads of 32,
//    24 and 29; four waves by two groups below 512 blocks: 1,000 rows on 400 states 18 and 25, on
//    4,000 states 129 and 113; four waves alone from there: 4,000 rows on 400 states 47 and 58.
//  - bf16 past 64 channels, four by two below 512 blocks: 500 rows on 400 states, 4 heads of 128,
//    16 and 16, on 4,000 states 71 and 58; four alone from there: 2,000 rows on 400 states 27 and
//    34.
//  - Few keys that stay in LDS for several tiles of queries: 120,011 rows of 4 fp32 heads on 2 of
//    32 over 40 states each, 56 and 85 loading them for each.
//  - Keys in parts: 2,000 rows of 8 samples on 7,500 states, 4 heads of 64 bf16, 179 and 210 in
//    one part; 64 rows of 4 samples on 50,000, 4 heads of 32 fp32, 69 and 904.
// A batch whose samples are far from their mean is cut as if they were not: one of 256 streams with
// a million states, the others with ten, takes 5 ms.
struct CrossPlan {
  int qw, kw, nb;  // qw 0: cross_few_kernel of nb tile rows
  int repeat;      // tiles of a work where the keys are few, or 0
  Parts parts;
};
CrossPlan plan(int type, int64_t nq, int64_t nk, int batch, int D, int Hk, int group) {
  CrossPlan p;
  const int used = (int)std::max<int64_t>(1, std::min<int64_t>(batch, nq));  // samples with queries
  const int64_t rows = ceil_div(nq * group, used), keys = nk / used;
  auto blocks = [&](int qb) { return used * ceil_div(rows, qb) * Hk; };
  const bool bf16 = type == SCN_BF16;
  if (!bf16 && rows <= 8)
    p = {0, 0, rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8, 0, {}};
  else if (rows <= 32 && bf16)
    p = {1, 4, 1, 0, {}};
  else if (bf16 && D <= 64)
    p = blocks(128) < 512 && keys > 128 ? CrossPlan{2, 2, 2, 0, {}} : CrossPlan{4, 1, 2, 0, {}};
  else if (!bf16 && D <= 64 && rows <= 64 && keys > 64)
    p = {2, 2, 1, 0, {}};
  else if ((bf16 || D <= 64) && (blocks(128) < 512 || (!bf16 && D > 32)) && keys > 64)
    p = {4, 2, 1, 0, {}};
  else
    p = {4, 1, 1, 0, {}};
  // Two blocks a CU, which is what resides; four where there are nearly as many anyway, for
  // samples' lengths differ.
  const int64_t n = p.qw ? blocks(32 * p.qw) : blocks(p.nb);
  p.parts = cut(n, n >= 256 && p.qw > 1 ? 1024 : 512, keys, p.qw ? 512 : 256, used);
  if (p.kw == 1 && keys <= 64 * p.nb)
    p.repeat = (int)std::max<int64_t>(1, std::min<int64_t>(8, n / FEW_BLOCKS));
  return p;
}

scn_status too_many() {
  set_error("scn_cross_attn_fwd: more than 2^31 blocks of rows and heads");
  return SCN_ERR_OVERFLOW;
}

template <int NS, int DP, int QW, int KW, int NB, bool FEW = false>
scn_status launch(CrossArgs<NS> a, const CrossPlan& p, hipStream_t st) {
  typedef Shape<NS, DP, QW, KW, NB> X;
  static LdsLimit limit;
  auto fn = cross_fwd_kernel<NS, DP, QW, KW, NB, FEW>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, X::SMEM)) return rc;
  a.deal.rows = X::QB * std::max(1, a.repeat);
  const int64_t blocks = a.deal.blocks();
  if (blocks > INT32_MAX) return too_many();
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(X::NT), X::SMEM, st, a);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}

template <int LP>
scn_status launch_few(CrossArgs<3> a, const CrossPlan& p, hipStream_t st) {
  a.deal.rows = p.nb;
  const int64_t blocks = a.deal.blocks();
  if (blocks > INT32_MAX) return too_many();
  const dim3 grid((unsigned)blocks), block(FEW_NT);
  if (p.nb == 1) hipLaunchKernelGGL((cross_few_kernel<LP, 1>), grid, block, 0, st, a);
  if (p.nb == 2) hipLaunchKernelGGL((cross_few_kernel<LP, 2>), grid, block, 0, st, a);
  if (p.nb == 4) hipLaunchKernelGGL((cross_few_kernel<LP, 4>), grid, block, 0, st, a);
  if (p.nb == 8) hipLaunchKernelGGL((cross_few_kernel<LP, 8>), grid, block, 0, st, a);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}
scn_status launch_few(const CrossArgs<3>& a, const CrossPlan& p, hipStream_t st) {
  if (a.D <= 8) return launch_few<1>(a, p, st);
  if (a.D <= 16) return launch_few<2>(a, p, st);
  if (a.D <= 32) return launch_few<4>(a, p, st);
  if (a.D <= 64) return launch_few<8>(a, p, st);
  return launch_few<16>(a, p, st);
}

template <int DP>
scn_status launch_thin(CrossArgs<1> a, const CrossPlan& p, hipStream_t st) {
  a.deal.rows = 32;
  const int64_t blocks = a.deal.blocks();
  if (blocks > INT32_MAX) return too_many();
  hipLaunchKernelGGL(cross_thin_kernel<DP>, dim3((unsigned)blocks), dim3(Thin<DP>::NT), 0, st, a);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}

template <int NS, int DP>
scn_status launch(const CrossArgs<NS>& a, const CrossPlan& p, hipStream_t st) {
  if constexpr (NS == 1)
    if (p.qw == 1) return launch_thin<DP>(a, p, st);
  if constexpr (NS == 1 && DP <= 64) {
    if (p.qw == 2) return launch<NS, DP, 2, 2, 2>(a, p, st);
    if (p.repeat) return launch<NS, DP, 4, 1, 2, true>(a, p, st);
    return launch<NS, DP, 4, 1, 2>(a, p, st);
  } else {
    if constexpr (NS == 3 && DP <= 64)
      if (p.qw == 2) return launch<NS, DP, 2, 2, 1>(a, p, st);
    if constexpr (NS == 1 || DP <= 64)
      if (p.kw == 2) return launch<NS, DP, 4, 2, 1>(a, p, st);
    if (p.repeat || (NS == 3 && DP == 64)) return launch<NS, DP, 4, 1, 1, true>(a, p, st);
    if constexpr (!(NS == 3 && DP == 64)) return launch<NS, DP, 4, 1, 1>(a, p, st);
  }
}

template <int NS>
scn_status run(const CrossArgs<NS>& a, const CrossPlan& p, hipStream_t st) {
  scn_status rc = SCN_OK;
  bool few = false;
  if constexpr (NS == 3)
    if ((few = p.qw == 0)) rc = launch_few(a, p, st);
  if (!few)
    rc = a.D <= 32   ? launch<NS, 32>(a, p, st)
         : a.D <= 64 ? launch<NS, 64>(a, p, st)
         : a.D <= 96 ? launch<NS, 96>(a, p, st)
                     : launch<NS, 128>(a, p, st);
  if (rc || p.parts.most == 1) return rc;
  // as many rows a block as leave the card some thousand blocks, of at most 256 threads
  CrossArgs<NS> j = a;
  j.deal.parts = Parts{1, INT32_MAX};
  j.deal.near = false;
  j.deal.rows = 1;
  while (j.deal.rows * 2 * (a.D / 4) <= 256 &&
         a.deal.tiles.n * a.group * a.deal.Hk / (j.deal.rows * 2) >= 1024)
    j.deal.rows *= 2;
  hipLaunchKernelGGL(cross_join_kernel<NS>, dim3((unsigned)j.deal.blocks()), dim3(256), 0,
                     st, j, p.parts);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}

size_t part_bytes(const CrossPlan& p, int64_t nq, int Hq, int D) {
  return p.parts.most > 1 ? (size_t)(nq * Hq * p.parts.most * (D + 2)) * 4 : 0;
}

template <int NS>
CrossArgs<NS> make(int64_t nq, int64_t nk, int batch, const int32_t* qr, const int32_t* kr, int D,
                   int Hq, int Hk, const scn_heads* q, const scn_heads* k, const scn_heads* v,
                   float scale, const scn_heads* o, float* lse, const CrossPlan& p, void* ws) {
  typedef typename Elem<NS>::T T;
  const Deal deal{{qr, nq, Hq / Hk}, {kr, nk, 1}, batch, 0, Hk, p.parts,
                  p.qw <= 1 && D * sizeof(T) < 128};
  return CrossArgs<NS>{deal, D, Hq / Hk, p.repeat, view<const T>(q), view<const T>(k),
                       view<const T>(v), view<T>(o), lse, scale, static_cast<float*>(ws)};
}

}  // namespace

scn_status check_cross(const char* who, int32_t type, int64_t nq, int64_t nk, int32_t batch,
                       const int32_t* q_ranges, const int32_t* k_ranges, int32_t D, int32_t Hq,
                       int32_t Hk, float scale) {
  if (scn_status rc = check_attn(who, type, std::min(nq, nk), batch, q_ranges, D, Hq, Hk, scale))
    return rc;
  if (!k_ranges) {
    set_error("%s: no ranges of the keys", who);
    return SCN_ERR_INVALID;
  }
  if (nq > ATTN_ROWS / (Hq / Hk) || nk > ATTN_ROWS) {
    set_error("%s: more than 2^30 keys, or rows of queries times heads on a key head", who);
    return SCN_ERR_OVERFLOW;
  }
  return SCN_OK;
}

}  // namespace scn

using namespace scn;

extern "C" {

size_t scn_cross_attn_fwd_workspace_bytes(int32_t type, int64_t nq, int64_t nk, int32_t batch,
                                          int32_t D, int32_t Hq, int32_t Hk) {
  if ((type != SCN_F32 && type != SCN_BF16) || nq < 1 || nk < 0 || nk > ATTN_ROWS || batch < 1 ||
      D < 1 || D > ATTN_D || Hk < 1 || Hq < 1 || Hq % Hk != 0 || nq > ATTN_ROWS / (Hq / Hk))
    return 0;
  return part_bytes(plan(type, nq, nk, batch, D, Hk, Hq / Hk), nq, Hq, D);
}

scn_status scn_cross_attn_fwd(int32_t type, int64_t nq, int64_t nk, int32_t batch,
                              const int32_t* q_ranges, const int32_t* k_ranges, int32_t D,
                              int32_t Hq, int32_t Hk, const scn_heads* q, const scn_heads* k,
                              const scn_heads* v, float scale, const scn_heads* o, float* lse,
                              void* ws, size_t ws_bytes, hipStream_t st) {
  clear_error();
  const char* const who = "scn_cross_attn_fwd";
  if (scn_status rc = check_cross(who, type, nq, nk, batch, q_ranges, k_ranges, D, Hq, Hk, scale))
    return rc;
  if (nq == 0) return SCN_OK;
  if (scn_status rc = check_heads(who, "q", q, type)) return rc;
  if (scn_status rc = check_heads(who, "o", o, type)) return rc;
  if (nk > 0) {
    if (scn_status rc = check_heads(who, "k", k, type)) return rc;
    if (scn_status rc = check_heads(who, "v", v, type)) return rc;
  }
  const CrossPlan p = plan(type, nq, nk, batch, D, Hk, Hq / Hk);
  const size_t need = part_bytes(p, nq, Hq, D);
  if (need && (!ws || (reinterpret_cast<uintptr_t>(ws) & 15) != 0 || ws_bytes < need)) {
    set_error("%s: workspace missing, misaligned or too small", who);
    return SCN_ERR_WORKSPACE;
  }
  if (type == SCN_BF16)
    return run<1>(make<1>(nq, nk, batch, q_ranges, k_ranges, D, Hq, Hk, q, k, v, scale, o, lse, p, ws),
                  p, st);
  return run<3>(make<3>(nq, nk, batch, q_ranges, k_ranges, D, Hq, Hk, q, k, v, scale, o, lse, p, ws),
                p, st);
}

}  // extern "C"
