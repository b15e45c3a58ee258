// Cross attention, forward: a sample's queries over the states of the same sample, which are
// rows of other arrays and of another number.
//
// As attn_fwd.hip's without a window: one pass over the keys with the running maximum and
// sum of the softmax, S^T = K Q^T and O^T += V^T P^T, 32 tile rows a wave (cross.h).  Where
// there are few queries the keys are split over blocks, whose outputs, maxima and sums a
// second kernel joins in order.
#include <cmath>

#include "cross.h"

#ifndef REPEAT_BLOCKS
#define REPEAT_BLOCKS 768
#endif
#ifndef WANT
#define WANT 1024
#endif
#ifndef LEAST
#define LEAST 512
#endif
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
__global__ void __launch_bounds__(64 * QW * KW, DP > 96 && (NS == 3 || QW == 1) ? 1 : 2)
    cross_fwd_kernel(CrossArgs<NS> a) {
  typedef Shape<NS, DP, QW, KW, NB> X;
  typedef typename X::L L;
  constexpr int QB = X::QB, KT = X::KT, NT = X::NT;
  // Single rows' weights keep 16 bits, in two parts: the matrix cores wait for memory there.
  constexpr bool TWO = NS == 1 && QW == 1;
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
        Frag<NS> P2;
        if constexpr (TWO) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            P2.s[0][j] = cvt2_bf16(p[2 * j] - __uint_as_float(P.s[0][j] << 16),
                                   p[2 * j + 1] - __uint_as_float(P.s[0][j] & 0xffff0000u));
        }
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
          const Frag<NS> W = EARLY ? V[b][s][d] : L::cols(vt, at, 32 * b + 16 * s, d);
          if constexpr (TWO) O[d] = mma<NS>(W, P2, O[d]);
          O[d] = mma<NS>(W, P, O[d]);
        }
      }
    }
  };
  auto sweep = [&](int first, bool stage) {
  const int r = first + (wave - kw * QW) * 32 + n32;  // the lane's tile row
  const bool mine = r < w.m;
  const int rr = min(r, w.m - 1);
  const int64_t row = w.base + rr / a.group;
  const int h = hk * a.group + rr % a.group;
  {
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
  const float inv = mk > 0 ? 1.f / sum : 0.f;
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
  const uint64_t bad = __ballot(mine && !fine && mk > 0);
  uint32_t rows = (uint32_t)bad | (uint32_t)(bad >> 32);
  const int w0 = first + wave * 32;
  for (; rows; rows &= rows - 1) {
    const int x = w0 + __builtin_ctz(rows);
    cross_row<NS>(a, w.base + x / a.group, hk * a.group + x % a.group, k0, mk);
  }
  };
  if constexpr (!FEW) {
    sweep(w.first, true);
  } else {
    const int end = min(w.m, w.first + QB * a.repeat);
    for (int first = w.first; first < end; first += QB)
      sweep(first, first == w.first || t1 - t0 > 2);
  }
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
struct CrossPlan {
  int qw, kw, nb, repeat;
  Parts parts;
};
CrossPlan plan(int type, int64_t nq, int64_t nk, int batch, int D, int Hk, int group) {
  CrossPlan p;
  const int used = (int)std::max<int64_t>(1, std::min<int64_t>(batch, nq));  // samples with queries
  const int64_t rows = ceil_div(nq * group, used), keys = nk / used;
  auto blocks = [&](int qb) { return used * ceil_div(rows, qb) * Hk; };
  const bool bf16 = type == SCN_BF16;
  if (rows <= 32 && bf16)
    p = {1, 4, 1, 1, {}};
  else if (bf16 && D <= 64)
    p = blocks(128) < 512 && keys > 128 ? CrossPlan{2, 2, 2, 1, {}} : CrossPlan{4, 1, 2, 1, {}};
  else if (!bf16 && D <= 64 && rows <= 64 && keys > 64)
    p = {2, 2, 1, 1, {}};
  else if ((bf16 || D <= 64) && (blocks(128) < 512 || (!bf16 && D > 32)) && keys > 64)
    p = {4, 2, 1, 1, {}};
  else
    p = {4, 1, 1, 1, {}};
  p.parts = cut(blocks(32 * p.qw), WANT, keys, LEAST, used);
  if (p.kw == 1 && keys <= 64 * p.nb)
    p.repeat = (int)std::max<int64_t>(1, std::min<int64_t>(8, blocks(32 * p.qw) / REPEAT_BLOCKS));
  return p;
}

template <int NS, int DP, int QW, int KW, int NB, bool FEW = false>
scn_status launch(CrossArgs<NS> a, const CrossPlan& p, hipStream_t st) {
  typedef Shape<NS, DP, QW, KW, NB> X;
  static LdsLimit limit;
  auto fn = cross_fwd_kernel<NS, DP, QW, KW, NB, FEW>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, X::SMEM)) return rc;
  a.deal.rows = X::QB * a.repeat;
  const int64_t blocks = a.deal.blocks();
  if (blocks > INT32_MAX) {
    set_error("scn_cross_attn_fwd: more than 2^31 blocks of rows and heads");
    return SCN_ERR_OVERFLOW;
  }
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(X::NT), X::SMEM, st, a);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}

template <int NS, int DP>
scn_status launch(const CrossArgs<NS>& a, const CrossPlan& p, hipStream_t st) {
  if constexpr (NS == 1)
    if (p.qw == 1) return launch<NS, DP, 1, 4, 1>(a, p, st);
  if constexpr (NS == 1 && DP <= 64) {
    if (p.qw == 2) return launch<NS, DP, 2, 2, 2>(a, p, st);
    if (p.repeat > 1) return launch<NS, DP, 4, 1, 2, true>(a, p, st);
    return launch<NS, DP, 4, 1, 2>(a, p, st);
  } else {
    if constexpr (NS == 3 && DP <= 64)
      if (p.qw == 2) return launch<NS, DP, 2, 2, 1>(a, p, st);
    if constexpr (NS == 1 || DP <= 64)
      if (p.kw == 2) return launch<NS, DP, 4, 2, 1>(a, p, st);
    if (p.repeat > 1) return launch<NS, DP, 4, 1, 1, true>(a, p, st);
    return launch<NS, DP, 4, 1, 1>(a, p, st);
  }
}

template <int NS>
scn_status run(const CrossArgs<NS>& a, const CrossPlan& p, hipStream_t st) {
  scn_status rc = a.D <= 32   ? launch<NS, 32>(a, p, st)
                  : a.D <= 64 ? launch<NS, 64>(a, p, st)
                  : a.D <= 96 ? launch<NS, 96>(a, p, st)
                              : launch<NS, 128>(a, p, st);
  if (rc || p.parts.most == 1) return rc;
  // as many rows a block as leave the card some thousand blocks, of at most 256 threads
  CrossArgs<NS> j = a;
  j.deal.parts = Parts{1, INT32_MAX};
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
  const Deal deal{{qr, nq, Hq / Hk}, {kr, nk, 1}, batch, 0, Hk, p.parts};
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
