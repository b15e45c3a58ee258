// Cross attention, backward, in two passes that each own their sums (attn_bwd.hip), without
// a window and with both axes split where the blocks are few: one over tiles of queries
// for dq and <do, o>, one over tiles of keys for dk and dv.
//
// Queries' pass: S^T = K Q^T and dP^T = V dO^T with a tile row per lane (cross.h),
// dQ^T += K^T dS^T.  Keys' pass: S = Q K^T and dP = dO V^T with a key per lane,
// dV^T += dO^T P and dK^T += Q^T dS over the queries of each head in turn.
// Split axes leave their sums in a workspace, and a join kernel adds them up in order.
#include "cross.h"

namespace scn {
namespace {

template <int NS>
struct CrossBwdArgs {
  typedef typename Elem<NS>::T T;
  int64_t nq, nk;
  int batch, D, Hk, group;
  const int32_t *qr, *kr;
  Heads<const T> q, k, v, o, d_o;
  Heads<T> dq, dk, dv;
  const float* lse;  // [Hq][nq]
  float* delta;      // [Hq][nq]
  float* lse2;       // [Hq][nq]: lse in log 2, or NaN where it is past LSE_MOST ...
  float* rest;       // [Hq][nq]: ... and what it lacks there
  float scale;
  int qs, ks;    // parts that the keys are split into for dq, and the queries for dk and dv
  float* qpart;  // [Hq][nq][qs][2][D] (dQ, PK), then [Hq][nq][qs] (the sum of dS)
  float* kpart;  // [Hk][nk][ks][2][D] (dK, dV)
  __device__ inline float* qout(int64_t at, int s) const { return qpart + (at * qs + s) * 2 * D; }
  __device__ inline float* over(int64_t at) const {
    return qpart + nq * Hk * group * qs * 2 * D + at * qs;
  }
  __device__ inline float* kout(int64_t at, int s) const { return kpart + (at * ks + s) * 2 * D; }
};

// dq of one row once more in fp32, over its cnt >= 1 keys, from weights of its own.  The
// keys' pass gets its delta, and what the row's lse is short of their log sum.
template <int NS>
__device__ inline void dq_row(const CrossBwdArgs<NS>& a, int64_t row, int h, int64_t k0, int cnt) {
  typedef Elem<NS> E;
  const int lane = threadIdx.x & 63;
  const auto* const q = a.q.p + row * a.q.row + h * a.q.head;
  const auto* const g = a.d_o.p + row * a.d_o.row + h * a.d_o.head;
  const auto* const k = a.k.p + k0 * a.k.row + (h / a.group) * a.k.head;
  const auto* const v = a.v.p + k0 * a.v.row + (h / a.group) * a.v.head;
  auto score = [&](int x) { return row_dot<NS>(q, k + x * a.k.row, a.D) * a.scale; };
  auto dp = [&](int x) { return row_dot<NS>(g, v + x * a.v.row, a.D); };
  RowSum r;
  for (int x = lane; x < cnt; x += 64) r.add(score(x));
  r.join();
  float delta = 0.f;
  for (int x = lane; x < cnt; x += 64) delta = fmaf(r.weight(score(x)), dp(x), delta);
  delta = wave_sum(delta);
  float o0 = 0.f, o1 = 0.f;
  for (int x0 = 0; x0 < cnt; x0 += 64) {
    const int x = x0 + lane;
    const float ds = x < cnt ? r.weight(score(x)) * (dp(x) - delta) : 0.f;
    for (int y = 0; y < min(64, cnt - x0); ++y) {
      const auto* const kj = k + (x0 + y) * a.k.row;
      const float d = __shfl(ds, y);
      if (lane < a.D) o0 = fmaf(d, E::get(kj[lane]), o0);
      if (64 + lane < a.D) o1 = fmaf(d, E::get(kj[64 + lane]), o1);
    }
  }
  auto* const o = a.dq.p + row * a.dq.row + h * a.dq.head;
  if (lane < a.D) o[lane] = E::put(o0 * a.scale);
  if (64 + lane < a.D) o[64 + lane] = E::put(o1 * a.scale);
  if (lane == 0) {
    const int64_t at = h * a.nq + row;
    a.delta[at] = delta;
    a.rest[at] = (r.top - a.lse[at]) + logf(r.sum);
  }
}

// dk and dv of one row once more in fp32, over the m queries from q0 on
template <int NS>
__device__ inline void dkv_row(const CrossBwdArgs<NS>& a, int64_t row, int hk, int64_t q0, int m) {
  typedef Elem<NS> E;
  const int lane = threadIdx.x & 63;
  const auto* const k = a.k.p + row * a.k.row + hk * a.k.head;
  const auto* const v = a.v.p + row * a.v.row + hk * a.v.head;
  auto* const dk = a.dk.p + row * a.dk.row + hk * a.dk.head;
  auto* const dv = a.dv.p + row * a.dv.row + hk * a.dv.head;
  // a row of no weights (its lse is NaN) leaves nothing to add up
  bool none = false;
  for (int h = hk * a.group; h < (hk + 1) * a.group; ++h)
    for (int i = lane; i < m; i += 64) {
      const float l = a.lse[h * a.nq + q0 + i];
      none |= l != l;
    }
  if (__ballot(none)) {
    for (int c = lane; c < a.D; c += 64) dk[c] = dv[c] = E::put(NAN);
    return;
  }
  float s0 = 0.f, s1 = 0.f, v0 = 0.f, v1 = 0.f;
  for (int h = hk * a.group; h < (hk + 1) * a.group; ++h) {
    const auto* const q = a.q.p + q0 * a.q.row + h * a.q.head;
    const auto* const g = a.d_o.p + q0 * a.d_o.row + h * a.d_o.head;
    for (int x0 = 0; x0 < m; x0 += 64) {
      float p = 0.f, ds = 0.f;
      const int i = x0 + lane;
      if (i < m) {
        const int64_t at = h * a.nq + q0 + i;
        p = row_dot<NS>(q + i * a.q.row, k, a.D) * a.scale - a.lse[at];
        p = expf(fabsf(a.lse[at]) <= LSE_MOST ? p : p - a.rest[at]);
        ds = p * (row_dot<NS>(g + i * a.d_o.row, v, a.D) - a.delta[at]);
      }
      for (int y = 0; y < min(64, m - x0); ++y) {
        const float py = __shfl(p, y), dy = __shfl(ds, y);
        const auto* const qi = q + (x0 + y) * a.q.row;
        const auto* const gi = g + (x0 + y) * a.d_o.row;
        if (lane < a.D) {
          v0 = fmaf(py, E::get(gi[lane]), v0);
          s0 = fmaf(dy, E::get(qi[lane]), s0);
        }
        if (64 + lane < a.D) {
          v1 = fmaf(py, E::get(gi[64 + lane]), v1);
          s1 = fmaf(dy, E::get(qi[64 + lane]), s1);
        }
      }
    }
  }
  if (lane < a.D) {
    dk[lane] = E::put(s0 * a.scale);
    dv[lane] = E::put(v0);
  }
  if (64 + lane < a.D) {
    dk[64 + lane] = E::put(s1 * a.scale);
    dv[64 + lane] = E::put(v1);
  }
}

// QW waves of 32 tile rows by KW groups that share out the keys of a tile, 32 each
template <int NS, int DP, int QW, int KW>
struct QueryShape {
  static constexpr int QB = 32 * QW, NT = 64 * QW * KW, KT = 32 * KW;
  typedef Tile<NS, DP, KT> L;
  // <do, o> has o's rounding to bf16, the same for all keys of a row, where the sum of dS is 0
  // by definition (attn_bwd.hip).  What is left of that sum (`over`) comes off dQ as over P K.
  static constexpr bool EXACT = NS == 1;
  static constexpr int SUMS = (EXACT ? 2 : 1) * DP / 32 * 16;  // floats a lane hands over
  static constexpr size_t SMEM =
      std::max<size_t>(4 * L::BYTES, (size_t)QW * (KW - 1) * SUMS * 256);
  static_assert(SMEM <= 160 * 1024, "LDS of a compute unit");
};

template <int NS, int DP, int QW, int KW>
__global__ void __launch_bounds__(64 * QW * KW, (NS == 3 && DP > 32) || DP > 64 ? 1 : 2)
    cross_dq_kernel(CrossBwdArgs<NS> a) {
  typedef QueryShape<NS, DP, QW, KW> X;
  typedef typename X::L L;
  constexpr int KT = X::KT, NT = X::NT, QB = X::QB;
  constexpr bool EXACT = X::EXACT;
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kw = KW == 1 ? 0 : wave / QW;
  const int split = blockIdx.x % a.qs, hk = blockIdx.x / a.qs % a.Hk;
  const Place sp = find_place(a.qr, a.batch, a.nq, blockIdx.x / a.qs / a.Hk, QB, a.group);
  if (sp.first >= sp.m) return;
  int64_t k0;
  int mk;
  find_rows(a.kr, sp.sample, a.nk, k0, mk);
  const int r = sp.first + (wave - kw * QW) * 32 + n32;
  const bool mine = r < sp.m;
  const int rr = min(r, sp.m - 1);
  const int64_t row = sp.base + rr / a.group;
  const int h = hk * a.group + rr % a.group;
  const float c2 = a.scale * LOG2E;

  Frag<NS> Q[DP / 16], G[DP / 16];
  float delta = 0.f;
  {
    const auto* const q = a.q.p + row * a.q.row + h * a.q.head;
    const auto* const g = a.d_o.p + row * a.d_o.row + h * a.d_o.head;
    const auto* const o = a.o.p + row * a.o.row + h * a.o.head;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      Q[s] = load_frag<NS>(q, s, a.D, lane);
      G[s] = load_frag<NS>(g, s, a.D, lane);
      const int c = 16 * s + 8 * half;
      if (c < a.D) {
        float x[8], y[8];
        load8<NS>(g + c, x);
        load8<NS>(o + c, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = fmaf(x[j], y[j], delta);
      }
    }
  }
  delta = both_sum(delta);
  const int64_t at = h * a.nq + row;
  const float lse2 = a.lse[at] * LOG2E;
  const bool far = !(fabsf(a.lse[at]) <= LSE_MOST);  // the row is formed again ...
  const bool none = a.lse[at] != a.lse[at];           // ... if it has weights at all
  float over = 0.f;
  v16f dQ[DP / 32], PK[EXACT ? DP / 32 : 1];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) dQ[d] = zero16();
  if constexpr (EXACT)
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) PK[d] = zero16();

  const int nt = (mk + KT - 1) / KT, per = (nt + a.qs - 1) / a.qs;
  const int t0 = min(nt, split * per), t1 = min(nt, t0 + per);
  const auto* const kp = a.k.p + k0 * a.k.row + hk * a.k.head;
  const auto* const vp = a.v.p + k0 * a.v.row + hk * a.v.head;
  typedef Stage<NS, DP, KT, NT> St;
  St sk, sv;
  uint32_t ko[St::N], vo[St::N];
  St::places(ko, a.k.row, a.D, tid);
  St::places(vo, a.v.row, a.D, tid);
  const typename L::Lane pl(lane);
  auto fetch = [&](int t) {
    sk.load(kp, a.k.row, ko, t * KT, mk - t * KT, a.D);
    sv.load(vp, a.v.row, vo, t * KT, mk - t * KT, a.D);
  };
  auto put = [&](int t) {
    char* const b = smem + ((t - t0) & 1) * 2 * L::BYTES;
    sk.store(b, tid);
    sv.store(b + L::BYTES, tid);
  };
  auto take = [&](int t) {
    char* const kt = smem + ((t - t0) & 1) * 2 * L::BYTES + kw * 32 * DP * 2;
    char* const vt = kt + L::BYTES;
    const int left = mk - t * KT - kw * 32;
    Frag<NS> KC[2][DP / 32];  // read early where the registers allow two waves only anyway
    if constexpr (EXACT) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) KC[s][d] = L::cols(kt, pl, 16 * s, d);
    }
    v16f S = zero16(), P = zero16();
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) S = mma<NS>(L::rows(kt, pl, 0, s), Q[s], S);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) P = mma<NS>(L::rows(vt, pl, 0, s), G[s], P);
    if (left < 32) {
#pragma unroll
      for (int x = 0; x < 16; ++x)
        S[x] = 8 * (x / 4) + 4 * half + x % 4 < left ? S[x] : -INFINITY;
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      S[x] = __builtin_amdgcn_exp2f(fmaf(S[x], c2, -lse2));
      P[x] = S[x] * (P[x] - delta);
      if constexpr (EXACT) over += P[x];
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float x[8], y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = S[8 * s + j];
        y[j] = P[8 * s + j];
      }
      const Frag<NS> X = to_frag<NS>(x), Y = to_frag<NS>(y);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        const Frag<NS> K = EXACT ? KC[s][d] : L::cols(kt, pl, 16 * s, d);
        dQ[d] = mma<NS>(K, Y, dQ[d]);
        if constexpr (EXACT) PK[d] = mma<NS>(K, X, PK[d]);
      }
    }
  };
  if (t0 < t1) {
    fetch(t0);
    put(t0);
    if (t0 + 1 < t1) fetch(t0 + 1);
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
      if (t + 1 < t1) put(t + 1);
      if (t + 2 < t1) fetch(t + 2);
      take(t);
      __syncthreads();
    }
  }
  // the groups' sums, joined in order
  over = both_sum(over);
  if constexpr (KW > 1) {
    float* const x = reinterpret_cast<float*>(smem) + lane;
    if constexpr (EXACT) {
      x[wave * 64] = over;
      __syncthreads();
      over = 0.f;
      for (int g = 0; g < KW; ++g) over += x[(g * QW + wave - kw * QW) * 64];
      __syncthreads();
    }
    float* const o = x + (wave - QW) * X::SUMS * 64;
    if (kw > 0) {
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          o[(d * 16 + e) * 64] = dQ[d][e];
          if constexpr (EXACT) o[((DP / 32 + d) * 16 + e) * 64] = PK[d][e];
        }
    }
    __syncthreads();
    if (kw > 0) return;
    for (int g = 0; g < KW - 1; ++g) {
      const float* const o = x + (g * QW + wave) * X::SUMS * 64;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          dQ[d][e] += o[(d * 16 + e) * 64];
          if constexpr (EXACT) PK[d][e] += o[((DP / 32 + d) * 16 + e) * 64];
        }
    }
  }
  if (a.qs > 1) {
    if (mine) {
      float* const o = a.qout(at, split);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        store_cols<3>(o, dQ[d], 1.f, d, a.D, lane);
        if constexpr (EXACT) store_cols<3>(o + a.D, PK[d], 1.f, d, a.D, lane);
      }
      if (half == 0) {
        a.over(at)[split] = over;
        if (split == 0) {
          a.delta[at] = delta;
          a.lse2[at] = far ? NAN : lse2;
        }
      }
    }
    return;
  }
  if constexpr (EXACT) {
    over = fabsf(over) < INFINITY ? over : 0.f;
    delta += over;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) dQ[d][e] = fmaf(-over, PK[d][e], dQ[d][e]);
  }
  bool fine = true;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) fine &= finite16(dQ[d]);
  if constexpr (NS == 3) fine &= !tiny(dQ, 1.f);
  if (mine) {
    if (half == 0) {
      a.delta[at] = delta;
      a.lse2[at] = far ? NAN : lse2;  // keys that see the row are formed again
    }
    auto* const o = a.dq.p + row * a.dq.row + h * a.dq.head;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) store_cols<NS>(o, dQ[d], a.scale, d, a.D, lane);
  }
  const uint64_t bad = __ballot(mine && !none && (far || !fine) && mk > 0);
  uint32_t rows = (uint32_t)bad | (uint32_t)(bad >> 32);
  const int w0 = sp.first + wave * 32;
  for (; rows; rows &= rows - 1) {
    const int x = w0 + __builtin_ctz(rows);
    dq_row<NS>(a, sp.base + x / a.group, hk * a.group + x % a.group, k0, mk);
  }
}

// The parts of a row's dq, a wave a row and head, channels along the lanes, added up in order
template <int NS>
__global__ void __launch_bounds__(256) cross_dq_join_kernel(CrossBwdArgs<NS> a) {
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= a.nq * a.Hk * a.group) return;
  const int h = (int)(at / a.nq);
  const int64_t row = at - h * a.nq;
  int sample;
  if (!find_row(a.qr, a.batch, a.nq, (int)row, sample)) return;
  int64_t k0;
  int mk;
  find_rows(a.kr, sample, a.nk, k0, mk);
  float over = 0.f, d[2] = {0.f, 0.f}, p[2] = {0.f, 0.f};
  for (int s0 = 0; s0 < a.qs; s0 += 4) {
    float x[4][2], y[4][2], z[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool on = s0 + j < a.qs;
      const float* const o = a.qout(at, on ? s0 + j : 0);
      z[j] = on ? a.over(at)[s0 + j] : 0.f;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const bool has = on && 64 * c + lane < a.D;
        x[j][c] = has ? o[64 * c + lane] : 0.f;
        y[j][c] = NS == 1 && has ? o[a.D + 64 * c + lane] : 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      over += z[j];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        d[c] += x[j][c];
        p[c] += y[j][c];
      }
    }
  }
  const float l = a.lse[at];
  const bool far = !(fabsf(l) <= LSE_MOST), none = l != l;
  if constexpr (NS == 1) {
    over = fabsf(over) < INFINITY ? over : 0.f;
    if (lane == 0) a.delta[at] += over;
    d[0] = fmaf(-over, p[0], d[0]);
    d[1] = fmaf(-over, p[1], d[1]);
  }
  bool fine = fabsf(d[0]) < INFINITY && fabsf(d[1]) < INFINITY;
  if constexpr (NS == 3) {
    const float big = wave_max(fmaxf(fabsf(d[0]), fabsf(d[1])));
    fine &= !(big > 0.f && big < 0x1p-95f);
  }
  if (mk > 0 && !none && (far || __ballot(!fine))) {
    dq_row<NS>(a, row, h, k0, mk);
    return;
  }
  auto* const o = a.dq.p + row * a.dq.row + h * a.dq.head;
  if (lane < a.D) o[lane] = Elem<NS>::put(d[0] * a.scale);
  if (64 + lane < a.D) o[64 + lane] = Elem<NS>::put(d[1] * a.scale);
}

// What a wave with 32 keys does with 32 queries of a tile: dV += P^T dO, dK += dS^T Q
// (transposed).  Queries past the sample's last have a log sum of +inf, and so no weight.
// EARLY reads each pair of products' operands ahead of them, for some 60 registers more.
template <int NS, int DP, int TB, bool EARLY>
__device__ inline void key_block(char* qt, char* gt, const typename Tile<NS, DP, TB>::Lane& pl,
                                 const float* lse2, const float* delta, int r0,
                                 const Frag<NS> (&K)[DP / 16], const Frag<NS> (&V)[DP / 16],
                                 float c2, v16f (&dK)[DP / 32], v16f (&dV)[DP / 32]) {
  typedef Tile<NS, DP, TB> L;
  const int half = (threadIdx.x & 63) >> 5;
  Frag<NS> QR[DP / 16], GR[DP / 16], QC[2][DP / 32], GC[2][DP / 32];
  v4f ls[4], de[4];
  auto sums = [&](int g) {
    ls[g] = *reinterpret_cast<const v4f*>(lse2 + r0 + 8 * g + 4 * half);
    de[g] = *reinterpret_cast<const v4f*>(delta + r0 + 8 * g + 4 * half);
  };
  if constexpr (EARLY) {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      QR[s] = L::rows(qt, pl, r0, s);
      GR[s] = L::rows(gt, pl, r0, s);
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) sums(g);
    __builtin_amdgcn_sched_barrier(0);
  }
  v16f S = zero16(), P = zero16();
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    S = mma<NS>(EARLY ? QR[s] : L::rows(qt, pl, r0, s), K[s], S);
    P = mma<NS>(EARLY ? GR[s] : L::rows(gt, pl, r0, s), V[s], P);
  }
  if constexpr (EARLY) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        GC[s][d] = L::cols(gt, pl, r0 + 16 * s, d);
        QC[s][d] = L::cols(qt, pl, r0 + 16 * s, d);
      }
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    if constexpr (!EARLY) sums(g);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = 4 * g + j;
      S[r] = __builtin_amdgcn_exp2f(fmaf(S[r], c2, -ls[g][j]));
      P[r] = S[r] * (P[r] - de[g][j]);
    }
  }
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    float x[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = S[8 * s + j];
      y[j] = P[8 * s + j];
    }
    const Frag<NS> X = to_frag<NS>(x), Y = to_frag<NS>(y);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      dV[d] = mma<NS>(EARLY ? GC[s][d] : L::cols(gt, pl, r0 + 16 * s, d), X, dV[d]);
      dK[d] = mma<NS>(EARLY ? QC[s][d] : L::cols(qt, pl, r0 + 16 * s, d), Y, dK[d]);
    }
  }
}

// KW waves of 32 keys by QW groups that share out the queries of a tile, 32 U each.  The
// groups' sums join in LDS at the end.
template <int NS, int DP, int KW, int QW, int U>
struct KeyShape {
  static constexpr int KB = 32 * KW, NT = 64 * KW * QW, TB = 32 * U * QW;
  typedef Tile<NS, DP, TB> L;
  typedef Stage<NS, DP, TB, NT> St;
  static constexpr int BUF = 2 * L::BYTES + 2 * TB * 4;
  static constexpr int JOIN = DP / 32 * 32;  // floats a lane hands over
  static constexpr size_t SMEM = std::max<size_t>(2 * BUF, (size_t)KW * (QW - 1) * JOIN * 256);
  static_assert(SMEM <= 160 * 1024, "LDS of a compute unit");
};

template <int NS, int DP, int KW, int QW, int U>
__global__ void __launch_bounds__(64 * KW * QW, NS == 3 || DP > 64 ? 1 : 2)
    cross_dkv_kernel(CrossBwdArgs<NS> a) {
  typedef KeyShape<NS, DP, KW, QW, U> X;
  typedef typename X::L L;
  typedef typename X::St St;
  constexpr int KB = X::KB, TB = X::TB;
  constexpr bool EARLY = NS == 1 && DP == 64 && QW < 4;
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), qw = QW == 1 ? 0 : wave / KW;
  const int split = blockIdx.x % a.ks, hk = blockIdx.x / a.ks % a.Hk;
  const Place sp = find_place(a.kr, a.batch, a.nk, blockIdx.x / a.ks / a.Hk, KB, 1);
  if (sp.first >= sp.m) return;
  int64_t q0;
  int mq;
  find_rows(a.qr, sp.sample, a.nq, q0, mq);
  const int j = min(sp.first + (wave - qw * KW) * 32 + n32, sp.m - 1);  // the lane's key
  const bool mine = sp.first + (wave - qw * KW) * 32 + n32 < sp.m;
  const float c2 = a.scale * LOG2E;

  Frag<NS> K[DP / 16], V[DP / 16];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    K[s] = load_frag<NS>(a.k.p + (sp.base + j) * a.k.row + hk * a.k.head, s, a.D, lane);
    V[s] = load_frag<NS>(a.v.p + (sp.base + j) * a.v.row + hk * a.v.head, s, a.D, lane);
  }
  v16f dK[DP / 32], dV[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) dK[d] = dV[d] = zero16();

  // the block's tiles of queries, those of each head in turn
  const int per = (mq + TB - 1) / TB;
  const int64_t nt = (int64_t)per * a.group, share = (nt + a.ks - 1) / a.ks;
  const int64_t t0 = min(nt, split * share), t1 = min(nt, t0 + share);
  St sq, sg;
  float lse2 = 0.f, delta = 0.f;
  uint32_t qo[St::N], go[St::N];
  St::places(qo, a.q.row, a.D, tid);
  St::places(go, a.d_o.row, a.D, tid);
  const typename L::Lane pl(lane);
  int h = per > 0 ? hk * a.group + (int)(t0 / per) : 0;  // of the next tile to fetch
  int i0 = per > 0 ? (int)(t0 % per) * TB : 0;
  auto fetch = [&]() {
    sq.load(a.q.p + q0 * a.q.row + h * a.q.head, a.q.row, qo, i0, mq - i0, a.D);
    sg.load(a.d_o.p + q0 * a.d_o.row + h * a.d_o.head, a.d_o.row, go, i0, mq - i0, a.D);
    if (tid < TB) {
      const int64_t at = h * a.nq + q0 + min(i0 + tid, mq - 1);
      lse2 = i0 + tid < mq ? a.lse2[at] : INFINITY;
      delta = i0 + tid < mq ? a.delta[at] : 0.f;
    }
    i0 += TB;
    if (i0 >= mq) {
      i0 = 0;
      ++h;
    }
  };
  auto put = [&](int64_t t) {
    char* const b = smem + ((t - t0) & 1) * X::BUF;
    sq.store(b, tid);
    sg.store(b + L::BYTES, tid);
    if (tid < TB) {
      float* const f = reinterpret_cast<float*>(b + 2 * L::BYTES);
      f[tid] = lse2;
      f[TB + tid] = delta;
    }
  };
  if (t0 < t1) {
    fetch();
    put(t0);
    if (t0 + 1 < t1) fetch();
    __syncthreads();
    for (int64_t t = t0; t < t1; ++t) {
      if (t + 1 < t1) put(t + 1);
      if (t + 2 < t1) fetch();
      char* const b = smem + ((t - t0) & 1) * X::BUF;
      const float* const f = reinterpret_cast<const float*>(b + 2 * L::BYTES);
#pragma unroll
      for (int u = 0; u < U; ++u)
        key_block<NS, DP, TB, EARLY>(b, b + L::BYTES, pl, f, f + TB, (qw * U + u) * 32, K, V, c2, dK,
                                     dV);
      __syncthreads();
    }
  }
  if constexpr (QW > 1) {
    float* const x = reinterpret_cast<float*>(smem) + lane;
    if (qw > 0) {
      float* const o = x + (wave - KW) * X::JOIN * 64;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          o[(d * 16 + r) * 64] = dK[d][r];
          o[((DP / 32 + d) * 16 + r) * 64] = dV[d][r];
        }
    }
    __syncthreads();
    if (qw > 0) return;
    for (int g = 1; g < QW; ++g) {
      const float* const o = x + ((g - 1) * KW + wave) * X::JOIN * 64;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          dK[d][r] += o[(d * 16 + r) * 64];
          dV[d][r] += o[((DP / 32 + d) * 16 + r) * 64];
        }
    }
  }
  if (a.ks > 1) {
    if (mine) {
      float* const o = a.kout(hk * a.nk + sp.base + j, split);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        store_cols<3>(o, dK[d], 1.f, d, a.D, lane);
        store_cols<3>(o + a.D, dV[d], 1.f, d, a.D, lane);
      }
    }
    return;
  }
  bool fine = true;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) fine &= finite16(dK[d]) && finite16(dV[d]);
  if constexpr (NS == 3) fine &= !tiny(dK, 1.f) && !tiny(dV, 1.f);
  if (mine) {
    auto* const dk = a.dk.p + (sp.base + j) * a.dk.row + hk * a.dk.head;
    auto* const dv = a.dv.p + (sp.base + j) * a.dv.row + hk * a.dv.head;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      store_cols<NS>(dk, dK[d], a.scale, d, a.D, lane);
      store_cols<NS>(dv, dV[d], 1.f, d, a.D, lane);
    }
  }
  const uint64_t bad = __ballot(mine && !fine);
  uint32_t rows = (uint32_t)bad | (uint32_t)(bad >> 32);
  const int64_t w0 = sp.base + sp.first + wave * 32;
  for (; rows; rows &= rows - 1) dkv_row<NS>(a, w0 + __builtin_ctz(rows), hk, q0, mq);
}

// The parts of a key's dk and dv, a wave a row and head, channels along the lanes, in order
template <int NS>
__global__ void __launch_bounds__(256) cross_dkv_join_kernel(CrossBwdArgs<NS> a) {
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= a.nk * a.Hk) return;
  const int hk = (int)(at / a.nk);
  const int64_t row = at - hk * a.nk;
  int sample;
  if (!find_row(a.kr, a.batch, a.nk, (int)row, sample)) return;
  // lane's elements of dK and dV side by side, 2 D <= 256 of them
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.ks; s0 += 4) {
    float x[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float* const o = a.kout(at, min(s0 + j, a.ks - 1));
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int e = 64 * c + lane;
        x[j][c] = s0 + j < a.ks && e < 2 * a.D ? o[e] : 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] += x[j][c];
  }
  bool fine = true;
  float bigk = 0.f, bigv = 0.f;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    fine &= fabsf(v[c]) < INFINITY;
    if (64 * c + lane < a.D) bigk = fmaxf(bigk, fabsf(v[c]));
    else bigv = fmaxf(bigv, fabsf(v[c]));
  }
  if constexpr (NS == 3) {
    bigk = wave_max(bigk);
    bigv = wave_max(bigv);
    fine &= !(bigk > 0.f && bigk < 0x1p-95f) && !(bigv > 0.f && bigv < 0x1p-95f);
  }
  if (__ballot(!fine)) {
    int64_t q0;
    int mq;
    find_rows(a.qr, sample, a.nq, q0, mq);
    dkv_row<NS>(a, row, hk, q0, mq);
    return;
  }
  auto* const dk = a.dk.p + row * a.dk.row + hk * a.dk.head;
  auto* const dv = a.dv.p + row * a.dv.row + hk * a.dv.head;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int e = 64 * c + lane;
    if (e < a.D) dk[e] = Elem<NS>::put(v[c] * a.scale);
    else if (e < 2 * a.D) dv[e - a.D] = Elem<NS>::put(v[c]);
  }
}

// Shapes and parts of both passes, by rules on sizes alone (cross_fwd.hip)
struct CrossBwdPlan {
  int qw, qkw, qs;  // queries' pass: waves of queries, groups of keys, parts of the keys
  int kw, kqw, ks;  // keys' pass: waves of keys, groups of queries, parts of the queries
};
CrossBwdPlan plan(int type, int64_t nq, int64_t nk, int batch, int D, int Hk, int group) {
  CrossBwdPlan p;
  const int64_t usedq = std::max<int64_t>(1, std::min<int64_t>(batch, nq));
  const int64_t usedk = std::max<int64_t>(1, std::min<int64_t>(batch, nk));
  const int64_t rows = ceil_div(nq * group, usedq), keys = ceil_div(nk, usedk);
  auto qblocks = [&](int b) { return usedq * ceil_div(rows, b) * Hk; };
  auto kblocks = [&](int b) { return usedk * ceil_div(keys, b) * Hk; };
  if (rows <= 32 && (type == SCN_BF16 || D <= 96)) {
    p.qw = 1;
    p.qkw = type == SCN_BF16 || D <= 32 ? 4 : 2;
  } else if (type == SCN_F32) {
    p.qw = D > 32 ? 4 : 2;
    p.qkw = D > 64 ? 1 : 2;
  } else {
    p.qw = D > 64 && qblocks(128) >= 512 ? 4 : 2;
    p.qkw = p.qw == 4 ? 1 : 2;
  }
  p.qs = parts(qblocks(32 * p.qw), 512, nk / usedq, 256);
  if (type == SCN_F32) {
    p.kw = keys <= 32 && D <= 32 ? 1 : D <= 64 ? 2 : 4;
    p.kqw = p.kw == 1 ? 4 : p.kw == 2 ? 2 : 1;
  } else {
    p.kw = D <= 64 && (keys <= 32 || kblocks(128) < 128) ? 1
           : kblocks(128) < (D <= 64 ? 1024 : 384)       ? 2
                                                         : 4;
    p.kqw = 4 / p.kw;
  }
  p.ks = parts(kblocks(32 * p.kw), 512, nq * group / usedk, 256);
  return p;
}

template <int NS, int DP, int QW, int KW>
scn_status launch_dq(const CrossBwdArgs<NS>& a, hipStream_t st) {
  typedef QueryShape<NS, DP, QW, KW> X;
  static LdsLimit limit;
  auto fn = cross_dq_kernel<NS, DP, QW, KW>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, X::SMEM)) return rc;
  const int64_t blocks = (a.nq * a.group / X::QB + a.batch) * a.Hk * a.qs;
  const int64_t joins = ceil_div(a.nq * a.Hk * a.group, 4);
  if (std::max(blocks, joins) > INT32_MAX) {
    set_error("scn_cross_attn_bwd: more than 2^31 blocks of rows, heads and parts");
    return SCN_ERR_OVERFLOW;
  }
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(X::NT), X::SMEM, st, a);
  SCN_LAUNCH_CHECK();
  if (a.qs > 1) {
    hipLaunchKernelGGL(cross_dq_join_kernel<NS>, dim3((unsigned)joins), dim3(256), 0, st, a);
    SCN_LAUNCH_CHECK();
  }
  return SCN_OK;
}

template <int NS, int DP, int KW, int QW, int U>
scn_status launch_dkv(const CrossBwdArgs<NS>& a, hipStream_t st) {
  typedef KeyShape<NS, DP, KW, QW, U> X;
  static LdsLimit limit;
  auto fn = cross_dkv_kernel<NS, DP, KW, QW, U>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, X::SMEM)) return rc;
  const int64_t blocks = (a.nk / X::KB + a.batch) * a.Hk * a.ks;
  const int64_t joins = ceil_div(a.nk * a.Hk, 4);
  if (std::max(blocks, joins) > INT32_MAX) {
    set_error("scn_cross_attn_bwd: more than 2^31 blocks of keys, heads and parts");
    return SCN_ERR_OVERFLOW;
  }
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(X::NT), X::SMEM, st, a);
  SCN_LAUNCH_CHECK();
  if (a.ks > 1) {
    hipLaunchKernelGGL(cross_dkv_join_kernel<NS>, dim3((unsigned)joins), dim3(256), 0, st, a);
    SCN_LAUNCH_CHECK();
  }
  return SCN_OK;
}

template <int NS, int DP>
scn_status launch(const CrossBwdArgs<NS>& a, const CrossBwdPlan& p, hipStream_t st) {
  scn_status rc = SCN_OK;
  if (a.nq > 0) {
    if constexpr (NS == 3) {
      if constexpr (DP <= 96)
        if (p.qw == 1) rc = launch_dq<NS, DP, 1, (DP == 32 ? 4 : 2)>(a, st);
      if (p.qw > 1) rc = launch_dq<NS, DP, (DP > 32 ? 4 : 2), (DP > 64 ? 1 : 2)>(a, st);
    } else if (p.qw == 1) {
      rc = launch_dq<NS, DP, 1, 4>(a, st);
    } else {
      constexpr int QW = DP > 64 ? 4 : 2, KW = DP > 64 ? 1 : 2;
      rc = p.qw == 2 ? launch_dq<NS, DP, 2, 2>(a, st) : launch_dq<NS, DP, QW, KW>(a, st);
    }
  }
  if (rc || a.nk == 0) return rc;
  if constexpr (NS == 3) {
    if constexpr (DP <= 32)
      if (p.kw == 1) return launch_dkv<NS, DP, 1, 4, 1>(a, st);
    if constexpr (DP <= 64) {
      return launch_dkv<NS, DP, 2, 2, 1>(a, st);
    } else {
      return launch_dkv<NS, DP, 4, 1, 1>(a, st);
    }
  } else {
    if constexpr (DP <= 64)
      if (p.kw == 1) return launch_dkv<NS, DP, 1, 4, 1>(a, st);
    if (p.kw == 2) return launch_dkv<NS, DP, 2, 2, 1>(a, st);
    return launch_dkv<NS, DP, 4, 1, 2>(a, st);
  }
}

template <int NS>
scn_status run(const CrossBwdArgs<NS>& a, const CrossBwdPlan& p, hipStream_t st) {
  if (a.D <= 32) return launch<NS, 32>(a, p, st);
  if (a.D <= 64) return launch<NS, 64>(a, p, st);
  if (a.D <= 96) return launch<NS, 96>(a, p, st);
  return launch<NS, 128>(a, p, st);
}

// floats of the workspace: three rows' statistics, then the parts of dq, then those of dk and dv
// (each needed by one pass and its join alone, so they lie in the same place)
int64_t stat_floats(int64_t nq, int Hq) { return (nq * Hq + 63) & ~int64_t(63); }
int64_t part_floats(const CrossBwdPlan& p, int64_t nq, int64_t nk, int Hq, int Hk, int D) {
  const int64_t q = p.qs > 1 ? nq * Hq * p.qs * (2 * D + 1) : 0;
  const int64_t k = p.ks > 1 ? nk * Hk * p.ks * 2 * D : 0;
  return std::max(q, k);
}

template <int NS>
CrossBwdArgs<NS> make(int64_t nq, int64_t nk, int batch, const int32_t* qr, const int32_t* kr, int D,
                      int Hq, int Hk, const scn_heads* q, const scn_heads* k, const scn_heads* v,
                      const scn_heads* o, const float* lse, const scn_heads* d_o, float scale,
                      const scn_heads* dq, const scn_heads* dk, const scn_heads* dv,
                      const CrossBwdPlan& p, void* ws) {
  typedef typename Elem<NS>::T T;
  float* const f = static_cast<float*>(ws);
  const int64_t n = stat_floats(nq, Hq);
  return CrossBwdArgs<NS>{nq, nk, batch, D, Hk, Hq / Hk, qr, kr, view<const T>(q), view<const T>(k),
                          view<const T>(v), view<const T>(o), view<const T>(d_o), view<T>(dq),
                          view<T>(dk), view<T>(dv), lse, f, f + n, f + 2 * n, scale, p.qs, p.ks,
                          f + 3 * n, f + 3 * n};
}

}  // namespace

}  // namespace scn

using namespace scn;

extern "C" {

size_t scn_cross_attn_bwd_workspace_bytes(int32_t type, int64_t nq, int64_t nk, int32_t batch,
                                          int32_t D, int32_t Hq, int32_t Hk) {
  if ((type != SCN_F32 && type != SCN_BF16) || nq < 0 || nk < 0 || nk > ATTN_ROWS || batch < 1 ||
      D < 1 || D > ATTN_D || Hk < 1 || Hq < 1 || Hq % Hk != 0 || nq > ATTN_ROWS / (Hq / Hk))
    return 0;
  const CrossBwdPlan p = plan(type, nq, nk, batch, D, Hk, Hq / Hk);
  return (size_t)(3 * stat_floats(nq, Hq) + part_floats(p, nq, nk, Hq, Hk, D)) * 4;
}

scn_status scn_cross_attn_bwd(int32_t type, int64_t nq, int64_t nk, int32_t batch,
                              const int32_t* q_ranges, const int32_t* k_ranges, int32_t D,
                              int32_t Hq, int32_t Hk, const scn_heads* q, const scn_heads* k,
                              const scn_heads* v, const scn_heads* o, const float* lse,
                              const scn_heads* d_o, float scale, const scn_heads* dq,
                              const scn_heads* dk, const scn_heads* dv, void* ws, size_t ws_bytes,
                              hipStream_t st) {
  clear_error();
  const char* const who = "scn_cross_attn_bwd";
  if (scn_status rc = check_cross(who, type, nq, nk, batch, q_ranges, k_ranges, D, Hq, Hk, scale))
    return rc;
  if (nq > 0 && !lse) {
    set_error("%s: lse is null", who);
    return SCN_ERR_INVALID;
  }
  const struct {
    const scn_heads* h;
    const char* name;
    int64_t rows;
  } all[] = {{q, "q", nq},     {k, "k", nk},   {v, "v", nk},   {o, "o", nq},
             {d_o, "d_o", nq}, {dq, "dq", nq}, {dk, "dk", nk}, {dv, "dv", nk}};
  for (const auto& x : all)
    if (x.rows > 0)
      if (scn_status rc = check_heads(who, x.name, x.h, type)) return rc;
  if (nq == 0 && nk == 0) return SCN_OK;
  const size_t need = scn_cross_attn_bwd_workspace_bytes(type, nq, nk, batch, D, Hq, Hk);
  if (need && (!ws || (reinterpret_cast<uintptr_t>(ws) & 15) != 0 || ws_bytes < need)) {
    set_error("%s: workspace missing, misaligned or too small", who);
    return SCN_ERR_WORKSPACE;
  }
  const CrossBwdPlan p = plan(type, nq, nk, batch, D, Hk, Hq / Hk);
  if (type == SCN_BF16)
    return run<1>(make<1>(nq, nk, batch, q_ranges, k_ranges, D, Hq, Hk, q, k, v, o, lse, d_o, scale,
                          dq, dk, dv, p, ws), p, st);
  return run<3>(make<3>(nq, nk, batch, q_ranges, k_ranges, D, Hq, Hk, q, k, v, o, lse, d_o, scale,
                        dq, dk, dv, p, ws), p, st);
}

}  // extern "C"
