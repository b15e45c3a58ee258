// Attention within samples, backward, in two passes that each own their sums, so that
// nothing is added atomically: one over tiles of queries for dq (and <do, o>, which
// the second pass needs), one over tiles of keys for dk and dv.  Both form the scores
// again from q, k and the forward's log sums.
//
// Queries' pass, as the forward: S^T = K Q^T and dP^T = V dO^T with a query per lane,
// dQ^T += K^T dS^T.  Keys' pass: S = Q K^T and dP = dO V^T with a key per lane,
// dV^T += dO^T P and dK^T += Q^T dS.
// A third kernel takes the queries that see the sinks from past their window, in
// shares that a fourth adds up in order.  P and dS are rounded to bf16 for their products
// (in three parts for fp32), all sums are in fp32.
//
// The waits between a tile's steps bound both passes: of the waves' cycles 26 to 41% go to
// loads and barriers and 20 to 33% to issuing, the vector unit issues in 25 to 44%, the
// matrix cores are busy in 25 to 31%.  60,007 rows, 4 heads of 64 channels, bf16, windows of
// 1025 rows and a sink: queries' pass 174 us, keys' pass 171, sinks 17 and 5.  34,567 rows, 4
// heads on 2 of 32 channels, fp32, 256 rows back and two sinks: 69, 90, 22 and 5 us.  30,000
// rows, 4 heads on 2 of 128 channels, bf16, windows of 1025: 158, 227, 25 and 5 us.  More
// keys a barrier (64 for 32), four waves side by side, or three waves a SIMD by spilling
// measure the same or worse.
#include "attn.h"

namespace scn {
namespace {

constexpr int SPLIT_SINKS = 256;

template <int NS>
struct BwdArgs {
  typedef typename Elem<NS>::T T;
  int64_t n;
  int batch, D, Hq, Hk, group;
  const int32_t* ranges;
  Heads<const T> q, k, v, o, d_o;
  Heads<T> dq, dk, dv;
  const float* lse;  // [Hq][n]
  float* delta;      // [Hq][n]
  float* lse2;       // [Hq][n]: lse in log 2, or NaN where it is past LSE_MOST ...
  float* rest;       // [Hq][n]: ... and what it lacks there
  float* share;      // the sinks' shares [chunk][Hk][sinks][2][D], or null
  int sc, cut;       // queries of a share; samples of more rows than cut have shares
  float scale;
  Window w;
};

// dq of one row once more in fp32, over the keys that it sees, from weights of its own.
// The keys' pass gets their delta, and what the row's lse is short of their log sum.
template <int NS>
__device__ inline void dq_row(const BwdArgs<NS>& a, const Span& sp, int h, int i) {
  typedef Elem<NS> E;
  const int lane = threadIdx.x & 63;
  const auto* const q = a.q.p + (sp.base + i) * a.q.row + h * a.q.head;
  const auto* const g = a.d_o.p + (sp.base + i) * a.d_o.row + h * a.d_o.head;
  const auto* const k = a.k.p + sp.base * a.k.row + (h / a.group) * a.k.head;
  const auto* const v = a.v.p + sp.base * a.v.row + (h / a.group) * a.v.head;
  const int lo = a.w.lo(i), hi = a.w.hi(i, sp.m), ns = min(a.w.sinks, lo);
  const int cnt = ns + hi - lo + 1;
  auto key = [&](int x) { return x < ns ? x : lo + x - ns; };
  auto score = [&](int x) { return row_dot<NS>(q, k + key(x) * a.k.row, a.D) * a.scale; };
  auto dp = [&](int x) { return row_dot<NS>(g, v + key(x) * a.v.row, a.D); };
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
      const auto* const kj = k + key(x0 + y) * a.k.row;
      const float d = __shfl(ds, y);
      if (lane < a.D) o0 = fmaf(d, E::get(kj[lane]), o0);
      if (64 + lane < a.D) o1 = fmaf(d, E::get(kj[64 + lane]), o1);
    }
  }
  auto* const o = a.dq.p + (sp.base + i) * a.dq.row + h * a.dq.head;
  if (lane < a.D) o[lane] = E::put(o0 * a.scale);
  if (64 + lane < a.D) o[64 + lane] = E::put(o1 * a.scale);
  if (lane == 0) {
    const int64_t at = h * a.n + sp.base + i;
    a.delta[at] = delta;
    a.rest[at] = (r.top - a.lse[at]) + logf(r.sum);
  }
}

// dk and dv of one row once more in fp32, over the queries that see it
template <int NS>
__device__ inline void dkv_row(const BwdArgs<NS>& a, const Span& sp, int hk, int j) {
  typedef Elem<NS> E;
  const int lane = threadIdx.x & 63;
  const auto* const k = a.k.p + (sp.base + j) * a.k.row + hk * a.k.head;
  const auto* const v = a.v.p + (sp.base + j) * a.v.row + hk * a.v.head;
  const int lo = max(0, j - a.w.right);
  const int hi = j < a.w.sinks ? sp.m - 1 : min(sp.m - 1, j + a.w.left);
  auto* const dk = a.dk.p + (sp.base + j) * a.dk.row + hk * a.dk.head;
  auto* const dv = a.dv.p + (sp.base + j) * a.dv.row + hk * a.dv.head;
  // a row of no weights (its lse is NaN) leaves nothing to add up
  bool none = false;
  for (int h = hk * a.group; h < (hk + 1) * a.group; ++h)
    for (int i = lo + lane; i <= hi; i += 64) {
      const float l = a.lse[h * a.n + sp.base + i];
      none |= l != l;
    }
  if (__ballot(none)) {
    for (int c = lane; c < a.D; c += 64) dk[c] = dv[c] = E::put(NAN);
    return;
  }
  float k0 = 0.f, k1 = 0.f, v0 = 0.f, v1 = 0.f;
  for (int h = hk * a.group; h < (hk + 1) * a.group; ++h) {
    const auto* const q = a.q.p + sp.base * a.q.row + h * a.q.head;
    const auto* const g = a.d_o.p + sp.base * a.d_o.row + h * a.d_o.head;
    for (int x0 = lo; x0 <= hi; x0 += 64) {
      float p = 0.f, ds = 0.f;
      const int i = x0 + lane;
      if (i <= hi) {
        const int64_t at = h * a.n + sp.base + i;
        p = row_dot<NS>(q + i * a.q.row, k, a.D) * a.scale - a.lse[at];
        p = expf(fabsf(a.lse[at]) <= LSE_MOST ? p : p - a.rest[at]);
        ds = p * (row_dot<NS>(g + i * a.d_o.row, v, a.D) - a.delta[at]);
      }
      for (int y = 0; y < min(64, hi - x0 + 1); ++y) {
        const float py = __shfl(p, y), dy = __shfl(ds, y);
        const auto* const qi = q + (x0 + y) * a.q.row;
        const auto* const gi = g + (x0 + y) * a.d_o.row;
        if (lane < a.D) {
          v0 = fmaf(py, E::get(gi[lane]), v0);
          k0 = fmaf(dy, E::get(qi[lane]), k0);
        }
        if (64 + lane < a.D) {
          v1 = fmaf(py, E::get(gi[64 + lane]), v1);
          k1 = fmaf(dy, E::get(qi[64 + lane]), k1);
        }
      }
    }
  }
  if (lane < a.D) {
    dk[lane] = E::put(k0 * a.scale);
    dv[lane] = E::put(v0);
  }
  if (64 + lane < a.D) {
    dk[64 + lane] = E::put(k1 * a.scale);
    dv[64 + lane] = E::put(v1);
  }
}

// QW waves of 32 queries by KW groups that share out the keys of a tile, 32 each
template <int NS, int DP, int QW, int KW>
struct QueryShape {
  static constexpr int QB = 32 * QW, NT = 64 * QW * KW, KT = 32 * KW;
  typedef Tile<NS, DP, KT> L;
  static constexpr size_t SMEM =
      std::max<size_t>(4 * L::BYTES, (size_t)QW * (KW - 1) * (DP / 32 * 16) * 256);
};

template <int NS, int DP, int QW, int KW>
__global__ void __launch_bounds__(64 * QW * KW, NS == 3 && DP > 32 ? 1 : 2)
    attn_dq_kernel(BwdArgs<NS> a) {
  typedef QueryShape<NS, DP, QW, KW> X;
  typedef typename X::L L;
  constexpr int KT = X::KT, NT = X::NT, QB = X::QB;
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kw = KW == 1 ? 0 : wave / QW;
  const int h = blockIdx.x % a.Hq;
  const Span sp = find_span(a.ranges, a.batch, a.n, blockIdx.x / a.Hq, QB);
  if (sp.first >= sp.m) return;
  const int i0 = sp.first + (wave - kw * QW) * 32, i1 = min(i0 + 31, sp.m - 1);
  const int i = min(i0 + n32, sp.m - 1);
  const bool mine = i0 + n32 < sp.m;
  const float c2 = a.scale * LOG2E;

  Frag<NS> Q[DP / 16], G[DP / 16];
  float delta = 0.f;
  {
    const auto* const q = a.q.p + (sp.base + i) * a.q.row + h * a.q.head;
    const auto* const g = a.d_o.p + (sp.base + i) * a.d_o.row + h * a.d_o.head;
    const auto* const o = a.o.p + (sp.base + i) * a.o.row + h * a.o.head;
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
  const int64_t at = h * a.n + sp.base + i;
  const float lse2 = a.lse[at] * LOG2E;
  const bool far = !(fabsf(a.lse[at]) <= LSE_MOST);  // the row is formed again ...
  const bool none = a.lse[at] != a.lse[at];           // ... if it has weights at all
  // <do, o> has the rounding of o to bf16, the same for all keys of a row, where the sum of
  // dS is 0 by definition.  (Left in, dq and dk are off by 1.7 to 4 times their own rounding
  // where a row sees few keys or few of its keys hold its weight.)  The sum of dS is
  // kept (`over`) and sets delta right for the keys' pass.  Up to 64 channels it is taken off
  // dQ as over P K at the end: 140 to 174 us at 60,007 rows of 4 heads, 64 channels, 1025
  // keys each.  Wider heads lack the registers (478 to 615 us for the gradients of 30,000
  // rows of 4 heads, 128 channels): blocks with a row where it counts take their keys again
  // with the delta set right.
  constexpr bool EXACT = NS == 1 && DP <= 64, AGAIN = NS == 1 && DP > 64;
  float over = 0.f, size = 0.f;
  v16f dQ[DP / 32], PK[EXACT ? DP / 32 : 1];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) dQ[d] = zero16();
  if constexpr (EXACT)
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) PK[d] = zero16();

  // the keys, as in the forward
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
  const typename L::Lane pl(lane);
  auto first_key = [&](int t) { return t < nst ? t * KT : lo + (t - nst) * KT; };
  auto fetch = [&](int t) {
    const int j = first_key(t), rows = (t < nst ? ns : hi + 1) - j;
    sk.load(kp, a.k.row, ko, j, rows, a.D);
    sv.load(vp, a.v.row, vo, j, rows, a.D);
  };
  auto put = [&](int t) {
    sk.store(smem + (t & 1) * 2 * L::BYTES, tid);
    sv.store(smem + (t & 1) * 2 * L::BYTES + L::BYTES, tid);
  };
  // S and dP of the wave's keys of tile t, at kt
  auto scores = [&](int t, char* kt, v16f& S, v16f& P) {
    const int j0 = first_key(t) + kw * 32;
    const bool sink = t < nst;
    char* const vt = kt + L::BYTES;
    S = P = zero16();
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) S = mma<NS>(L::rows(kt, pl, 0, s), Q[s], S);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) P = mma<NS>(L::rows(vt, pl, 0, s), G[s], P);
    if (sink ? j0 + 32 > ns : j0 < al || j0 + 31 > ah) {
      const int l = (sink ? 0 : a.w.lo(i)) - j0 - 4 * half;
      const int u = (sink ? ns - 1 : a.w.hi(i, sp.m)) - j0 - 4 * half;
      const int z = (sink ? 0 : a.w.sinks - j0) - 4 * half;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int e = 8 * (r / 4) + r % 4;
        S[r] = ((e <= u) & ((e >= l) | (e < z))) ? S[r] : -INFINITY;
      }
    }
  };
  auto tile = [&](int t) { return smem + (t & 1) * 2 * L::BYTES + kw * 32 * DP * 2; };
  auto take = [&](int t) {
    char* const kt = tile(t);
    v16f S, P;
    Frag<NS> KC[2][DP / 32];  // read early where the registers allow two waves only anyway
    if constexpr (EXACT) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) KC[s][d] = L::cols(kt, pl, 16 * s, d);
    }
    scores(t, kt, S, P);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      S[r] = __builtin_amdgcn_exp2f(fmaf(S[r], c2, -lse2));
      P[r] = S[r] * (P[r] - delta);
      if constexpr (EXACT || AGAIN) over += P[r];
      if constexpr (AGAIN) size += fabsf(P[r]);
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
  auto pass = [&](int t) {
    if (t + 1 < nt) put(t + 1);
    if (t + 2 < nt) fetch(t + 2);
  };
  auto place = [&](int x) { return nst + max(0, x - kw * 32) / KT; };
  const int some = i0 <= i1 && wh - lo >= kw * 32;
  const int e0 = i0 <= i1 ? nst : 0;
  const int s1 = some ? place(wl - lo) : nt, e1 = some ? place(wh - lo) + 1 : nt;
  auto sweep = [&](auto what) {
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
        what(t);
        __syncthreads();
      }
    }
    for (; t < nt; ++t) {
      pass(t);
      __syncthreads();
    }
  };
  // the sum over the row's groups of keys, in order
  auto joined = [&](float v) {
    v = both_sum(v);
    if constexpr (KW > 1) {
      float* const x = reinterpret_cast<float*>(smem) + lane;
      x[wave * 64] = v;
      __syncthreads();
      v = 0.f;
      for (int g = 0; g < KW; ++g) v += x[(g * QW + wave - kw * QW) * 64];
      __syncthreads();
    }
    return v;
  };
  sweep(take);
  if constexpr (EXACT) {
    over = joined(over);
    over = fabsf(over) < INFINITY ? over : 0.f;
    delta += over;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) dQ[d][r] = fmaf(-over, PK[d][r], dQ[d][r]);
  }
  if constexpr (AGAIN) {
    over = joined(over);
    size = joined(size);
    if (fabsf(over) < INFINITY) delta += over;
    // The threshold is what the rounding of dS leaves of it: rows of 1024 keys and scores of
    // N(0, 1.5) stay below, with N(0, 2) one in 200 is above, with N(0, 4) one in five.
    if (__syncthreads_or(fabsf(over) > 0x1p-9f * size)) {
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) dQ[d] = zero16();
      sweep(take);
    }
  }
  if (mine && half == 0 && kw == 0) {
    a.delta[at] = delta;
    a.lse2[at] = far ? NAN : lse2;  // keys that see the row are formed again
  }
  if constexpr (KW > 1) {
    float* const x = reinterpret_cast<float*>(smem) + lane;
    if (kw > 0)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          x[((wave - QW) * (DP / 32) * 16 + d * 16 + r) * 64] = dQ[d][r];
    __syncthreads();
    if (kw > 0) return;
    for (int g = 0; g < KW - 1; ++g)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          dQ[d][r] += x[((g * QW + wave) * (DP / 32) * 16 + d * 16 + r) * 64];
  }
  bool fine = true;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) fine &= finite16(dQ[d]);
  if constexpr (NS == 3) fine &= !tiny(dQ, 1.f);
  if (mine) {
    auto* const o = a.dq.p + (sp.base + i) * a.dq.row + h * a.dq.head;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) store_cols<NS>(o, dQ[d], a.scale, d, a.D, lane);
  }
  const uint64_t bad = __ballot(mine && !none && (far || !fine));
  uint32_t rows = (uint32_t)bad | (uint32_t)(bad >> 32);
  for (; rows; rows &= rows - 1) dq_row<NS>(a, sp, h, i0 + __builtin_ctz(rows));
}

// What a wave with 32 keys does with 32 queries of a tile: dV += P^T dO, dK += dS^T Q
// (transposed).  see(i, j) masks the pairs of query i0 + row and key j if `mask`.  EARLY
// reads each pair of products' operands ahead of them, for some 60 registers more.
template <int NS, int DP, int TB, bool EARLY, class See>
__device__ inline void key_block(char* qt, char* gt, const typename Tile<NS, DP, TB>::Lane& pl,
                                 const float* lse2, const float* delta, int r0,
                                 const Frag<NS> (&K)[DP / 16], const Frag<NS> (&V)[DP / 16],
                                 float c2, bool mask, const See& see, v16f (&dK)[DP / 32],
                                 v16f (&dV)[DP / 32]) {
  typedef Tile<NS, DP, TB> L;
  const int lane = threadIdx.x & 63, half = lane >> 5;
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
  if (mask) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      S[r] = see(r0 + 8 * (r / 4) + 4 * half + r % 4) ? S[r] : -INFINITY;
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

// The tiles of queries that stream past a block's keys, over its query heads
template <int NS, int DP, int TB, int THREADS>
struct QueryTiles {
  typedef Tile<NS, DP, TB> L;
  static constexpr int BUF = 2 * L::BYTES + 2 * TB * 4;
  typedef Stage<NS, DP, TB, THREADS> St;
  St q, g;
  uint32_t qo[St::N], go[St::N];
  float lse2, delta;
  __device__ inline void init(const BwdArgs<NS>& a, int tid) {
    St::places(qo, a.q.row, a.D, tid);
    St::places(go, a.d_o.row, a.D, tid);
  }
  __device__ inline void fetch(const BwdArgs<NS>& a, const Span& sp, int h, int i0, int last,
                               int tid) {
    q.load(a.q.p + sp.base * a.q.row + h * a.q.head, a.q.row, qo, i0, last + 1 - i0, a.D);
    g.load(a.d_o.p + sp.base * a.d_o.row + h * a.d_o.head, a.d_o.row, go, i0, last + 1 - i0, a.D);
    if (tid < TB) {
      const int64_t at = h * a.n + sp.base + min(i0 + tid, last);
      lse2 = a.lse2[at];
      delta = a.delta[at];
    }
  }
  __device__ inline void store(char* b, int tid) const {
    q.store(b, tid);
    g.store(b + L::BYTES, tid);
    if (tid < TB) {
      float* const f = reinterpret_cast<float*>(b + 2 * L::BYTES);
      f[tid] = lse2;
      f[TB + tid] = delta;
    }
  }
};

// Sinks are seen by every later query, so a block that owned them would run far longer
// than the others.  Their pairs past the window go here, in shares of sc queries:
// block (chunk, sink tile of 32, key head), two waves with 32 queries of each tile.
template <int NS, int DP>
__global__ void __launch_bounds__(128, 1) attn_sink_kernel(BwdArgs<NS> a, int nst) {
  constexpr int TB = 64;
  typedef QueryTiles<NS, DP, TB, 128> QT;
  typedef typename QT::L L;
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hk = blockIdx.x % a.Hk, j0 = blockIdx.x / a.Hk % nst * 32;
  const int chunk = blockIdx.x / a.Hk / nst;
  const Span sp = find_span(a.ranges, a.batch, a.n, chunk, a.sc, a.cut);
  const int ns = a.w.sinks;
  const int end = min(sp.first + a.sc, sp.m) - 1;       // the share's queries
  const int first = max(sp.first, j0 + a.w.left + 1);   // ... past the window of j0
  if (sp.m <= a.cut || sp.first >= sp.m || first > end) return;
  const int j = min(j0 + n32, ns - 1);
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
  QT st;
  st.init(a, tid);
  const typename L::Lane pl(lane);
  const int per = (end - first + TB) / TB, ntile = per * a.group;
  st.fetch(a, sp, hk * a.group, first, end, tid);
  for (int t = 0; t < ntile; ++t) {
    st.store(smem, tid);
    __syncthreads();
    const int i0 = first + t % per * TB;
    if (t + 1 < ntile)
      st.fetch(a, sp, hk * a.group + (t + 1) / per, first + (t + 1) % per * TB, end, tid);
    const float* const f = reinterpret_cast<const float*>(smem + 2 * L::BYTES);
    auto see = [&](int r) { return (i0 + r <= end) & (j < i0 + r - a.w.left); };
    key_block<NS, DP, TB, false>(smem, smem + L::BYTES, pl, f, f + TB, 32 * wave, K, V, c2, true, see,
                                 dK, dV);
    __syncthreads();
  }
  // the second wave's sums through LDS, then out
  float* const x = reinterpret_cast<float*>(smem);
  if (wave == 1)
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[(d * 16 + r) * 64 + lane] = dK[d][r];
        x[((DP / 32 + d) * 16 + r) * 64 + lane] = dV[d][r];
      }
  __syncthreads();
  if (wave == 1 || j0 + n32 >= ns) return;
  float* const out =
      a.share + (((int64_t)chunk * a.Hk + hk) * a.w.sinks + j) * 2 * a.D;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int c = 32 * d + 8 * (r / 4) + 4 * half + r % 4;
      if (c < a.D) {
        out[c] = dK[d][r] + x[(d * 16 + r) * 64 + lane];
        out[a.D + c] = dV[d][r] + x[((DP / 32 + d) * 16 + r) * 64 + lane];
      }
    }
}

// A sink's shares, added up in order into the first of them: block (sample of more than cut
// rows, head, sink), an element a thread.
template <int NS>
__global__ void __launch_bounds__(256) attn_share_kernel(BwdArgs<NS> a) {
  const int j = blockIdx.x % a.w.sinks, hk = blockIdx.x / a.w.sinks % a.Hk;
  const Span sp = find_span(a.ranges, a.batch, a.n, blockIdx.x / a.w.sinks / a.Hk, INT32_MAX, a.cut);
  if ((int)threadIdx.x >= 2 * a.D || sp.m <= a.cut || sp.first > 0) return;
  const int far = (j & ~31) + a.w.left + 1;  // the first query past the window
  const int64_t step = (int64_t)a.Hk * a.w.sinks * 2 * a.D;
  float* const p =
      a.share + (int64_t)(tile_start((int)sp.base, sp.sample, a.sc, a.cut) + far / a.sc) * step +
      ((int64_t)hk * a.w.sinks + j) * 2 * a.D + threadIdx.x;
  const int n = (sp.m + a.sc - 1) / a.sc - far / a.sc;
  float s = 0.f;
  int c = 0;
  for (; c + 8 <= n; c += 8) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = p[(c + e) * step];
#pragma unroll
    for (int e = 0; e < 8; ++e) s += x[e];
  }
  for (; c < n; ++c) s += p[c * step];
  *p = s;
}

// KW waves of 32 keys by QW groups that share out the queries of a tile, 32 U each.  The
// groups' sums join in LDS at the end.
template <int NS, int DP, int KW, int QW, int U>
struct KeyShape {
  static constexpr int KB = 32 * KW, NT = 64 * KW * QW, TB = 32 * U * QW;
  typedef QueryTiles<NS, DP, TB, NT> QT;
  static constexpr int JOIN = DP / 32 * 32;  // floats a lane hands over
  static constexpr size_t SMEM =
      std::max<size_t>(2 * QT::BUF, (size_t)KW * (QW - 1) * JOIN * 256);
};

template <int NS, int DP, int KW, int QW, int U>
__global__ void __launch_bounds__(64 * KW * QW, NS == 3 || DP > 64 ? 1 : 2)
    attn_dkv_kernel(BwdArgs<NS> a) {
  typedef KeyShape<NS, DP, KW, QW, U> X;
  constexpr int KB = X::KB, TB = X::TB;
  // 183 to 174 us at 60,007 rows of 4 heads; narrower heads lose 1%, the others lack the
  // registers, as do four groups
  constexpr bool EARLY = NS == 1 && DP == 64 && QW < 4;
  typedef typename X::QT QT;
  typedef typename QT::L L;
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), qw = QW == 1 ? 0 : wave / KW;
  const int hk = blockIdx.x % a.Hk;
  const Span sp = find_span(a.ranges, a.batch, a.n, blockIdx.x / a.Hk, KB);
  if (sp.first >= sp.m) return;
  const int j0 = sp.first + (wave - qw * KW) * 32, j1 = min(j0 + 31, sp.m - 1);  // the wave's keys
  const int j = min(j0 + n32, sp.m - 1);
  const float c2 = a.scale * LOG2E;
  // sinks whose far queries other blocks have taken are ordinary keys here
  const bool shared = a.share && sp.m > a.cut;
  const int sinks = shared ? 0 : a.w.sinks;
  const Window w{a.w.left, a.w.right, sinks};

  Frag<NS> K[DP / 16], V[DP / 16];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    K[s] = load_frag<NS>(a.k.p + (sp.base + j) * a.k.row + hk * a.k.head, s, a.D, lane);
    V[s] = load_frag<NS>(a.v.p + (sp.base + j) * a.v.row + hk * a.v.head, s, a.D, lane);
  }
  v16f dK[DP / 32], dV[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) dK[d] = dV[d] = zero16();

  const int first = max(0, sp.first - w.right);
  const int end = sp.first < sinks ? sp.m - 1
                                   : min(sp.m - 1, min(sp.first + KB, sp.m) - 1 + w.left);
  const int per = (end - first + TB) / TB, ntile = per * a.group;
  QT st;
  st.init(a, tid);
  const typename L::Lane pl(lane);
  auto fetch = [&](int t) {
    st.fetch(a, sp, hk * a.group + t / per, first + t % per * TB, end, tid);
  };
  auto put = [&](int t) { st.store(smem + (t & 1) * QT::BUF, tid); };
  auto pass = [&](int t) {
    if (t + 1 < ntile) put(t + 1);
    if (t + 2 < ntile) fetch(t + 2);
  };
  // The wave takes the tiles [s, e) of each query head: the queries that see one of its
  // keys.
  const int q0 = qw * 32 * U;  // the wave's queries of a tile
  const int ql = max(0, j0 - w.right) - first - q0;
  const int qh = (j0 < sinks ? sp.m - 1 : min(sp.m - 1, j1 + w.left)) - first - q0;
  const bool some = j0 <= j1 && qh >= 0;
  const int s = some ? min(per, max(0, ql) / TB) : per, e = some ? min(per, qh / TB + 1) : per;
  fetch(0);
  put(0);
  if (ntile > 1) fetch(1);
  __syncthreads();
  for (int t = 0; t < ntile;) {
    const int t0 = t;
    for (; t < t0 + s; ++t) {
      pass(t);
      __syncthreads();
    }
    for (; t < t0 + e; ++t) {
      pass(t);
      char* const b = smem + (t & 1) * QT::BUF;
      const float* const f = reinterpret_cast<const float*>(b + 2 * L::BYTES);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i0 = first + (t - t0) * TB + q0 + 32 * u, i1 = i0 + 31;
        const bool all = i1 <= end && j0 + 31 <= i0 + w.right && j0 >= i1 - w.left;
        auto see = [&](int r) {
          const int i = i0 - q0 - 32 * u + r;
          return (i <= end) & (j <= i + w.right) & ((j >= i - w.left) | (j < sinks));
        };
        key_block<NS, DP, TB, EARLY>(b, b + L::BYTES, pl, f, f + TB, q0 + 32 * u, K, V, c2, !all,
                                     see, dK, dV);
      }
      __syncthreads();
    }
    for (; t < t0 + per; ++t) {
      pass(t);
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
  const bool mine = j0 + n32 < sp.m;
  if (shared && mine && j < a.w.sinks) {
    const int far = (j & ~31) + a.w.left + 1;  // first query past the window of the sink tile
    // where their sum lies
    const int64_t c = tile_start((int)sp.base, sp.sample, a.sc, a.cut) + far / a.sc;
    const float* const p = a.share + ((c * a.Hk + hk) * a.w.sinks + j) * 2 * a.D;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int ch = 32 * d + 8 * g + 4 * half;
        if (ch >= a.D) continue;
        const v4f x = *reinterpret_cast<const v4f*>(p + ch);
        const v4f y = *reinterpret_cast<const v4f*>(p + a.D + ch);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          dK[d][4 * g + e] += x[e];
          dV[d][4 * g + e] += y[e];
        }
      }
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
  while (rows) {
    const int r = __builtin_ctz(rows);
    rows &= rows - 1;
    dkv_row<NS>(a, sp, hk, j0 + r);
  }
}

// Sinks get their own blocks when a window ends before them (a left bound) and they
// are few; many sinks keep the blocks of their keys busy anyway.  So do those of samples
// with fewer than SPLIT_SINKS queries past the window (gradients of 2000 samples of 50
// rows, 16 sinks: 435 us against 638 with blocks of their own; 800 of 125 in fp32: 329 against
// 370).
bool split_sinks(int64_t n, int64_t left, int64_t sinks) {
  return left >= 0 && left < n && sinks > 0 && sinks <= SPLIT_SINKS;
}
int sink_cut(int64_t left) { return (int)left + SPLIT_SINKS; }
// Shares of at least 256 queries (some tiles' work for a block), and not more than about
// 256 of them to add up.
int share_rows(int64_t n) {
  int sc = 256;
  while (n / sc > 256) sc *= 2;
  return sc;
}
int64_t sink_chunks(int64_t n, int batch, int64_t left) {
  return ceil_div(n, share_rows(n)) + std::min<int64_t>(batch, n / sink_cut(left));
}

template <int NS, int DP, int KW, int QW, int U>
scn_status launch_dkv(const BwdArgs<NS>& a, hipStream_t st) {
  typedef KeyShape<NS, DP, KW, QW, U> X;
  static LdsLimit limit;
  auto fn = attn_dkv_kernel<NS, DP, KW, QW, U>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, X::SMEM)) return rc;
  const int64_t blocks = (a.n / X::KB + a.batch) * a.Hk;
  if (blocks > INT32_MAX) {
    set_error("scn_attn_bwd: more than 2^31 blocks of rows and heads");
    return SCN_ERR_OVERFLOW;
  }
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(X::NT), X::SMEM, st, a);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}

template <int NS, int DP, int QW, int KW>
scn_status launch_dq(const BwdArgs<NS>& a, hipStream_t st) {
  typedef QueryShape<NS, DP, QW, KW> X;
  static LdsLimit limit;
  auto fn = attn_dq_kernel<NS, DP, QW, KW>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, X::SMEM)) return rc;
  const int64_t blocks = (a.n / X::QB + a.batch) * a.Hq;
  if (blocks > INT32_MAX) {
    set_error("scn_attn_bwd: more than 2^31 blocks of rows and heads");
    return SCN_ERR_OVERFLOW;
  }
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(X::NT), X::SMEM, st, a);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}

template <int NS, int DP>
scn_status launch_sinks(const BwdArgs<NS>& a, hipStream_t st) {
  const int nst = (a.w.sinks + 31) / 32;
  const int64_t blocks = sink_chunks(a.n, a.batch, a.w.left) * a.Hk * nst;
  const int64_t sums = std::min<int64_t>(a.batch, a.n / a.cut) * a.Hk * a.w.sinks;
  if (std::max(blocks, sums) > INT32_MAX) {
    set_error("scn_attn_bwd: more than 2^31 blocks of sinks and heads");
    return SCN_ERR_OVERFLOW;
  }
  constexpr size_t smem = std::max<size_t>(QueryTiles<NS, DP, 64, 128>::BUF, DP * 2 * 32 * 4);
  static LdsLimit limit;
  auto fn = attn_sink_kernel<NS, DP>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, smem)) return rc;
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(128), smem, st, a, nst);
  SCN_LAUNCH_CHECK();
  hipLaunchKernelGGL(attn_share_kernel<NS>, dim3((unsigned)sums), dim3(256), 0, st, a);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}

// The shapes, by measurement (us; queries' pass, keys' pass):
//  - Two waves by two groups serve most: four waves side by side and no groups are better
//    in the keys' pass once there are over a thousand blocks of 128 keys (60,007 rows of 4
//    heads, 64 channels: 188 against 207 before the reads ahead), and with more than 64
//    channels, where two groups' tiles and sums crowd the registers (30,000 rows of 2 key
//    heads, 128 channels: 223 against 272).  The queries' pass of wide heads does so from
//    512 blocks of 128 queries on (forward and gradients: 511 against 522 at 30,000 rows of 4
//    heads, 158 against 142 at 2000).
//  - Few blocks, counted against the query heads that each has to take in turn: a wave's
//    32 keys by four groups (2000 rows of 4 heads: 54 to 27; 32,001 rows, 4 heads on one:
//    310 to 190).
//  - fp32, 64 channels: four waves by two groups in the queries' pass (20,000 rows of 4
//    heads: 381 to 300).
template <int NS, int DP>
scn_status launch(const BwdArgs<NS>& a, hipStream_t st) {
  const int64_t tiles = a.n / 128 + a.batch;
  scn_status rc;
  if constexpr (NS == 3 && DP > 64) {
    rc = launch_dq<NS, DP, 4, 1>(a, st);
  } else if constexpr (NS == 3 && DP == 64) {
    rc = launch_dq<NS, DP, 4, 2>(a, st);
  } else {
    constexpr int QW = DP > 64 ? 4 : 2, KW = DP > 64 ? 1 : 2;
    rc = tiles * a.Hq < 512 ? launch_dq<NS, DP, 2, 2>(a, st) : launch_dq<NS, DP, QW, KW>(a, st);
  }
  if (rc) return rc;
  if (a.share && (rc = launch_sinks<NS, DP>(a, st))) return rc;
  const int64_t blocks = tiles * a.Hk;
  if constexpr (NS == 3) {
    if constexpr (DP <= 64)
      return launch_dkv<NS, DP, 2, 2, 1>(a, st);
    else
      return launch_dkv<NS, DP, 4, 1, 1>(a, st);
  } else {
    if constexpr (DP <= 64)
      if (blocks < 128 * a.group) return launch_dkv<NS, DP, 1, 4, 1>(a, st);
    if (blocks < (DP <= 64 ? 1024 : 384)) return launch_dkv<NS, DP, 2, 2, 1>(a, st);
    return launch_dkv<NS, DP, 4, 1, 2>(a, st);
  }
}

template <int NS>
scn_status run(const BwdArgs<NS>& a, hipStream_t st) {
  if (a.D <= 32) return launch<NS, 32>(a, st);
  if (a.D <= 64) return launch<NS, 64>(a, st);
  if (a.D <= 96) return launch<NS, 96>(a, st);
  return launch<NS, 128>(a, st);
}

int64_t delta_floats(int64_t n, int Hq) { return (n * Hq + 63) & ~int64_t(63); }

}  // namespace
}  // namespace scn

using namespace scn;

extern "C" {

size_t scn_attn_bwd_workspace_bytes(int64_t n, int32_t batch, int32_t D, int32_t Hq, int32_t Hk,
                                    int64_t left, int64_t sinks) {
  if (n <= 0 || n > ATTN_ROWS || batch < 1 || D < 1 || D > ATTN_D || Hq < 1 || Hk < 1 || sinks < 0)
    return 0;
  int64_t f = 3 * delta_floats(n, Hq);
  if (split_sinks(n, left, sinks))
    f += sink_chunks(n, batch, left) * Hk * std::min(sinks, n) * 2 * D;
  return (size_t)f * 4;
}

scn_status scn_attn_bwd(int32_t type, int64_t n, int32_t batch, const int32_t* ranges, int32_t D,
                        int32_t Hq, int32_t Hk, const scn_heads* q, const scn_heads* k,
                        const scn_heads* v, const scn_heads* o, const float* lse,
                        const scn_heads* d_o, float scale, int64_t left, int64_t right,
                        int64_t sinks, const scn_heads* dq, const scn_heads* dk,
                        const scn_heads* dv, void* ws, size_t ws_bytes, hipStream_t st) {
  clear_error();
  const char* const who = "scn_attn_bwd";
  if (scn_status rc = check_attn(who, type, n, batch, ranges, D, Hq, Hk, scale)) return rc;
  if (sinks < 0 || (n > 0 && !lse)) {
    set_error("%s: negative number of sinks, or lse is null", who);
    return SCN_ERR_INVALID;
  }
  if (n == 0) return SCN_OK;
  const struct {
    const scn_heads* h;
    const char* name;
  } all[] = {{q, "q"}, {k, "k"}, {v, "v"}, {o, "o"}, {d_o, "d_o"}, {dq, "dq"}, {dk, "dk"},
             {dv, "dv"}};
  for (const auto& x : all)
    if (scn_status rc = check_heads(who, x.name, x.h, type)) return rc;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 15) != 0 ||
      ws_bytes < scn_attn_bwd_workspace_bytes(n, batch, D, Hq, Hk, left, sinks)) {
    set_error("%s: workspace missing, misaligned or too small", who);
    return SCN_ERR_WORKSPACE;
  }
  float* const delta = static_cast<float*>(ws);
  float* const lse2 = delta + delta_floats(n, Hq);
  float* const rest = lse2 + delta_floats(n, Hq);
  const int cut = split_sinks(n, left, sinks) ? sink_cut(left) : 0;
  float* const share = cut && n > cut ? rest + delta_floats(n, Hq) : nullptr;
  const Window w{bound(left, n), bound(right, n), bound(sinks, n)};
  if (type == SCN_BF16) {
    typedef uint16_t T;
    return run<1>(BwdArgs<1>{n, batch, D, Hq, Hk, Hq / Hk, ranges, view<const T>(q),
                             view<const T>(k), view<const T>(v), view<const T>(o),
                             view<const T>(d_o), view<T>(dq), view<T>(dk), view<T>(dv), lse, delta,
                             lse2, rest, share, share_rows(n), cut, scale, w}, st);
  }
  typedef float T;
  return run<3>(BwdArgs<3>{n, batch, D, Hq, Hk, Hq / Hk, ranges, view<const T>(q),
                           view<const T>(k), view<const T>(v), view<const T>(o),
                           view<const T>(d_o), view<T>(dq), view<T>(dk), view<T>(dv), lse, delta,
                           lse2, rest, share, share_rows(n), cut, scale, w}, st);
}

}  // extern "C"
