// Cross attention, backward, in two passes that each own their sums (attn_bwd.hip), without
// a window and with both axes split where the blocks are few: one over tiles of queries
// for dq and <do, o>, one over tiles of keys for dk and dv.
//
// Queries' pass: S^T = K Q^T and dP^T = V dO^T with a tile row per lane (cross.h),
// dQ^T += K^T dS^T.  Keys' pass: S = Q K^T and dP = dO V^T with a key per lane,
// dV^T += dO^T P and dK^T += Q^T dS over the queries of each head in turn.
// Split axes leave their sums in a workspace, and a join kernel adds them up in order.
//
// Seven products where the mathematics takes five (S and dP twice), for sums without atomics.
// On long samples the passes wait to issue and for data by turns: one sample of 16,384 rows and
// states, 2 bf16 heads of 128, 809 and 726 us and 47 for the joins, 434 TFLOP/s by the flops of
// five; 120,011 rows of 4 fp32 heads on 2 of 32 over 40 states: 81 and 69 us.
#include "cross.h"

namespace scn {
namespace {

template <int NS>
struct CrossBwdArgs {
  typedef typename Elem<NS>::T T;
  Deal qdeal;  // tiles of queries, parts of their keys
  Deal kdeal;  // tiles of keys, parts of their queries
  int D, group;
  int repeat;  // tiles of queries that a work is, where the keys are few
  Heads<const T> q, k, v, o, d_o;
  Heads<T> dq, dk, dv;
  const float* lse;  // [Hq][nq]
  float* delta;      // [Hq][nq]
  float* lse2;       // [Hq][nq]: lse in log 2, or NaN where it is past LSE_MOST ...
  float* rest;       // [Hq][nq]: ... and what it lacks there
  float scale;
  float* qpart;  // [Hq][nq][parts][2][D] (dQ, PK), then [Hq][nq][parts] (the sum of dS)
  float* kpart;  // [Hk][nk][parts][2][D] (dK, dV)
  __device__ inline int64_t at(int64_t row, int h) const { return h * qdeal.tiles.n + row; }
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
    const int64_t at = a.at(row, h);
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
      const float l = a.lse[a.at(q0 + i, h)];
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
        const int64_t at = a.at(q0 + i, h);
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

// where the sums of dS lie that parts of the keys leave
template <int NS>
__device__ inline float* over_part(const CrossBwdArgs<NS>& a) {
  return a.qpart + a.qdeal.tiles.n * a.qdeal.Hk * a.group * a.qdeal.parts.most * 2 * a.D;
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

// FEW: a work is several tiles of queries in turn
template <int NS, int DP, int QW, int KW, bool FEW>
__global__ void __launch_bounds__(64 * QW * KW, (NS == 3 && DP > 32) || DP > 64 ? 1 : 2)
    cross_dq_kernel(CrossBwdArgs<NS> a) {
  typedef QueryShape<NS, DP, QW, KW> X;
  typedef typename X::L L;
  constexpr int KT = X::KT, NT = X::NT, QB = X::QB;
  constexpr bool EXACT = X::EXACT;
  constexpr bool TWO = NS == 1 && (FEW || QW == 1);  // few terms, or few rows: low_part
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kw = KW == 1 ? 0 : wave / QW;
  const float c2 = a.scale * LOG2E;
  typedef Stage<NS, DP, KT, NT> St;
  uint32_t ko[St::N], vo[St::N];
  St::places(ko, a.k.row, a.D, tid);
  St::places(vo, a.v.row, a.D, tid);
  const typename L::Lane pl(lane);

  const Work w = a.qdeal.find(blockIdx.x);
  if (w.first >= w.m) return;
  const int mk = w.mo, hk = w.hk;
  const int64_t k0 = w.other;
  Frag<NS> Q[DP / 16], G[DP / 16];
  v16f dQ[DP / 32], PK[EXACT ? DP / 32 : 1];
  float delta, lse2, over;

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
      Frag<NS> low;
      if constexpr (TWO) low = low_part(y, Y);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        const Frag<NS> K = EXACT ? KC[s][d] : L::cols(kt, pl, 16 * s, d);
        if constexpr (TWO) dQ[d] = mma<NS>(K, low, dQ[d]);
        dQ[d] = mma<NS>(K, Y, dQ[d]);
        if constexpr (EXACT) PK[d] = mma<NS>(K, X, PK[d]);
      }
    }
  };
  // Works of several tiles load the next one's rows while they take one.
  constexpr bool PRE = FEW && DP <= 32;
  Ahead<NS, PRE ? DP : 16> nq, ng, no;
  float nl;
  auto ahead = [&](int first) {
    const int r = min(first + (wave - kw * QW) * 32 + n32, w.m - 1);
    const int h = hk * a.group + r % a.group;
    const int64_t row = w.base + r / a.group;
    nq.load(a.q.p + row * a.q.row + h * a.q.head, a.D, lane);
    ng.load(a.d_o.p + row * a.d_o.row + h * a.d_o.head, a.D, lane);
    no.load(a.o.p + row * a.o.row + h * a.o.head, a.D, lane);
    nl = a.lse[a.at(row, h)];
  };
  auto sweep = [&](int first, bool stage) {
    const int r = first + (wave - kw * QW) * 32 + n32;
    const bool mine = r < w.m;
    const int rr = min(r, w.m - 1);
    const int64_t row = w.base + rr / a.group;
    const int h = hk * a.group + rr % a.group;
    delta = over = 0.f;
    float lse;
    auto dot8 = [&](const float (&x)[8], const float (&y)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = fmaf(x[j], y[j], delta);
    };
    if constexpr (PRE) {
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) {
        Q[s] = nq.frag(s);
        G[s] = ng.frag(s);
        float x[8], y[8];
        ng.floats(s, x);
        no.floats(s, y);
        dot8(x, y);
      }
      lse = nl;
      ahead(first + QB);
    } else {
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
          dot8(x, y);
        }
      }
      lse = a.lse[a.at(row, h)];
    }
    delta = both_sum(delta);
    const int64_t at = a.at(row, h);
    lse2 = lse * LOG2E;
    const bool far = !(fabsf(lse) <= LSE_MOST);  // the row is formed again ...
    const bool none = lse != lse;                 // ... if it has weights at all
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) dQ[d] = zero16();
    if constexpr (EXACT)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) PK[d] = zero16();
    // the keys, as in cross_fwd.hip
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
    if (w.parts > 1) {
      if (mine) {
        const int64_t to = at * a.qdeal.parts.most + w.part;
        float* const o = a.qpart + to * 2 * a.D;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
          store_cols<3>(o, dQ[d], 1.f, d, a.D, lane);
          if constexpr (EXACT) store_cols<3>(o + a.D, PK[d], 1.f, d, a.D, lane);
        }
        if (half == 0) {
          over_part(a)[to] = over;
          if (w.part == 0) {
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
    const int w0 = first + wave * 32;
    for (; rows; rows &= rows - 1) {
      const int x = w0 + __builtin_ctz(rows);
      dq_row<NS>(a, w.base + x / a.group, hk * a.group + x % a.group, k0, mk);
    }
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

// A block's threads over `rows` rows of `wide` floats, four a thread, and what threads are left
// over the rows' parts: each thread's share of the parts of its floats, then all of them, in order, in
// the threads of slice 0.
struct Slices {
  int c, r, sl, slices, lanes, rows;
  __device__ inline Slices(int wide, int rows_) : rows(rows_) {
    lanes = wide >> 2;
    slices = (int)blockDim.x / (lanes * rows);
    c = threadIdx.x % lanes * 4;
    r = threadIdx.x / lanes % rows;
    sl = threadIdx.x / (lanes * rows);
  }
  // part s of the thread's floats lies at p[s * step]
  __device__ inline v4f sum(const float* p, int64_t step, int n, v4f* x, bool on) const {
    v4f v = {0.f, 0.f, 0.f, 0.f};
    const int per = (n + slices - 1) / slices, s1 = min(n, (sl + 1) * per);
    if (on)
      for (int s0 = sl * per; s0 < s1; s0 += 4) {
        v4f o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          o[j] = *reinterpret_cast<const v4f*>(p + min(s0 + j, s1 - 1) * step);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (s0 + j < s1) v += o[j];
      }
    if (slices > 1) {
      x[threadIdx.x] = v;
      __syncthreads();
      if (on && sl == 0)
        for (int s = 1; s < slices; ++s) v += x[s * lanes * rows + threadIdx.x];
      __syncthreads();
    }
    return v;
  }
};
// attn.h's tiny, and what is not finite, of four of a row's floats
template <int NS>
__device__ inline bool fine4(v4f v) {
  bool fine = true, large = false, any = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    fine &= fabsf(v[j]) < INFINITY;
    large |= fabsf(v[j]) >= 0x1p-95f;
    any |= v[j] != 0.f;
  }
  return fine && (NS == 1 || large || !any);
}
template <int NS>
__device__ inline void store4(typename Elem<NS>::T* p, v4f v, float f) {
  if constexpr (NS == 1)
    *reinterpret_cast<v2u*>(p) = v2u{cvt2_bf16(v[0] * f, v[1] * f), cvt2_bf16(v[2] * f, v[3] * f)};
  else
    *reinterpret_cast<v4f*>(p) = v4f{v[0] * f, v[1] * f, v[2] * f, v[3] * f};
}

// The parts of the rows' dq: `qdeal.rows` tile rows a block
template <int NS>
__global__ void __launch_bounds__(256) cross_dq_join_kernel(CrossBwdArgs<NS> a, Parts parts) {
  __shared__ v4f x[256];
  __shared__ bool bad[128];
  const Work w = a.qdeal.find(blockIdx.x);
  const int n = parts.of(w.mo);
  if (w.first >= w.m || n == 1) return;
  const Slices z(a.D, a.qdeal.rows);
  const bool on = z.sl < z.slices && w.first + z.r < w.m;
  const int rr = min(w.first + z.r, w.m - 1), h = w.hk * a.group + rr % a.group;
  const int64_t row = w.base + rr / a.group, at = a.at(row, h);
  const float* const p = a.qpart + at * parts.most * 2 * a.D + z.c;
  if (threadIdx.x < 128) bad[threadIdx.x] = false;
  v4f d = z.sum(p, 2 * a.D, n, x, on);
  if constexpr (NS == 1) {
    const v4f k = z.sum(p + a.D, 2 * a.D, n, x, on);
    if (on && z.sl == 0) {
      const float* const o =
          a.qpart + a.qdeal.tiles.n * a.qdeal.Hk * a.group * parts.most * 2 * a.D + at * parts.most;
      float over = 0.f;
      for (int s = 0; s < n; ++s) over += o[s];
      over = fabsf(over) < INFINITY ? over : 0.f;
      if (z.c == 0) a.delta[at] += over;
#pragma unroll
      for (int j = 0; j < 4; ++j) d[j] = fmaf(-over, k[j], d[j]);
    }
  }
  __syncthreads();
  if (on && z.sl == 0) {
    store4<NS>(a.dq.p + row * a.dq.row + h * a.dq.head + z.c, d, a.scale);
    const float l = a.lse[at];
    // (a row without weights stays, one past LSE_MOST takes weights of its own)
    if (l == l && (!(fabsf(l) <= LSE_MOST) || !fine4<NS>(d))) bad[z.r] = true;
  }
  __syncthreads();
  for (int i = threadIdx.x >> 6; i < min(z.rows, w.m - w.first); i += 4)
    if (bad[i]) {
      const int y = w.first + i;
      dq_row<NS>(a, w.base + y / a.group, w.hk * a.group + y % a.group, w.other, w.mo);
    }
}

// What a wave with 32 keys does with 32 queries of a tile: dV += P^T dO, dK += dS^T Q
// (transposed).  Queries past the sample's last have a log sum of +inf, and so no weight.
// EARLY reads each pair of products' operands ahead of them, for some 60 registers more.
template <int NS, int DP, int TB, bool EARLY, bool TWO>
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
    Frag<NS> xl, yl;
    if constexpr (TWO) {
      xl = low_part(x, X);
      yl = low_part(y, Y);
    }
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      const Frag<NS> G = EARLY ? GC[s][d] : L::cols(gt, pl, r0 + 16 * s, d);
      const Frag<NS> Q = EARLY ? QC[s][d] : L::cols(qt, pl, r0 + 16 * s, d);
      if constexpr (TWO) {
        dV[d] = mma<NS>(G, xl, dV[d]);
        dK[d] = mma<NS>(Q, yl, dK[d]);
      }
      dV[d] = mma<NS>(G, X, dV[d]);
      dK[d] = mma<NS>(Q, Y, dK[d]);
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

template <int NS, int DP, int KW, int QW, int U, bool TWO>
__global__ void __launch_bounds__(64 * KW * QW, NS == 3 || DP > 64 ? 1 : 2)
    cross_dkv_kernel(CrossBwdArgs<NS> a) {
  typedef KeyShape<NS, DP, KW, QW, U> X;
  typedef typename X::L L;
  typedef typename X::St St;
  constexpr int TB = X::TB;
  constexpr bool EARLY = NS == 1 && DP == 64 && QW < 4 && !TWO;
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), qw = QW == 1 ? 0 : wave / KW;
  const float c2 = a.scale * LOG2E;
  uint32_t qo[St::N], go[St::N];
  St::places(qo, a.q.row, a.D, tid);
  St::places(go, a.d_o.row, a.D, tid);
  const typename L::Lane pl(lane);

  const Work w = a.kdeal.find(blockIdx.x);
  if (w.first >= w.m) return;
  const int mq = w.mo, hk = w.hk;
  const int64_t q0 = w.other;
  const int j = min(w.first + (wave - qw * KW) * 32 + n32, w.m - 1);  // the lane's key
  const bool mine = w.first + (wave - qw * KW) * 32 + n32 < w.m;

  Frag<NS> K[DP / 16], V[DP / 16];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    K[s] = load_frag<NS>(a.k.p + (w.base + j) * a.k.row + hk * a.k.head, s, a.D, lane);
    V[s] = load_frag<NS>(a.v.p + (w.base + j) * a.v.row + hk * a.v.head, s, a.D, lane);
  }
  v16f dK[DP / 32], dV[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) dK[d] = dV[d] = zero16();

  // the block's tiles of queries, those of each head in turn
  const int per = (mq + TB - 1) / TB;
  const int64_t nt = (int64_t)per * a.group, share = (nt + w.parts - 1) / w.parts;
  const int64_t t0 = min(nt, w.part * share), t1 = min(nt, t0 + share);
  St sq, sg;
  float lse2 = 0.f, delta = 0.f;
  int h = per > 0 ? hk * a.group + (int)(t0 / per) : 0;  // of the next tile to fetch
  int i0 = per > 0 ? (int)(t0 % per) * TB : 0;
  auto fetch = [&]() {
    sq.load(a.q.p + q0 * a.q.row + h * a.q.head, a.q.row, qo, i0, mq - i0, a.D);
    sg.load(a.d_o.p + q0 * a.d_o.row + h * a.d_o.head, a.d_o.row, go, i0, mq - i0, a.D);
    if (tid < TB) {
      const int64_t at = a.at(q0 + min(i0 + tid, mq - 1), h);
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
        key_block<NS, DP, TB, EARLY, TWO>(b, b + L::BYTES, pl, f, f + TB, (qw * U + u) * 32, K, V, c2, dK,
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
  if (w.parts > 1) {
    if (mine) {
      float* const o =
          a.kpart + ((hk * a.kdeal.tiles.n + w.base + j) * a.kdeal.parts.most + w.part) * 2 * a.D;
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
    auto* const dk = a.dk.p + (w.base + j) * a.dk.row + hk * a.dk.head;
    auto* const dv = a.dv.p + (w.base + j) * a.dv.row + hk * a.dv.head;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      store_cols<NS>(dk, dK[d], a.scale, d, a.D, lane);
      store_cols<NS>(dv, dV[d], 1.f, d, a.D, lane);
    }
  }
  const uint64_t bad = __ballot(mine && !fine);
  uint32_t rows = (uint32_t)bad | (uint32_t)(bad >> 32);
  const int64_t w0 = w.base + w.first + wave * 32;
  for (; rows; rows &= rows - 1) dkv_row<NS>(a, w0 + __builtin_ctz(rows), hk, q0, mq);
}

// The parts of the keys' dk and dv: `kdeal.rows` keys a block
template <int NS>
__global__ void __launch_bounds__(256) cross_dkv_join_kernel(CrossBwdArgs<NS> a, Parts parts) {
  __shared__ v4f x[256];
  __shared__ bool bad[128];
  const Work w = a.kdeal.find(blockIdx.x);
  const int n = parts.of(w.mo * (int64_t)a.group);
  if (w.first >= w.m || n == 1) return;
  const Slices z(2 * a.D, a.kdeal.rows);
  const bool on = z.sl < z.slices && w.first + z.r < w.m;
  const int64_t row = w.base + min(w.first + z.r, w.m - 1);
  const float* const p =
      a.kpart + (w.hk * a.kdeal.tiles.n + row) * parts.most * 2 * a.D + z.c;
  if (threadIdx.x < 128) bad[threadIdx.x] = false;
  const v4f d = z.sum(p, 2 * a.D, n, x, on);
  __syncthreads();
  if (on && z.sl == 0) {
    if (z.c < a.D)
      store4<NS>(a.dk.p + row * a.dk.row + w.hk * a.dk.head + z.c, d, a.scale);
    else
      store4<NS>(a.dv.p + row * a.dv.row + w.hk * a.dv.head + z.c - a.D, d, 1.f);
    if (!fine4<NS>(d)) bad[z.r] = true;
  }
  __syncthreads();
  for (int i = threadIdx.x >> 6; i < min(z.rows, w.m - w.first); i += 4)
    if (bad[i]) dkv_row<NS>(a, w.base + w.first + i, w.hk, w.other, w.mo);
}

// Shapes and parts of both passes, by rules on sizes alone (cross_fwd.hip).  Both sides of each, as
// whole calls in us, the rule's first:
//  - Few keys stay in LDS for several tiles of queries: the case of 40 states above 85, and 133
//    loading them for each; 2,000 rows of 32 samples on 40, 4 fp32 heads on 2 of 32, 92 in four
//    waves side by side and 116 in two by two.
//  - Queries' pass of more than 64 bf16 channels, two by two below 512 blocks: 8 samples of 400
//    states, 4 heads of 128, 500 rows 48 and 53, 1,000 rows 101 and 89; four waves from there:
//    2,000 rows 153 and 179, 4,000 rows 265 and 321.
//  - Keys' pass to 64 bf16 channels, one wave of keys below 128 blocks: 2 samples of 300 rows on
//    400 states, 4 heads on 1 of 64, 28 and 30 with two, 33 with four; 2,000 rows of 32 samples on
//    40 states 99 and 82 with two.  Two below 1,024: 8 samples of 300 rows on 1,000 states, 2 key
//    heads, 58, 65 with one and 55 with four.  Four from there: 4,000 states, 4 key heads, 99, 136
//    and 109.
//  - Past 64 channels, two below 384: 8 samples of 300 rows on 1,000 states, 2 key heads of 128,
//    115 and 104, of 2,000 rows 339 and 341; four from there: 4,000 states, 4 key heads, 242 and
//    272.
//  - fp32 heads to 32 channels, one wave for 32 keys or fewer: 2,000 rows of 32 samples on 32
//    states 91 and 83 with two; two past them: on 40 states 92 and 123 with one.
struct CrossBwdPlan {
  int qw, qkw, repeat;  // queries' pass: waves of queries, groups of keys; tiles of a work
                        // where the keys are few, or 0
  int kw;               // keys' pass: waves of keys (the others share out the queries)
  bool two;             // ... few of which need their weights in two parts
  Parts qparts, kparts;
};
CrossBwdPlan plan(int type, int64_t nq, int64_t nk, int batch, int D, int Hk, int group) {
  CrossBwdPlan p;
  const int usedq = (int)std::max<int64_t>(1, std::min<int64_t>(batch, nq));
  const int usedk = (int)std::max<int64_t>(1, std::min<int64_t>(batch, nk));
  const int64_t rows = ceil_div(nq * group, usedq), keys = ceil_div(nk, usedk);
  auto qblocks = [&](int b) { return usedq * ceil_div(rows, b) * Hk; };
  auto kblocks = [&](int b) { return usedk * ceil_div(keys, b) * Hk; };
  const bool bf16 = type == SCN_BF16;
  if (rows <= 32 && bf16) {
    p.qw = 1;
    p.qkw = 4;
  } else if (!bf16) {
    p.qw = D > 32 || keys <= 64 ? 4 : 2;
    p.qkw = D > 64 || keys <= 64 ? 1 : 2;
  } else {
    p.qw = keys <= 64 || (D > 64 && qblocks(128) >= 512) ? 4 : 2;
    p.qkw = p.qw == 4 ? 1 : 2;
  }
  p.qparts = cut(qblocks(32 * p.qw), 1024, nk / usedq, 512, usedq);
  p.repeat = 0;
  if (p.qkw == 1 && keys <= 64)
    p.repeat = (int)std::max<int64_t>(1, std::min<int64_t>(8, qblocks(32 * p.qw) / FEW_BLOCKS));
  p.two = bf16 && nq * group / usedk <= 128;
  if (!bf16) {
    p.kw = keys <= 32 && D <= 32 ? 1 : D <= 64 ? 2 : 4;
  } else if (p.two) {
    p.kw = 2;
  } else {
    p.kw = D <= 64 && (keys <= 32 || kblocks(128) < 128) ? 1
           : kblocks(128) < (D <= 64 ? 1024 : 384)       ? 2
                                                         : 4;
  }
  p.kparts = cut(kblocks(32 * p.kw), 1024, nq * group / usedk, 512, usedk);
  return p;
}

scn_status too_many() {
  set_error("scn_cross_attn_bwd: more than 2^31 blocks of rows and heads");
  return SCN_ERR_OVERFLOW;
}
// Tile rows of a join's block: as many as leave the card some thousand blocks, of at most 256
// threads
Deal join_deal(Deal d, int wide) {
  d.parts = Parts{1, INT32_MAX};
  d.rows = 1;
  while (d.rows * 2 * (wide / 4) <= 256 && d.tiles.n * d.tiles.many * d.Hk / (d.rows * 2) >= 1024)
    d.rows *= 2;
  return d;
}

template <int NS, int DP, int QW, int KW, bool FEW = false>
scn_status launch_dq(CrossBwdArgs<NS> a, const CrossBwdPlan& p, hipStream_t st) {
  typedef QueryShape<NS, DP, QW, KW> X;
  static LdsLimit limit;
  auto fn = cross_dq_kernel<NS, DP, QW, KW, FEW>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, X::SMEM)) return rc;
  a.qdeal.rows = X::QB * std::max(1, a.repeat);
  const int64_t blocks = a.qdeal.blocks();
  if (blocks > INT32_MAX) return too_many();
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(X::NT), X::SMEM, st, a);
  SCN_LAUNCH_CHECK();
  if (p.qparts.most > 1) {
    a.qdeal = join_deal(a.qdeal, a.D);
    hipLaunchKernelGGL(cross_dq_join_kernel<NS>, dim3((unsigned)a.qdeal.blocks()),
                       dim3(256), 0, st, a, p.qparts);
    SCN_LAUNCH_CHECK();
  }
  return SCN_OK;
}

template <int NS, int DP, int KW, int QW, int U, bool TWO>
scn_status launch_dkv(CrossBwdArgs<NS> a, const CrossBwdPlan& p, hipStream_t st) {
  typedef KeyShape<NS, DP, KW, QW, U> X;
  static LdsLimit limit;
  auto fn = cross_dkv_kernel<NS, DP, KW, QW, U, TWO>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, X::SMEM)) return rc;
  a.kdeal.rows = X::KB;
  const int64_t blocks = a.kdeal.blocks();
  if (blocks > INT32_MAX) return too_many();
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(X::NT), X::SMEM, st, a);
  SCN_LAUNCH_CHECK();
  if (p.kparts.most > 1) {
    a.kdeal = join_deal(a.kdeal, 2 * a.D);
    hipLaunchKernelGGL(cross_dkv_join_kernel<NS>, dim3((unsigned)a.kdeal.blocks()),
                       dim3(256), 0, st, a, p.kparts);
    SCN_LAUNCH_CHECK();
  }
  return SCN_OK;
}

template <int NS, int DP>
scn_status launch(const CrossBwdArgs<NS>& a, const CrossBwdPlan& p, hipStream_t st) {
  scn_status rc = SCN_OK;
  if (a.qdeal.tiles.n > 0) {
    if (p.qkw == 1) {
      if constexpr (DP <= 64)  // (narrow heads take four waves side by side for few keys alone)
        rc = launch_dq<NS, DP, 4, 1, true>(a, p, st);
      else
        rc = p.repeat ? launch_dq<NS, DP, 4, 1, true>(a, p, st) : launch_dq<NS, DP, 4, 1>(a, p, st);
    } else if constexpr (NS == 1) {
      rc = p.qw == 1 ? launch_dq<NS, DP, 1, 4>(a, p, st) : launch_dq<NS, DP, 2, 2>(a, p, st);
    } else if constexpr (DP <= 64) {
      rc = launch_dq<NS, DP, (DP > 32 ? 4 : 2), 2>(a, p, st);
    }
  }
  if (rc || a.kdeal.tiles.n == 0) return rc;
  if constexpr (NS == 3) {
    if constexpr (DP <= 32)
      if (p.kw == 1) return launch_dkv<NS, DP, 1, 4, 1, false>(a, p, st);
    if constexpr (DP <= 64)
      return launch_dkv<NS, DP, 2, 2, 1, false>(a, p, st);
    else
      return launch_dkv<NS, DP, 4, 1, 1, false>(a, p, st);
  } else {
    if (p.two) return launch_dkv<NS, DP, 2, 2, 1, true>(a, p, st);
    if constexpr (DP <= 64)
      if (p.kw == 1) return launch_dkv<NS, DP, 1, 4, 1, false>(a, p, st);
    if (p.kw == 2) return launch_dkv<NS, DP, 2, 2, 1, false>(a, p, st);
    return launch_dkv<NS, DP, 4, 1, 2, false>(a, p, st);
  }
}

template <int NS>
scn_status run(const CrossBwdArgs<NS>& a, const CrossBwdPlan& p, hipStream_t st) {
  if (a.D <= 32) return launch<NS, 32>(a, p, st);
  if (a.D <= 64) return launch<NS, 64>(a, p, st);
  if (a.D <= 96) return launch<NS, 96>(a, p, st);
  return launch<NS, 128>(a, p, st);
}

// floats of the workspace: the rows' statistics, then the parts of dq, or those of dk and dv
// (each of use to one pass and its join alone, so they lie in the same place)
int64_t stat_floats(int64_t nq, int Hq) { return (nq * Hq + 63) & ~int64_t(63); }
int64_t part_floats(const CrossBwdPlan& p, int64_t nq, int64_t nk, int Hq, int Hk, int D) {
  const int64_t q = p.qparts.most > 1 ? nq * Hq * p.qparts.most * (2 * D + 1) : 0;
  const int64_t k = p.kparts.most > 1 ? nk * Hk * p.kparts.most * 2 * D : 0;
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
  const Side qs{qr, nq, Hq / Hk}, ks{kr, nk, 1};
  return CrossBwdArgs<NS>{Deal{qs, ks, batch, 0, Hk, p.qparts, false},
                          Deal{ks, qs, batch, 0, Hk, p.kparts, false},
                          D, Hq / Hk, p.repeat, view<const T>(q), view<const T>(k), view<const T>(v),
                          view<const T>(o), view<const T>(d_o), view<T>(dq), view<T>(dk),
                          view<T>(dv), lse, f, f + n, f + 2 * n, scale, f + 3 * n, f + 3 * n};
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
