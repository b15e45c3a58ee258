// Attention within samples, forward: one pass over the keys that a tile of queries
// sees, with the running maximum and sum of the softmax.
//
// A block holds QB = 128 consecutive queries of one sample and head, 32 a wave, and
// takes their keys in tiles of 64 from LDS: first the sinks below the window, then the
// window from its first key.  Per tile and wave S^T = K Q^T has a query in each lane
// (its keys along the registers), so the maximum and the sum stay in the lane but for
// one exchange with the other half, and P^T goes on into O^T += V^T P^T as it is.
#include <cmath>

#include "attn.h"

namespace scn {
namespace {

constexpr int QB = 128, KB = 64, NT = 256;

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

// One row once more in fp32, over the keys that it sees and no others: two passes over
// its keys, a key per lane for the scores, channels along the lanes for the sum.
template <int NS>
__device__ inline void fwd_row(const FwdArgs<NS>& a, const Span& sp, int h, int i) {
  typedef Elem<NS> E;
  const int lane = threadIdx.x & 63;
  const auto* const q = a.q.p + (sp.base + i) * a.q.row + h * a.q.head;
  const auto* const k = a.k.p + sp.base * a.k.row + (h / a.group) * a.k.head;
  const auto* const v = a.v.p + sp.base * a.v.row + (h / a.group) * a.v.head;
  const int lo = a.w.lo(i), hi = a.w.hi(i, sp.m), ns = min(a.w.sinks, lo);
  const int cnt = ns + hi - lo + 1;  // the keys: [0, ns), then [lo, hi]
  auto score = [&](int x) -> float {
    const int j = x < ns ? x : lo + x - ns;
    return row_dot<NS>(q, k + j * a.k.row, a.D) * a.scale;
  };
  float top = -INFINITY, sum = 0.f, o0 = 0.f, o1 = 0.f;
  bool nan = false;
  for (int x0 = 0; x0 < cnt; x0 += 64) {
    const float s = x0 + lane < cnt ? score(x0 + lane) : -INFINITY;
    nan |= s != s;
    top = fmaxf(top, wave_max(s));
  }
  if (__ballot(nan)) top = NAN;
  for (int x0 = 0; x0 < cnt; x0 += 64) {
    const float p = x0 + lane < cnt ? expf(score(x0 + lane) - top) : 0.f;
    sum += wave_sum(p);
    for (int y = 0; y < min(64, cnt - x0); ++y) {
      const int x = x0 + y, j = x < ns ? x : lo + x - ns;
      const float py = __shfl(p, y);
      if (lane < a.D) o0 = fmaf(py, E::get(v[j * a.v.row + lane]), o0);
      if (64 + lane < a.D) o1 = fmaf(py, E::get(v[j * a.v.row + 64 + lane]), o1);
    }
  }
  auto* const o = a.o.p + (sp.base + i) * a.o.row + h * a.o.head;
  if (lane < a.D) o[lane] = E::put(o0 / sum);
  if (64 + lane < a.D) o[64 + lane] = E::put(o1 / sum);
  if (a.lse && lane == 0) a.lse[h * a.n + sp.base + i] = top + logf(sum);
}

template <int NS, int DP>
__global__ void __launch_bounds__(NT, NS == 3 && DP > 64 ? 1 : 2) attn_fwd_kernel(FwdArgs<NS> a) {
  typedef Tile<NS, DP, KB> L;
  constexpr int NBUF = NS == 1 ? 2 : 1;  // split tiles are three times as large
  extern __shared__ char smem[];
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % a.Hq;
  const Span sp = find_span<QB>(a.ranges, a.batch, a.n, blockIdx.x / a.Hq);
  if (sp.first >= sp.m) return;
  const int i0 = sp.first + wave * 32, i1 = min(i0 + 31, sp.m - 1);  // the wave's queries
  const int i = min(i0 + n32, sp.m - 1);                             // the lane's
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
  float top = -INFINITY, sum = 0.f;  // sum: of this half's keys

  // the block's keys: the sinks [0, ns), then the window [lo, hi]
  const int lo = a.w.lo(sp.first), hi = a.w.hi(min(sp.first + QB, sp.m) - 1, sp.m);
  const int ns = min(a.w.sinks, lo), nst = (ns + KB - 1) / KB;
  const int ntile = nst + (hi - lo + KB) / KB;
  const auto* const kp = a.k.p + sp.base * a.k.row + (h / a.group) * a.k.head;
  const auto* const vp = a.v.p + sp.base * a.v.row + (h / a.group) * a.v.head;
  Stage<NS, DP, KB, NT> sk, sv;
  auto fetch = [&](int t) {
    const int j0 = t < nst ? t * KB : lo + (t - nst) * KB, last = t < nst ? ns - 1 : hi;
    sk.load(kp, a.k.row, j0, last, a.D, tid);
    sv.load(vp, a.v.row, j0, last, a.D, tid);
  };
  fetch(0);
  sk.store(smem, tid);
  sv.store(smem + L::BYTES, tid);
  __syncthreads();
  for (int t = 0; t < ntile; ++t) {
    if (t + 1 < ntile) fetch(t + 1);
    char* const kt = smem + (NBUF == 2 ? (t & 1) * 2 * L::BYTES : 0);
    char* const vt = kt + L::BYTES;
    const bool sink = t < nst;
    const int j0 = sink ? t * KB : lo + (t - nst) * KB, last = sink ? ns - 1 : hi;
    // (a wave past the sample's rows has i1 < i0: nothing)
    const bool any = i0 <= i1 && j0 <= a.w.hi(i1, sp.m) &&
                     (sink || j0 + KB > a.w.lo(i0) || j0 < a.w.sinks);
    if (any) {
      const bool all = j0 + KB - 1 <= last &&
                       (sink || (j0 + KB - 1 <= i0 + a.w.right && j0 >= a.w.lo(i0 + 31)));
      v16f S[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        S[b] = zero16();
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) S[b] = mma<NS>(L::rows(kt, 32 * b, s, lane), Q[s], S[b]);
      }
      if (!all) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int j = j0 + 32 * b + 8 * (r / 4) + 4 * half + r % 4;
            if (!(j <= last && (sink || a.w.sees(i, j)))) S[b][r] = -INFINITY;
          }
      }
      float mx = S[0][0];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, S[b][r]);
      mx = fmaxf(mx, other_half(mx)) * c2;
      // The maximum moves only when a score passes it by 2^8: until then the terms
      // stay below 2^8 and the sums far from fp32's range.
      if (__ballot(mx > top + 8.f)) {
        const float now = fmaxf(top, mx);
        const float f = now == top ? 1.f : exp2f(top - now);
        top = now;
        sum *= f;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) O[d][r] *= f;
      }
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          S[b][r] = __builtin_amdgcn_exp2f(fmaf(S[b][r], c2, -base));
          sum += S[b][r];
        }
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = S[s / 2][8 * (s & 1) + j];
        const Frag<NS> P = to_frag<NS>(p);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
          O[d] = mma<NS>(L::cols(vt, 16 * s, d, lane), P, O[d]);
      }
    }
    if (t + 1 < ntile) {
      if (NBUF == 1) __syncthreads();
      char* const nx = smem + (NBUF == 2 ? ((t & 1) ^ 1) * 2 * L::BYTES : 0);
      sk.store(nx, tid);
      sv.store(nx + L::BYTES, tid);
      __syncthreads();
    }
  }
  sum += other_half(sum);
  const float inv = 1.f / sum;
  bool fine = fabsf(top) < INFINITY && sum < INFINITY;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) fine &= finite16(O[d]);
  const bool mine = i0 + n32 < sp.m;
  if (mine) {
    auto* const o = a.o.p + (sp.base + i) * a.o.row + h * a.o.head;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) store_cols<NS>(o, O[d], inv, d, a.D, lane);
    if (a.lse && half == 0) a.lse[h * a.n + sp.base + i] = (top + log2f(sum)) * LN2;
  }
  // A term that is infinite or NaN spoils sums it does not enter (0 times it is NaN)
  const uint64_t bad = __ballot(mine && !fine);
  uint32_t rows = (uint32_t)bad | (uint32_t)(bad >> 32);
  while (rows) {
    const int r = __builtin_ctz(rows);
    rows &= rows - 1;
    fwd_row<NS>(a, sp, h, i0 + r);
  }
}

template <int NS, int DP>
scn_status launch(const FwdArgs<NS>& a, hipStream_t st) {
  constexpr size_t smem = (NS == 1 ? 4 : 2) * Tile<NS, DP, KB>::BYTES;
  static LdsLimit limit;
  auto fn = attn_fwd_kernel<NS, DP>;
  if (scn_status rc = allow_lds(reinterpret_cast<const void*>(fn), limit, smem)) return rc;
  const int64_t blocks = (a.n / QB + a.batch) * a.Hq;
  if (blocks > INT32_MAX) {
    set_error("scn_attn_fwd: more than 2^31 blocks of rows and heads");
    return SCN_ERR_OVERFLOW;
  }
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(NT), smem, st, a);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
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
