// Attention of one new token of each stream over its cache: the sinks and the last
// positions of the ring, each row read once.  Memory bounds it (two flops a byte and
// query head).  A stream's rows are split over blocks where there are few streams; the
// parts' outputs, maxima and sums join in a second kernel, always in the same order.
// Measured, reading the visible rows: 128 streams of 2064 rows, 8 heads on 2 of 64
// channels, bf16: 29 us, 3.9 TB/s (64 channels' rows lie 256 bytes apart); one stream of
// 262,144 rows, 4 heads of 32, fp32: 47 us, 5.7 TB/s.
#include "attn.h"

namespace scn {
namespace {

constexpr int NT = 256;
constexpr int U = 4;  // rows of a lane group in flight
constexpr int MAX_SPLITS = 1024;

struct Ring {
  int64_t stream, row, head;
};

template <int NS>
struct StepArgs {
  typedef typename Elem<NS>::T T;
  int streams, cap, D, Hq, Hk, group, passes, splits;
  Heads<const T> q, k, v;
  T *kc, *vc;
  Ring ks, vs;
  const int32_t* length;
  float scale;
  int reach, sinks;
  Heads<T> o;
  float* part;  // [stream][Hq][split][D + 2]: output, maximum, sum; null if splits == 1
};

// m, l: maximum and sum of the terms that o holds.  A side without terms has
// m = -inf and l = 0.
__device__ inline void join(float& m, float& l, float m2, float l2, float& f, float& f2) {
  const float t = fmaxf(m, m2);
  const float b = t == -INFINITY ? 0.f : t;
  f = __builtin_amdgcn_exp2f(m - b);
  f2 = __builtin_amdgcn_exp2f(m2 - b);
  l = l * f + l2 * f2;
  m = t;
}

// One stream's head once more in fp32, term by term, by W waves (this is wave w; all of a
// block if W > 1, which hands over in `x`): the maximum and the sum first, a key per lane,
// then the values by their weights, channels along the lanes.  For results that came out
// infinite or NaN (an infinite value that the token sees, but also one that a weight's low
// part, or a zero that fills a tile, was multiplied with), and for bf16 scores whose weights
// all ended at 0 or infinity (attn.h: SUM_LEAST).
template <int NS, int W>
__device__ inline void step_row(const StepArgs<NS>& a, int s, int h, int w, float* x) {
  typedef Elem<NS> E;
  const int lane = threadIdx.x & 63, hk = h / a.group;
  const int p = min(max(0, a.length[s]), INT32_MAX - 1);
  const int lo = min(p + 1, max(a.sinks, p - a.reach)), ns = min(a.sinks, p + 1);
  const int cnt = ns + p - lo + 1, ring = a.cap - a.sinks;
  const int r0 = lo < a.sinks ? 0 : (lo - a.sinks) % ring;
  const auto* const q = a.q.p + s * a.q.row + h * a.q.head;
  // the i-th key's row: the token's own (the last) as it came, the others in the cache
  auto row = [&](int i, const Ring& r, const typename E::T* cache,
                 const Heads<const typename E::T>& now) {
    const int y = r0 + i - ns;
    const int64_t t = i < ns ? i : a.sinks + (y < ring ? y : y - ring);
    return i == cnt - 1 ? now.p + s * now.row + hk * now.head
                        : cache + s * r.stream + hk * r.head + t * r.row;
  };
  auto score = [&](int i) { return row_dot<NS>(q, row(i, a.ks, a.kc, a.k), a.D) * a.scale; };
  RowSum r;
  for (int64_t i = w * 64 + lane; i < cnt; i += 64 * W) r.add(score((int)i));
  r.join();
  if constexpr (W > 1) {
    if (lane == 0) {
      x[w] = r.top;
      x[W + w] = r.sum;
    }
    __syncthreads();
    if (lane < W) r = RowSum{x[lane], x[W + lane]};
    else r = RowSum{};
    r.join();
    __syncthreads();
  }
  float o0 = 0.f, o1 = 0.f;
  for (int64_t i0 = w * 64; i0 < cnt; i0 += 64 * W) {
    const int n = (int)min<int64_t>(64, cnt - i0);
    const float weight = lane < n ? r.weight(score((int)i0 + lane)) : 0.f;
    for (int y = 0; y < n; ++y) {
      const auto* const v = row((int)i0 + y, a.vs, a.vc, a.v);
      const float wy = __shfl(weight, y);
      if (lane < a.D) o0 = fmaf(wy, E::get(v[lane]), o0);
      if (64 + lane < a.D) o1 = fmaf(wy, E::get(v[64 + lane]), o1);
    }
  }
  if constexpr (W > 1) {
    x[w * 128 + lane] = o0;
    x[w * 128 + 64 + lane] = o1;
    __syncthreads();
    if (w > 0) return;
    for (int g = 1; g < W; ++g) {
      o0 += x[g * 128 + lane];
      o1 += x[g * 128 + 64 + lane];
    }
  }
  auto* const o = a.o.p + s * a.o.row + h * a.o.head;
  if (lane < a.D) o[lane] = E::put(o0);
  if (64 + lane < a.D) o[64 + lane] = E::put(o1);
}

// fp32, on the vector unit: LP lanes hold a key's channels, eight a lane, and take GC query
// heads of the key head while its row is in registers.  Each group of LP lanes keeps a
// running maximum, sum and output of its own, which join within the wave and the block.
template <int NS, int LP, int GC>
__global__ void __launch_bounds__(NT) attn_step_kernel(StepArgs<NS> a) {
  typedef Elem<NS> E;
  typedef typename E::T T;
  constexpr int KW = 64 / LP;         // keys of a wave at once
  constexpr int KB = KW * (NT / 64);  // ... of the block
  __shared__ float red[NT / 64][GC][LP * 8 + 2];
  __shared__ bool bad[GC];
  const int split = blockIdx.x % a.splits, pass = blockIdx.x / a.splits % a.passes;
  const int hk = blockIdx.x / a.splits / a.passes % a.Hk;
  const int s = blockIdx.x / a.splits / a.passes / a.Hk;
  const int h0 = hk * a.group + pass * GC, nh = min(GC, a.group - pass * GC);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = lane % LP * 8;
  const bool on = c < a.D;
  const int p = min(max(0, a.length[s]), INT32_MAX - 1);
  // the visible positions: [0, ns), then [lo, p], lo in the ring's row r0
  const int lo = min(p + 1, max(a.sinks, p - a.reach)), ns = min(a.sinks, p + 1);
  const int cnt = ns + p - lo + 1, ring = a.cap - a.sinks;
  const int r0 = lo < a.sinks ? 0 : (lo - a.sinks) % ring;
  const int per = (cnt + a.splits - 1) / a.splits;
  const int x0 = min(cnt, split * per), x1 = min(cnt, x0 + per);
  const T* const kn = a.k.p + s * a.k.row + hk * a.k.head;
  const T* const vn = a.v.p + s * a.v.row + hk * a.v.head;
  T* const kc = a.kc + s * a.ks.stream + hk * a.ks.head;
  T* const vc = a.vc + s * a.vs.stream + hk * a.vs.head;
  auto slot = [&](int x) -> int64_t {
    const int y = r0 + x - ns;
    return x < ns ? x : a.sinks + (y < ring ? y : y - ring);
  };

  float q[GC][8], o[GC][8], m[GC], l[GC];
#pragma unroll
  for (int g = 0; g < GC; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) q[g][j] = o[g][j] = 0.f;
    if (on && g < nh) load8<NS>(a.q.p + s * a.q.row + (h0 + g) * a.q.head + c, q[g]);
#pragma unroll
    for (int j = 0; j < 8; ++j) q[g][j] *= a.scale * LOG2E;
  }
  for (int x = x0 + wave * KW + lane / LP; x - lane / LP < x1; x += KB * U) {
    float kk[U][8], vv[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int y = x + u * KB;
#pragma unroll
      for (int j = 0; j < 8; ++j) kk[u][j] = vv[u][j] = 0.f;
      if (on && y < x1) {
        // the new token's row is not in the cache yet
        const bool now = y == cnt - 1;
        const int64_t t = slot(y);
        load8<NS>((now ? kn : kc + t * a.ks.row) + c, kk[u]);
        load8<NS>((now ? vn : vc + t * a.vs.row) + c, vv[u]);
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
      const float f = __builtin_amdgcn_exp2f(m[g] - b);
      m[g] = top;
      l[g] *= f;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[g][j] *= f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float e = __builtin_amdgcn_exp2f(sc[u] - b);
        l[g] += e;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[g][j] = fmaf(e, vv[u][j], o[g][j]);
      }
    }
  }
  // the lane groups of the wave, then the waves
#pragma unroll
  for (int g = 0; g < GC; ++g) {
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
  for (int i = tid; i < nh * a.D; i += NT) {
    const int g = i / a.D, ch = i % a.D;
    float mm = red[0][g][LP * 8], ll = red[0][g][LP * 8 + 1], v = red[0][g][ch], f, f2;
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) {
      join(mm, ll, red[w][g][LP * 8], red[w][g][LP * 8 + 1], f, f2);
      v = v * f + red[w][g][ch] * f2;
    }
    if (a.splits == 1) {
      v /= ll;
      red[0][g][ch] = v;
      if (!(fabsf(v) < INFINITY || ll != ll)) bad[g] = true;
    } else {
      float* const out = a.part + (((int64_t)s * a.Hq + h0 + g) * a.splits + split) * (a.D + 2);
      out[ch] = v;
      if (ch == 0) {
        out[a.D] = mm;
        out[a.D + 1] = ll;
      }
    }
  }
  if (a.splits == 1) {
    __syncthreads();
    for (int i = tid; i < nh * a.D; i += NT) {
      const int g = i / a.D, ch = i % a.D;
      if (!bad[g]) a.o.p[s * a.o.row + (h0 + g) * a.o.head + ch] = E::put(red[0][g][ch]);
    }
    for (int g = wave; g < nh; g += NT / 64)
      if (bad[g]) step_row<NS, 1>(a, s, h0 + g, 0, nullptr);
  }
  // The new rows go to the cache.  No block reads that row: what it held is a
  // capacity's ring before the new token, past the reach.
  if (split == 0 && pass == 0 && tid < a.D) {
    const int64_t t = slot(cnt - 1);
    kc[t * a.ks.row + tid] = kn[tid];
    vc[t * a.vs.row + tid] = vn[tid];
  }
}

// bf16, on matrix cores: the query heads of a key head are the columns of the
// forward's products, up to 32 of them, and a wave takes 32 cache rows at a time through
// its own part of LDS.  A row then costs the same whether one head or 32 read it, where
// the kernel above takes 28 vector instructions a lane for each (16 heads on one of 128
// channels, 64 streams of 4096 rows: 109 us that way, 28 this way).
template <int DP>
__global__ void __launch_bounds__(NT, 2) attn_step_wide_kernel(StepArgs<1> a) {
  typedef uint16_t T;
  typedef Tile<1, DP, 32> L;
  typedef Stage<1, DP, 32, 64> St;
  constexpr int JOIN = DP / 32 * 16 + 2;
  constexpr int WAVES = NT / 64;
  __shared__ __align__(16) char smem[std::max(WAVES * 2 * L::BYTES, (WAVES - 1) * JOIN * 256)];
  const int split = blockIdx.x % a.splits, pass = blockIdx.x / a.splits % a.passes;
  const int hk = blockIdx.x / a.splits / a.passes % a.Hk;
  const int s = blockIdx.x / a.splits / a.passes / a.Hk;
  const int h0 = hk * a.group + pass * 32, nh = min(32, a.group - pass * 32);
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int p = __builtin_amdgcn_readfirstlane(min(max(0, a.length[s]), INT32_MAX - 1));
  const float c2 = a.scale * LOG2E;
  // What the new token sees, in runs of cache rows: the sinks, the ring's part up to its
  // end, the part from its begin, and the token's own row, which is not in the cache yet.
  const int ring = a.cap - a.sinks;
  const int lo = min(p, max(a.sinks, p - a.reach)), ns = min(a.sinks, p);
  const int old = p - lo, r0 = old > 0 ? (lo - a.sinks) % ring : 0;
  const int nb = min(old, ring - r0), nc = old - nb;
  const int ta = (ns + 31) / 32, tb = ta + (nb + 31) / 32, tc = tb + (nc + 31) / 32;
  const int per = (tc + a.splits) / a.splits;  // of tc + 1 tiles
  const int t1 = min(tc + 1, (split + 1) * per);
  const T* const kn = a.k.p + s * a.k.row + hk * a.k.head;
  const T* const vn = a.v.p + s * a.v.row + hk * a.v.head;
  T* const kc = a.kc + s * a.ks.stream + hk * a.ks.head;
  T* const vc = a.vc + s * a.vs.stream + hk * a.vs.head;

  Frag<1> Q[DP / 16];
#pragma unroll
  for (int c = 0; c < DP / 16; ++c) {
    Q[c].s[0] = v4u{0, 0, 0, 0};
    if (n32 < nh) Q[c] = load_frag<1>(a.q.p + s * a.q.row + (h0 + n32) * a.q.head, c, a.D, lane);
  }
  v16f O[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) O[d] = zero16();
  float top = -INFINITY, base = 0.f, sum = 0.f;
  St sk, sv;
  uint32_t ko[St::N], vo[St::N];
  St::places(ko, a.ks.row, a.D, lane);
  St::places(vo, a.vs.row, a.D, lane);
  const typename L::Lane at(lane);
  auto fetch = [&](int t) -> int {
    // tile t's rows
    int row, n;
    if (t < ta) {
      row = t * 32;
      n = ns - row;
    } else if (t < tb) {
      row = a.sinks + r0 + (t - ta) * 32;
      n = nb - (t - ta) * 32;
    } else if (t < tc) {
      row = a.sinks + (t - tb) * 32;
      n = nc - (t - tb) * 32;
    } else {
      sk.load(kn, 0, ko, 0, 1, a.D);
      sv.load(vn, 0, vo, 0, 1, a.D);
      return 1;
    }
    sk.load(kc, a.ks.row, ko, row, n, a.D);
    sv.load(vc, a.vs.row, vo, row, n, a.D);
    return min(n, 32);
  };
  char* const kt = smem + wave * 2 * L::BYTES;
  char* const vt = kt + L::BYTES;
  int n = 0, t = split * per + wave;
  if (t < t1) n = fetch(t);
  for (; t < t1; t += WAVES) {
    sk.store(kt, lane);
    sv.store(vt, lane);
    const int now = n;
    if (t + WAVES < t1) n = fetch(t + WAVES);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    v16f S = zero16();
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) S = mma<1>(L::rows(kt, at, 0, c), Q[c], S);
    if (now < 32)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        S[r] = 8 * (r / 4) + 4 * half + r % 4 < now ? S[r] : -INFINITY;
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
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = S[8 * e + j];
      // The weights keep 16 bits, in two parts: the matrix cores have time to spare
      // here, and one stream's output is all that a step gives.
      Frag<1> P[2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t hi = cvt2_bf16(x[2 * j], x[2 * j + 1]);
        P[0].s[0][j] = hi;
        P[1].s[0][j] = cvt2_bf16(x[2 * j] - __uint_as_float(hi << 16),
                                 x[2 * j + 1] - __uint_as_float(hi & 0xffff0000u));
      }
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        const Frag<1> V = L::cols(vt, at, 16 * e, d);
        O[d] = mma<1>(V, P[1], O[d]);
        O[d] = mma<1>(V, P[0], O[d]);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  sum = both_sum(sum);
  // the waves, joined in order
  float* const x = reinterpret_cast<float*>(smem) + lane;
  __syncthreads();
  if (wave > 0) {
    float* const o = x + (wave - 1) * JOIN * 64;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[(d * 16 + r) * 64] = O[d][r];
    o[(JOIN - 2) * 64] = top;
    o[(JOIN - 1) * 64] = sum;
  }
  __syncthreads();
  if (wave == 0) {
    bool fine = true;
    for (int g = 0; g < WAVES - 1; ++g) {
      const float* const o = x + g * JOIN * 64;
      float f, f2;
      join(top, sum, o[(JOIN - 2) * 64], o[(JOIN - 1) * 64], f, f2);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[d][r] = O[d][r] * f + o[(d * 16 + r) * 64] * f2;
    }
    if (n32 < nh) {
      if (a.splits == 1) {
        const float inv = 1.f / sum;
        T* const o = a.o.p + s * a.o.row + (h0 + n32) * a.o.head;
        fine = fabsf(top) < INFINITY && sum > SUM_LEAST && sum < SUM_MOST;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
          fine &= finite16(O[d]);
          store_cols<1>(o, O[d], inv, d, a.D, lane);
        }
        fine |= a.D == DP && nan_score(top, sum);  // NaN, as it stands
      } else {
        float* const o =
            a.part + (((int64_t)s * a.Hq + h0 + n32) * a.splits + split) * (a.D + 2);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int c = 32 * d + 8 * (r / 4) + 4 * half + r % 4;
            if (c < a.D) o[c] = O[d][r];
          }
        if (half == 0) {
          o[a.D] = top;
          o[a.D + 1] = sum;
        }
      }
    }
    const uint64_t bad = __ballot(!fine);
    uint32_t heads = (uint32_t)bad | (uint32_t)(bad >> 32);
    for (; heads; heads &= heads - 1) step_row<1, 1>(a, s, h0 + __builtin_ctz(heads), 0, nullptr);
  }
  if (split == 0 && pass == 0 && tid < a.D) {
    const int64_t r = p < a.sinks ? p : a.sinks + (p - a.sinks) % ring;
    kc[r * a.ks.row + tid] = kn[tid];
    vc[r * a.vs.row + tid] = vn[tid];
  }
}

// The splits of a stream's head (blockIdx.x = stream * Hq + head): their weights first,
// a split a thread, then the outputs, channels side by side.
template <int NS>
__global__ void __launch_bounds__(NT) attn_step_join_kernel(StepArgs<NS> a) {
  __shared__ float w[MAX_SPLITS], red[NT];
  const int s = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, tid = threadIdx.x;
  const int64_t step = a.D + 2;
  const float* const part = a.part + (int64_t)blockIdx.x * a.splits * step;
  float m = -INFINITY, l = 0.f;
  for (int i = tid; i < a.splits; i += NT) {
    w[i] = part[i * step + a.D];
    m = fmaxf(m, w[i]);  // (a split whose scores are NaN has a sum that is)
  }
  red[tid] = wave_max(m);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT; i += 64) m = fmaxf(m, red[i]);
  __syncthreads();
  const float b = m == -INFINITY ? 0.f : m;
  for (int i = tid; i < a.splits; i += NT) {
    w[i] = __builtin_amdgcn_exp2f(w[i] - b);
    l = fmaf(w[i], part[i * step + a.D + 1], l);
  }
  red[tid] = wave_sum(l);
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int i = 0; i < NT; i += 64) l += red[i];
  __syncthreads();
  const int slices = NT / a.D, sl = tid / a.D, ch = tid % a.D;
  float v = 0.f;
  if (sl < slices)
#pragma unroll 8
    for (int i = sl; i < a.splits; i += slices) v = fmaf(w[i], part[i * step + ch], v);
  red[tid] = v;
  __syncthreads();
  bool fine = true;
  if (tid < a.D) {
    for (int i = 1; i < slices; ++i) v += red[i * a.D + ch];
    v /= l;
    fine = (fabsf(v) < INFINITY && l > SUM_LEAST && l < SUM_MOST) ||
           (NS == 3 ? l != l : a.D % 32 == 0 && nan_score(m, l));
  }
  if (__syncthreads_or(!fine)) {
    step_row<NS, NT / 64>(a, s, h, tid >> 6, w);
  } else if (tid < a.D) {
    a.o.p[s * a.o.row + h * a.o.head + ch] = Elem<NS>::put(v);
  }
}

int lanes_per_key(int D) {
  int lp = 1;
  while (lp * 8 < D) lp <<= 1;
  return lp;
}

// bf16 goes to the matrix cores.  fp32 stays on the vector unit: 64 streams of 4096 rows, 2
// key heads of 64, take 46, 47, 49, 54 and 93 us with 1, 2, 4, 8 and 16 query heads on each (5.9
// to 5.0 TB/s, then 16 read the cache twice), in bf16 31 and, with 16, 33.
struct Plan {
  int gc, passes, splits;
};
// Query heads of a pass: 32 columns, or up to eight (registers).  Splits: blocks for four
// (bf16) or two a CU, with at least 1024 or 256 rows to each (131,072 rows of 2 heads of
// 128 channels, bf16: 48 us in parts of 256, 37 of 512, 34 of 1024; one fp32 stream of
// 262,144: 55 us in 4096 blocks, 47 in 512).
Plan plan(int type, int streams, int64_t cap, int Hq, int Hk, int64_t left, int64_t sinks) {
  Plan p;
  const int group = Hq / Hk;
  const bool wide = type == SCN_BF16;
  p.gc = wide ? 32 : group <= 1 ? 1 : group <= 2 ? 2 : group <= 4 ? 4 : 8;
  p.passes = (int)ceil_div(group, p.gc);
  const int64_t ring = cap - sinks;
  const int64_t see = sinks + (left < 0 || left >= ring ? ring : left + 1);
  const int64_t blocks = (int64_t)streams * Hk * p.passes;
  const int64_t want = wide ? 1024 : 512, rows = wide ? 1024 : 256;
  p.splits = (int)std::max<int64_t>(1, std::min({ceil_div(want, blocks), ceil_div(see, rows),
                                                 (int64_t)MAX_SPLITS}));
  return p;
}

template <int NS, int LP>
void launch_gc(const StepArgs<NS>& a, int gc, hipStream_t st) {
  const dim3 grid((unsigned)(a.splits * a.passes * a.Hk * a.streams)), block(NT);
  if (gc == 1) hipLaunchKernelGGL((attn_step_kernel<NS, LP, 1>), grid, block, 0, st, a);
  if (gc == 2) hipLaunchKernelGGL((attn_step_kernel<NS, LP, 2>), grid, block, 0, st, a);
  if (gc == 4) hipLaunchKernelGGL((attn_step_kernel<NS, LP, 4>), grid, block, 0, st, a);
  if (gc == 8) hipLaunchKernelGGL((attn_step_kernel<NS, LP, 8>), grid, block, 0, st, a);
}

template <int DP>
void launch_wide(const StepArgs<1>& a, hipStream_t st) {
  hipLaunchKernelGGL(attn_step_wide_kernel<DP>,
                     dim3((unsigned)(a.splits * a.passes * a.Hk * a.streams)), dim3(NT), 0, st, a);
}

template <int NS>
scn_status run(const StepArgs<NS>& a, int gc, hipStream_t st) {
  if constexpr (NS == 1) {
    if (a.D <= 32)
      launch_wide<32>(a, st);
    else if (a.D <= 64)
      launch_wide<64>(a, st);
    else if (a.D <= 96)
      launch_wide<96>(a, st);
    else
      launch_wide<128>(a, st);
  } else {
    switch (lanes_per_key(a.D)) {
      case 1: launch_gc<NS, 1>(a, gc, st); break;
      case 2: launch_gc<NS, 2>(a, gc, st); break;
      case 4: launch_gc<NS, 4>(a, gc, st); break;
      case 8: launch_gc<NS, 8>(a, gc, st); break;
      default: launch_gc<NS, 16>(a, gc, st);
    }
  }
  SCN_LAUNCH_CHECK();
  if (a.splits > 1) {
    hipLaunchKernelGGL(attn_step_join_kernel<NS>, dim3((unsigned)(a.streams * a.Hq)), dim3(NT), 0,
                       st, a);
    SCN_LAUNCH_CHECK();
  }
  return SCN_OK;
}

template <int NS>
StepArgs<NS> make(int streams, int64_t cap, int D, int Hq, int Hk, const Plan& p,
                  const scn_heads* q, const scn_heads* k, const scn_heads* v, const scn_cache* kc,
                  const scn_cache* vc, const int32_t* length, float scale, int64_t left,
                  int64_t sinks, const scn_heads* o, void* ws) {
  typedef typename Elem<NS>::T T;
  const int64_t ring = cap - sinks;
  return StepArgs<NS>{streams, (int)cap, D, Hq, Hk, Hq / Hk, p.passes, p.splits,
                      view<const T>(q), view<const T>(k), view<const T>(v),
                      static_cast<T*>(kc->p), static_cast<T*>(vc->p),
                      Ring{kc->stream, kc->row, kc->head}, Ring{vc->stream, vc->row, vc->head},
                      length, scale, (int)(left < 0 || left >= ring ? ring - 1 : left), (int)sinks,
                      view<T>(o), p.splits > 1 ? static_cast<float*>(ws) : nullptr};
}

scn_status check_cache(const char* who, const char* name, const scn_cache* c, int type) {
  if (!c) {
    set_error("%s: %s is null", who, name);
    return SCN_ERR_INVALID;
  }
  const int64_t unit = type == SCN_BF16 ? 8 : 4;
  const scn_heads h{c->p, c->row, c->head};
  if (c->stream % unit != 0) {
    set_error("%s: %s must have strides of whole 16 bytes", who, name);
    return SCN_ERR_INVALID;
  }
  return check_heads(who, name, &h, type);
}

}  // namespace
}  // namespace scn

using namespace scn;

extern "C" {

size_t scn_attn_step_workspace_bytes(int32_t type, int32_t streams, int64_t capacity, int32_t D,
                                     int32_t Hq, int32_t Hk, int64_t left, int64_t sinks) {
  if ((type != SCN_F32 && type != SCN_BF16) || streams < 1 || streams > 65535 || capacity < 1 || capacity > ATTN_ROWS || D < 1 ||
      D > ATTN_D || Hk < 1 || Hq < 1 || Hq % Hk != 0 || sinks < 0 || sinks >= capacity)
    return 0;
  const Plan p = plan(type, streams, capacity, Hq, Hk, left, sinks);
  return p.splits > 1 ? (size_t)streams * Hq * p.splits * (D + 2) * 4 : 0;
}

scn_status scn_attn_step(int32_t type, int32_t streams, int64_t capacity, int32_t D, int32_t Hq,
                         int32_t Hk, const scn_heads* q, const scn_heads* k, const scn_heads* v,
                         const scn_cache* k_cache, const scn_cache* v_cache,
                         const int32_t* length, float scale, int64_t left, int64_t sinks,
                         const scn_heads* o, void* ws, size_t ws_bytes, hipStream_t st) {
  clear_error();
  const char* const who = "scn_attn_step";
  // (length stands for the ranges: both are arrays that the call cannot do without)
  if (scn_status rc = check_attn(who, type, std::max(0, streams), 1, length, D, Hq, Hk, scale))
    return rc;
  if (streams < 0 || sinks < 0 || capacity <= sinks) {
    set_error("%s: negative sizes, or a capacity that leaves no row past the sinks", who);
    return SCN_ERR_INVALID;
  }
  if (streams > 65535 || capacity > ATTN_ROWS) {
    set_error("%s: more than 65535 streams or 2^30 cache rows", who);
    return SCN_ERR_OVERFLOW;
  }
  if (streams == 0) return SCN_OK;
  if (scn_status rc = check_heads(who, "q", q, type)) return rc;
  if (scn_status rc = check_heads(who, "k", k, type)) return rc;
  if (scn_status rc = check_heads(who, "v", v, type)) return rc;
  if (scn_status rc = check_heads(who, "o", o, type)) return rc;
  if (scn_status rc = check_cache(who, "k_cache", k_cache, type)) return rc;
  if (scn_status rc = check_cache(who, "v_cache", v_cache, type)) return rc;
  const Plan p = plan(type, streams, capacity, Hq, Hk, left, sinks);
  if ((int64_t)streams * Hk * p.passes * p.splits > INT32_MAX || (int64_t)streams * Hq > INT32_MAX) {
    set_error("%s: more than 2^31 blocks of streams and heads", who);
    return SCN_ERR_OVERFLOW;
  }
  if (p.splits > 1 &&
      (!ws || ws_bytes < scn_attn_step_workspace_bytes(type, streams, capacity, D, Hq, Hk, left,
                                                      sinks))) {
    set_error("%s: workspace missing or too small", who);
    return SCN_ERR_WORKSPACE;
  }
  if (type == SCN_BF16)
    return run<1>(make<1>(streams, capacity, D, Hq, Hk, p, q, k, v, k_cache, v_cache, length, scale,
                          left, sinks, o, ws), p.gc, st);
  return run<3>(make<3>(streams, capacity, D, Hq, Hk, p, q, k, v, k_cache, v_cache, length, scale,
                        left, sinks, o, ws), p.gc, st);
}

}  // extern "C"
