// Attention of one new token of each stream over its cache: the sinks and the last
// positions of the ring, each row read once.  Memory bounds it (two flops a byte and
// query head), so there is nothing to stage: LP lanes hold a key's channels, eight a
// lane, and take every query head of the key head while its row is in registers.  Each
// group of LP lanes keeps a running maximum, sum and output of its own; they join
// within the wave, the block and, where a stream's keys are split over blocks, in a
// second kernel, always in the same order.
#include "attn.h"

namespace scn {
namespace {

constexpr int NT = 256;
constexpr int U = 4;  // rows of a lane group in flight

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

// GC query heads of a key head (pass), one split of a stream's visible positions
template <int NS, int LP, int GC>
__global__ void __launch_bounds__(NT) attn_step_kernel(StepArgs<NS> a) {
  typedef Elem<NS> E;
  typedef typename E::T T;
  constexpr int KW = 64 / LP;         // keys of a wave at once
  constexpr int KB = KW * (NT / 64);  // ... of the block
  __shared__ float red[NT / 64][GC][LP * 8 + 2];
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
      a.o.p[s * a.o.row + (h0 + g) * a.o.head + ch] = E::put(v / ll);
    } else {
      float* const out = a.part + (((int64_t)s * a.Hq + h0 + g) * a.splits + split) * (a.D + 2);
      out[ch] = v;
      if (ch == 0) {
        out[a.D] = mm;
        out[a.D + 1] = ll;
      }
    }
  }
  // The new rows go to the cache.  No block reads that row: what it held is a
  // capacity's ring before the new token, past the reach.
  if (split == 0 && pass == 0 && tid < a.D) {
    const int64_t t = slot(cnt - 1);
    kc[t * a.ks.row + tid] = kn[tid];
    vc[t * a.vs.row + tid] = vn[tid];
  }
}

// The splits of a stream's head: blockIdx.x = stream * Hq + head
template <int NS>
__global__ void __launch_bounds__(NT) attn_step_join_kernel(StepArgs<NS> a) {
  __shared__ float red[3][NT];
  const int s = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, tid = threadIdx.x;
  const float* const part = a.part + (int64_t)blockIdx.x * a.splits * (a.D + 2);
  const int slices = NT / a.D, sl = tid / a.D, ch = tid % a.D;
  float m = -INFINITY, l = 0.f, v = 0.f, f, f2;
  if (sl < slices)
    for (int i = sl; i < a.splits; i += slices) {
      const float* const p = part + (int64_t)i * (a.D + 2);
      join(m, l, p[a.D], p[a.D + 1], f, f2);
      v = v * f + p[ch] * f2;
    }
  red[0][tid] = m;
  red[1][tid] = l;
  red[2][tid] = v;
  __syncthreads();
  if (tid >= a.D) return;
  for (int i = 1; i < slices; ++i) {
    const int x = i * a.D + ch;
    join(m, l, red[0][x], red[1][x], f, f2);
    v = v * f + red[2][x] * f2;
  }
  a.o.p[s * a.o.row + h * a.o.head + ch] = Elem<NS>::put(v / l);
}

int lanes_per_key(int D) {
  int lp = 1;
  while (lp * 8 < D) lp <<= 1;
  return lp;
}

struct Plan {
  int gc, passes, splits;
};
// Query heads of a pass: all of the key head's up to eight (registers).  Splits: blocks
// for four a CU, of at least 256 keys.
Plan plan(int streams, int64_t cap, int Hq, int Hk, int64_t left, int64_t sinks) {
  Plan p;
  const int group = Hq / Hk;
  p.gc = group <= 1 ? 1 : group <= 2 ? 2 : group <= 4 ? 4 : 8;
  p.passes = (int)ceil_div(group, p.gc);
  const int64_t ring = cap - sinks;
  const int64_t see = sinks + (left < 0 || left >= ring ? ring : left + 1);
  const int64_t blocks = (int64_t)streams * Hk * p.passes;
  p.splits = (int)std::max<int64_t>(1, std::min(ceil_div(1024, blocks), ceil_div(see, 256)));
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

template <int NS>
scn_status run(const StepArgs<NS>& a, int gc, hipStream_t st) {
  switch (lanes_per_key(a.D)) {
    case 1: launch_gc<NS, 1>(a, gc, st); break;
    case 2: launch_gc<NS, 2>(a, gc, st); break;
    case 4: launch_gc<NS, 4>(a, gc, st); break;
    case 8: launch_gc<NS, 8>(a, gc, st); break;
    default: launch_gc<NS, 16>(a, gc, st);
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

size_t scn_attn_step_workspace_bytes(int32_t streams, int64_t capacity, int32_t D, int32_t Hq,
                                     int32_t Hk, int64_t left, int64_t sinks) {
  if (streams < 1 || streams > 65535 || capacity < 1 || capacity > ATTN_ROWS || D < 1 ||
      D > ATTN_D || Hk < 1 || Hq < 1 || Hq % Hk != 0 || sinks < 0 || sinks >= capacity)
    return 0;
  const Plan p = plan(streams, capacity, Hq, Hk, left, sinks);
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
  const Plan p = plan(streams, capacity, Hq, Hk, left, sinks);
  if ((int64_t)streams * Hk * p.passes * p.splits > INT32_MAX || (int64_t)streams * Hq > INT32_MAX) {
    set_error("%s: more than 2^31 blocks of streams and heads", who);
    return SCN_ERR_OVERFLOW;
  }
  if (p.splits > 1 &&
      (!ws || ws_bytes < scn_attn_step_workspace_bytes(streams, capacity, D, Hq, Hk, left, sinks))) {
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
