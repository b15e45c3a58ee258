// The norms around a block, with its gate and its residual, in one pass each way.
//
// With n(t) = t / sqrt(mean t^2 + eps), g = sigmoid(z) and u = wf n(f):
//   y = alpha x + g u,   h = wh n(y)
// and backward, with r = 1 / sqrt(mean t^2 + eps) of each norm, a = dh wh, b = dY g wf:
//   dY = dy + r_y (a - n(y) mean(a n(y))),   dx = alpha dY,   dz = dY u g (1 - g),
//   df = r_f (b - n(f) mean(b n(f))),   dwf = sum dY g n(f),   dwh = sum dh n(y).
// Each row is read and written once, y is not read back by the backward (it is formed again
// from x, f and z): memory bounds both.  A lane holds eight channels, LP lanes a row.
#include <cmath>

#include "attn.h"

namespace scn {
namespace {

constexpr int BLOCK_C = 4096;  // most channels
constexpr int NT = 256;

template <class T>
struct Rows {
  T* p;
  int64_t row;
};

template <int RS, int TS>
struct BlockArgs {
  typedef typename Elem<RS>::T R;
  typedef typename Elem<TS>::T T;
  int64_t n;
  int C;
  float alpha, eps, inv;  // inv = 1 / C
  Rows<const R> x, dy;
  Rows<const T> f, z, dh;
  const float *wf, *wh;
  Rows<R> y;     // or dx
  Rows<T> h;     // or df
  Rows<T> dz;
  float* part;   // [2][blocks][C]: dwf, dwh
};

// Eight channels from any element on.  (The hardware takes loads and stores of 16 bytes at
// any element's place.)
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
template <int NS>
__device__ inline void get8(const typename Elem<NS>::T* p, int n, float (&v)[8]) {
  if (n < 8) {  // rows of fewer than eight channels
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? Elem<NS>::get(p[j]) : 0.f;
  } else if constexpr (NS == 1) {
    const v4u a = *reinterpret_cast<const v4u_any*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(a[j] << 16);
      v[2 * j + 1] = __uint_as_float(a[j] & 0xffff0000u);
    }
  } else {
    const v4f a = *reinterpret_cast<const v4f_any*>(p), b = *reinterpret_cast<const v4f_any*>(p + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = a[j];
      v[4 + j] = b[j];
    }
  }
}
template <int NS>
__device__ inline void put8(typename Elem<NS>::T* p, int n, const float (&v)[8]) {
  if (n < 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = Elem<NS>::put(v[j]);
  } else if constexpr (NS == 1) {
    v4u_any a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = cvt2_bf16(v[2 * j], v[2 * j + 1]);
    *reinterpret_cast<v4u_any*>(p) = a;
  } else {
    *reinterpret_cast<v4f_any*>(p) = v4f_any{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<v4f_any*>(p + 4) = v4f_any{v[4], v[5], v[6], v[7]};
  }
}

// LP lanes of a row: parts of a wave, or whole blocks of LP threads
template <int LP>
struct Group {
  static constexpr int THREADS = LP > 64 ? LP : NT;
  static constexpr int ROWS = THREADS / LP;  // rows of a block at once
  static constexpr int WAVES = LP > 64 ? LP / 64 : 1;
  // (two places in turn: a sum's readers are past it when the one after the next is written)
  float (*red)[WAVES];
  int turn = 0;

  __device__ inline float sum(float v) {
    v = group_sum<(LP < 16 ? LP : 16)>(v);
    if constexpr (LP >= 32) {
      const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                      false);
      v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (LP >= 64) v = both_sum(v);
    if constexpr (LP > 64) {
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) red[turn][threadIdx.x >> 6] = v;
      __syncthreads();
      v = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v += red[turn][w];
    }
    return v;
  }
  // <a, b> over the row.  Channels below `own` of a lane are its neighbour's too, which
  // counts them; only rows of other than whole eights have such.
  __device__ inline float dot(const float (&a)[8], const float (&b)[8], int own, bool odd) {
    float s = 0.f;
    if (odd) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(j >= own ? a[j] : 0.f, b[j], s);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(a[j], b[j], s);
    }
    return sum(s);
  }
};

// v to its norm; returns 1 / sqrt(mean v^2 + eps).  Rows whose squares leave fp32's range, or
// its best part where eps does not hide it, are scaled by a power of two first.
template <int LP>
__device__ inline float norm8(Group<LP>& g, const float (&v)[8], int own, bool odd, float eps,
                              float inv, float (&out)[8]) {
  const float s = g.dot(v, v, own, odd);
  if (s < 0x1p120f && (s > 0x1p-100f || eps > 0x1p-80f)) {
    const float r = __builtin_amdgcn_rsqf(fmaf(s, inv, eps));
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = v[j] * r;
    return r;
  }
  const float by = s < 1.f ? 0x1p100f : 0x1p-72f;
#pragma unroll
  for (int j = 0; j < 8; ++j) out[j] = v[j] * by;
  const float r = __builtin_amdgcn_rsqf(fmaf(g.dot(out, out, own, odd), inv, eps * by * by));
#pragma unroll
  for (int j = 0; j < 8; ++j) out[j] *= r;
  return fminf(r * by, 0x1.fffffep127f);
}

// sigmoid(z) and what it lacks to 1, both without cancellation and within some units: with
// t = -|z| log2(e) rounded, exp(-|z|) = 2^t (1 + what t lacks ln 2)
__device__ inline void gate(float z, float& g, float& rest) {
  const float y = -fabsf(z), t = y * 0x1.715476p+0f;
  const float lack = fmaf(y, 0x1.4ae0bep-26f, fmaf(y, 0x1.715476p+0f, -t));
  float e = __builtin_amdgcn_exp2f(t);
  e = fmaf(e, lack * LN2, e);
  e = y < -126.f ? 0.f : e;  // (an infinite z has no t to lack from)
  const float a = __builtin_amdgcn_rcpf(1.f + e), b = e * a;
  g = z < 0.f ? b : a;
  rest = z < 0.f ? a : b;
}

// A lane's channels: c .. c + 7, of which those from `own` on are its alone (the last lane of
// a row of 8 m + k channels starts 8 - k channels early); n < 8 only in rows that short.
struct Channels {
  int c, own, n;
  bool on;
  template <int LP>
  static __device__ inline Channels of(int C) {
    Channels x;
    const int c = threadIdx.x % LP * 8;
    x.on = c < C;
    x.c = x.on ? min(c, max(0, C - 8)) : 0;
    x.own = x.on ? c - x.c : 8;
    x.n = min(8, C);
    return x;
  }
};

__device__ inline void ones8(const float* w, const Channels& ch, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = 1.f;
  if (ch.on && w) get8<3>(w + ch.c, ch.n, v);
}

template <int RS, int TS, int LP>
__global__ void __launch_bounds__(Group<LP>::THREADS) block_fwd_kernel(BlockArgs<RS, TS> a) {
  __shared__ float red[2][Group<LP>::WAVES];
  Group<LP> g{red};
  const Channels ch = Channels::of<LP>(a.C);
  const bool odd = a.C % 8 != 0;
  float wf[8], wh[8];
  ones8(a.wf, ch, wf);
  ones8(a.wh, ch, wh);
  constexpr int ROWS = Group<LP>::ROWS;
  // whole groups of LP lanes run the loop together
  for (int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / LP; t < a.n;
       t += (int64_t)gridDim.x * ROWS) {
    float x[8], f[8], z[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = f[j] = z[j] = 0.f;
    if (ch.on) {
      get8<RS>(a.x.p + t * a.x.row + ch.c, ch.n, x);
      if (a.f.p) get8<TS>(a.f.p + t * a.f.row + ch.c, ch.n, f);
      if (a.z.p) get8<TS>(a.z.p + t * a.z.row + ch.c, ch.n, z);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= a.alpha;
    if (a.f.p) {
      float u[8];
      norm8(g, f, ch.own, odd, a.eps, a.inv, u);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float s = 1.f, rest;
        if (a.z.p) gate(z[j], s, rest);
        x[j] = fmaf(s, u[j] * wf[j], x[j]);
      }
    }
    // (y may lie over x, and a row's last lane reads channels that the lane before it writes too:
    // where that is another wave's, and no norm of f has had all waves past their loads, they wait)
    if constexpr (LP > 64)
      if (!a.f.p) __syncthreads();
    if (a.y.p && ch.on) put8<RS>(a.y.p + t * a.y.row + ch.c, ch.n, x);
    if (!a.h.p) continue;
    float u[8];
    norm8(g, x, ch.own, odd, a.eps, a.inv, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] *= wh[j];
    if (ch.on) put8<TS>(a.h.p + t * a.h.row + ch.c, ch.n, u);
  }
}

// Blocks keep their rows' share of dwf and dwh in registers; the shares are summed within the
// block and written to `part`, and block_dw_kernel sums the blocks' in order.
template <int RS, int TS, int LP>
__global__ void __launch_bounds__(Group<LP>::THREADS) block_bwd_kernel(BlockArgs<RS, TS> a) {
  constexpr int ROWS = Group<LP>::ROWS;
  __shared__ float red[2][Group<LP>::WAVES];
  __shared__ float share[NT / 64][2][LP * 8];
  Group<LP> g{red};
  const Channels ch = Channels::of<LP>(a.C);
  const bool odd = a.C % 8 != 0;
  float wf[8], wh[8], dwf[8], dwh[8];
  ones8(a.wf, ch, wf);
  ones8(a.wh, ch, wh);
#pragma unroll
  for (int j = 0; j < 8; ++j) dwf[j] = dwh[j] = 0.f;
  for (int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / LP; t < a.n;
       t += (int64_t)gridDim.x * ROWS) {
    float x[8], f[8], z[8], dy[8], dh[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = f[j] = z[j] = dy[j] = dh[j] = 0.f;
    if (ch.on) {
      get8<RS>(a.x.p + t * a.x.row + ch.c, ch.n, x);
      if (a.f.p) get8<TS>(a.f.p + t * a.f.row + ch.c, ch.n, f);
      if (a.z.p) get8<TS>(a.z.p + t * a.z.row + ch.c, ch.n, z);
      if (a.dy.p) get8<RS>(a.dy.p + t * a.dy.row + ch.c, ch.n, dy);
      if (a.dh.p) get8<TS>(a.dh.p + t * a.dh.row + ch.c, ch.n, dh);
    }
    float s[8], rest[8], rf = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] *= a.alpha;
      s[j] = 1.f;
      rest[j] = 0.f;
      if (a.z.p) gate(z[j], s[j], rest[j]);
    }
    if (a.f.p) {
      rf = norm8(g, f, ch.own, odd, a.eps, a.inv, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = fmaf(s[j], f[j] * wf[j], x[j]);
    }
    if (a.dh.p) {
      const float ry = norm8(g, x, ch.own, odd, a.eps, a.inv, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dwh[j] = fmaf(dh[j], x[j], dwh[j]);
        dh[j] *= wh[j];
      }
      const float m = g.dot(dh, x, ch.own, odd) * a.inv;
#pragma unroll
      for (int j = 0; j < 8; ++j) dy[j] = fmaf(ry, dh[j] - x[j] * m, dy[j]);
    }
    if (a.f.p) {
      float d[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float du = dy[j] * s[j];
        z[j] = du * (f[j] * wf[j]) * rest[j];
        dwf[j] = fmaf(du, f[j], dwf[j]);
        d[j] = du * wf[j];
      }
      const float m = g.dot(d, f, ch.own, odd) * a.inv;
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = rf * (d[j] - f[j] * m);
      if (ch.on) {
        put8<TS>(a.h.p + t * a.h.row + ch.c, ch.n, d);
        if (a.dz.p) put8<TS>(a.dz.p + t * a.dz.row + ch.c, ch.n, z);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) dy[j] *= a.alpha;
    if (ch.on) put8<RS>(a.y.p + t * a.y.row + ch.c, ch.n, dy);
  }
  if (!a.part) return;
  if constexpr (LP <= 64) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#pragma unroll
      for (int d = LP; d < 64; d <<= 1) {
        dwf[j] += __shfl_xor(dwf[j], d);
        dwh[j] += __shfl_xor(dwh[j], d);
      }
      if ((threadIdx.x & 63) < LP) {
        share[threadIdx.x >> 6][0][threadIdx.x % LP * 8 + j] = dwf[j];
        share[threadIdx.x >> 6][1][threadIdx.x % LP * 8 + j] = dwh[j];
      }
    }
    __syncthreads();
  }
  if ((int)threadIdx.x >= LP || !ch.on) return;
  float* const out = a.part + (int64_t)blockIdx.x * a.C + ch.c;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (j < ch.own || j >= ch.n) continue;
    float p = dwf[j], q = dwh[j];
    if constexpr (LP <= 64) {
      p = q = 0.f;
#pragma unroll
      for (int w = 0; w < NT / 64; ++w) {
        p += share[w][0][threadIdx.x * 8 + j];
        q += share[w][1][threadIdx.x * 8 + j];
      }
    }
    out[j] = p;
    out[(int64_t)gridDim.x * a.C + j] = q;
  }
}

// dwf and dwh: the blocks' shares part[2][blocks][C], in a fixed order: block (weight, eight
// channels), 128 threads to a channel
__global__ void __launch_bounds__(1024) block_dw_kernel(const float* part, int blocks, int C,
                                                        float* dwf, float* dwh) {
  __shared__ float red[16][8];
  float* const out = blockIdx.x & 1 ? dwh : dwf;
  if (!out) return;
  const int c = (blockIdx.x >> 1) * 8 + threadIdx.x % 8;
  const float* const p = part + (int64_t)(blockIdx.x & 1) * blocks * C;
  float v = 0.f;
  if (c < C)
#pragma unroll 8
    for (int i = threadIdx.x / 8; i < blocks; i += 128) v += p[(int64_t)i * C + c];
#pragma unroll
  for (int d = 8; d < 64; d <<= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) < 8) red[threadIdx.x >> 6][threadIdx.x & 7] = v;
  __syncthreads();
  if (threadIdx.x >= 8 || c >= C) return;
  for (int i = 1; i < 16; ++i) v += red[i][threadIdx.x];
  out[c] = v;
}

// Blocks of a call at most.  Forward: 300,001 rows of 256 channels, bf16, take 139 us in one row a
// lane group, 150 in 4096 blocks and 177 in 2048.  Backward: as many as reside at once, whose
// registers hold the weights' gradients (257 us in 1024, the same in 2048, 290 in 768).
constexpr int FWD_BLOCKS = 1 << 16;
constexpr int BWD_BLOCKS = 1024;

int lanes(int C) {
  int lp = 4;
  while (lp * 8 < C) lp <<= 1;
  return lp;
}
int row_blocks(int64_t n, int C, int most) {
  const int lp = lanes(C);
  const int64_t need = ceil_div(n, lp > 64 ? 1 : NT / lp);
  return (int)std::max<int64_t>(1, std::min<int64_t>(need, most));
}

struct BlockCall {
  const char* who;
  int32_t res, type;
  int64_t n;
  int32_t C;
  const scn_rows *x, *f, *z, *dy, *dh, *y, *h, *dz;
  const float *wf, *wh;
  float alpha, eps;
  float* part;
  bool bwd;
};

scn_status check_rows(const char* who, const char* name, const scn_rows* r, int type) {
  if (!r || !r->p) {
    set_error("%s: %s is null", who, name);
    return SCN_ERR_INVALID;
  }
  if (reinterpret_cast<uintptr_t>(r->p) % (type == SCN_BF16 ? 2 : 4) != 0 || r->row < 0) {
    set_error("%s: %s is misaligned, or its rows are in falling order", who, name);
    return SCN_ERR_INVALID;
  }
  return SCN_OK;
}

scn_status check(const BlockCall& c) {
  for (int t : {c.res, c.type})
    if (t != SCN_F32 && t != SCN_BF16) {
      set_error("%s: unknown type %d", c.who, t);
      return SCN_ERR_INVALID;
    }
  if (c.res == SCN_BF16 && c.type == SCN_F32) {
    set_error("%s: a residual of bf16 beside rows of fp32", c.who);
    return SCN_ERR_UNSUPPORTED;
  }
  if (c.n < 0 || c.C < 1 || !(c.eps >= 0.f) || !std::isfinite(c.eps) || !std::isfinite(c.alpha)) {
    set_error("%s: bad size, eps or alpha", c.who);
    return SCN_ERR_INVALID;
  }
  if (c.C > BLOCK_C) {
    set_error("%s: rows of %d channels (up to %d are supported)", c.who, c.C, BLOCK_C);
    return SCN_ERR_UNSUPPORTED;
  }
  if (c.n > ATTN_ROWS) {
    set_error("%s: more than 2^30 rows", c.who);
    return SCN_ERR_OVERFLOW;
  }
  const bool norm = c.bwd ? c.dh != nullptr : c.h != nullptr;
  if ((c.z && !c.f) || (!c.f && !norm)) {
    set_error("%s: a gate without a block's result, or neither of the norms", c.who);
    return SCN_ERR_INVALID;
  }
  if (c.n == 0) return SCN_OK;
  const struct {
    const scn_rows* r;
    const char* name;
    int type;
    bool need;
  } all[] = {{c.x, "x", c.res, true},
             {c.f, "f", c.type, false},
             {c.z, "z", c.type, false},
             {c.dy, "dy", c.res, false},
             {c.dh, "dh", c.type, false},
             {c.y, c.bwd ? "dx" : "y", c.res, c.bwd},
             {c.h, c.bwd ? "df" : "h", c.type, c.bwd && c.f},
             {c.dz, "dz", c.type, c.bwd && c.z}};
  for (const auto& a : all)
    if (a.need || a.r)
      if (scn_status rc = check_rows(c.who, a.name, a.r, a.type)) return rc;
  for (const float* w : {c.wf, c.wh})
    if (reinterpret_cast<uintptr_t>(w) % 4 != 0) {
      set_error("%s: misaligned weights", c.who);
      return SCN_ERR_INVALID;
    }
  return SCN_OK;
}

template <class T>
Rows<T> rows(const scn_rows* r) {
  return r ? Rows<T>{static_cast<T*>(r->p), r->row} : Rows<T>{nullptr, 0};
}

template <int RS, int TS, int LP>
void launch(const BlockArgs<RS, TS>& a, bool bwd, int blocks, hipStream_t st) {
  const dim3 grid((unsigned)blocks), block(Group<LP>::THREADS);
  if (bwd)
    hipLaunchKernelGGL((block_bwd_kernel<RS, TS, LP>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((block_fwd_kernel<RS, TS, LP>), grid, block, 0, st, a);
}

template <int RS, int TS>
scn_status run(const BlockCall& c, int blocks, hipStream_t st) {
  typedef typename Elem<RS>::T R;
  typedef typename Elem<TS>::T T;
  const BlockArgs<RS, TS> a{c.n, c.C, c.alpha, c.eps, 1.f / (float)c.C, rows<const R>(c.x),
                            rows<const R>(c.dy), rows<const T>(c.f), rows<const T>(c.z),
                            rows<const T>(c.dh), c.wf, c.wh, rows<R>(c.y), rows<T>(c.h),
                            rows<T>(c.dz), c.part};
  switch (lanes(c.C)) {
    case 4: launch<RS, TS, 4>(a, c.bwd, blocks, st); break;
    case 8: launch<RS, TS, 8>(a, c.bwd, blocks, st); break;
    case 16: launch<RS, TS, 16>(a, c.bwd, blocks, st); break;
    case 32: launch<RS, TS, 32>(a, c.bwd, blocks, st); break;
    case 64: launch<RS, TS, 64>(a, c.bwd, blocks, st); break;
    case 128: launch<RS, TS, 128>(a, c.bwd, blocks, st); break;
    case 256: launch<RS, TS, 256>(a, c.bwd, blocks, st); break;
    default: launch<RS, TS, 512>(a, c.bwd, blocks, st);
  }
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}
scn_status run(const BlockCall& c, int blocks, hipStream_t st) {
  if (c.res == SCN_BF16) return run<1, 1>(c, blocks, st);
  return c.type == SCN_BF16 ? run<3, 1>(c, blocks, st) : run<3, 3>(c, blocks, st);
}

}  // namespace
}  // namespace scn

using namespace scn;

extern "C" {

scn_status scn_block_norm_fwd(int32_t res_type, int32_t type, int64_t n, int32_t C,
                              const scn_rows* x, const scn_rows* f, const scn_rows* z,
                              const float* wf, const float* wh, float alpha, float eps,
                              const scn_rows* y, const scn_rows* h, hipStream_t st) {
  clear_error();
  const BlockCall c{"scn_block_norm_fwd", res_type, type, n,  C,     x,   f,       z,    nullptr,
                    nullptr,              y,        h,    nullptr, wf, wh, alpha, eps, nullptr,
                    false};
  if (scn_status rc = check(c)) return rc;
  if (n == 0) return SCN_OK;
  return run(c, row_blocks(n, C, FWD_BLOCKS), st);
}

size_t scn_block_norm_bwd_workspace_bytes(int64_t n, int32_t C) {
  if (n < 1 || n > ATTN_ROWS || C < 1 || C > BLOCK_C) return 0;
  return (size_t)row_blocks(n, C, BWD_BLOCKS) * 2 * C * 4;
}

scn_status scn_block_norm_bwd(int32_t res_type, int32_t type, int64_t n, int32_t C,
                              const scn_rows* x, const scn_rows* f, const scn_rows* z,
                              const float* wf, const float* wh, float alpha, float eps,
                              const scn_rows* dy, const scn_rows* dh, const scn_rows* dx,
                              const scn_rows* df, const scn_rows* dz, float* dwf, float* dwh,
                              void* ws, size_t ws_bytes, hipStream_t st) {
  clear_error();
  BlockCall c{"scn_block_norm_bwd", res_type, type, n,  C,  x,     f,   z,       dy,  dh, dx,
              df,                   dz,       wf,   wh, alpha, eps, nullptr, true};
  if (scn_status rc = check(c)) return rc;
  const bool want = dwf || dwh;
  if (want && n > 0) {
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 4 != 0 ||
        ws_bytes < scn_block_norm_bwd_workspace_bytes(n, C)) {
      set_error("scn_block_norm_bwd: workspace missing, misaligned or too small");
      return SCN_ERR_WORKSPACE;
    }
    c.part = static_cast<float*>(ws);
  }
  const int blocks = n > 0 ? row_blocks(n, C, BWD_BLOCKS) : 0;
  if (n > 0)
    if (scn_status rc = run(c, blocks, st)) return rc;
  if (want) {
    hipLaunchKernelGGL(block_dw_kernel, dim3((unsigned)(2 * ceil_div(C, 8))), dim3(1024), 0, st,
                       c.part, blocks, C, dwf, dwh);
    SCN_LAUNCH_CHECK();
  }
  return SCN_OK;
}

}  // extern "C"
