// Norm of queries and keys for each head and their rotation by the site's
// coordinates, forward and backward, and the samples' row ranges.
//
// u = w x / sqrt(mean x^2 + eps), and each channel pair of u turned by its angle.
// With g the gradient turned back, r = 1 / sqrt(mean x^2 + eps) and a = g w:
//   dx = r a - r^3 x mean(a x),   dw = sum over rows and heads of g x r.
// Both passes read and write each row once: memory bounds them.  A lane holds
// eight channels of a row in registers, LP lanes a head; the row's sines and
// cosines are formed once and serve HC heads, since forming them (two 64-bit
// products and a reduction to one turn, then two polynomials) takes as long as
// reading about three heads.
#include "attn.h"

namespace scn {

scn_status check_heads(const char* who, const char* name, const scn_heads* h, int type) {
  if (!h || !h->p) {
    set_error("%s: %s is null", who, name);
    return SCN_ERR_INVALID;
  }
  const int64_t unit = type == SCN_BF16 ? 8 : 4;
  if ((reinterpret_cast<uintptr_t>(h->p) & 15) != 0 || h->row % unit != 0 || h->head % unit != 0) {
    set_error("%s: %s must be 16-byte aligned with strides of whole 16 bytes", who, name);
    return SCN_ERR_INVALID;
  }
  if (h->row < 0 || h->row > (1 << 22)) {
    set_error("%s: %s has rows more than 2^22 elements apart, or in falling order", who, name);
    return SCN_ERR_UNSUPPORTED;
  }
  return SCN_OK;
}

namespace {

constexpr int NT = 256;
constexpr int MAX_AXES = 8;

struct Axes {
  int32_t width;
  int32_t end[MAX_AXES];  // pairs up to end[a] turn with column 1 + a
  int32_t n;
};

template <int NS>
struct NormArgs {
  typedef typename Elem<NS>::T T;
  int64_t n;
  int D, Hq, Hk, cq;  // cq: head chunks of q; the following ones are k's
  Heads<const T> q, k, dqr, dkr;
  Heads<T> oq, ok;    // the results, or dq and dk
  const float *wq, *wk;
  float eps;
  const int32_t* coords;
  const float* freq;
  Axes axes;
  float* part;  // [chunks][blocks][D]
};

// The lane's four pairs: their coordinate columns (0: not rotated) and frequencies.
struct Turns {
  int col[4];
  float f[4];
  __device__ inline Turns(const Axes& ax, const float* freq, int c, bool on) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      col[j] = 0;
      f[j] = 0.f;
      const int pair = (c >> 1) + j;
      if (on)
        for (int a = ax.n - 1; a >= 0; --a)
          if (pair < ax.end[a]) col[j] = 1 + a;
      if (col[j]) f[j] = freq[pair];
    }
  }
  // The product of a coordinate and a frequency has up to 55 bits and its turns
  // are what counts, so both are formed in 64 bits and reduced before rounding.
  __device__ inline void at(const int32_t* site, float (&sn)[4], float (&cs)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sn[j] = 0.f;
      cs[j] = 1.f;
      if (col[j]) {
        const double t = (double)site[col[j]] * (double)f[j] * 0.15915494309189535;
        sincospif(2.f * (float)(t - rint(t)), &sn[j], &cs[j]);
      }
    }
  }
};

// One row and HC heads for LP lanes; blockIdx.y is the chunk of heads.
template <int NS, int LP, int HC>
__global__ void __launch_bounds__(NT) norm_rotate_fwd_kernel(NormArgs<NS> a) {
  const int64_t t = (int64_t)blockIdx.x * (NT / LP) + threadIdx.x / LP;
  if (t >= a.n) return;
  const bool isq = (int)blockIdx.y < a.cq;
  const int h0 = ((int)blockIdx.y - (isq ? 0 : a.cq)) * HC;
  const int nh = min(HC, (isq ? a.Hq : a.Hk) - h0);
  const int c = (threadIdx.x % LP) * 8;
  const bool on = c < a.D;
  const auto& in = isq ? a.q : a.k;
  const auto& out = isq ? a.oq : a.ok;
  const float* const w = isq ? a.wq : a.wk;
  float x[HC][8];
#pragma unroll
  for (int i = 0; i < HC; ++i)
    if (on && i < nh) load8<NS>(in.p + t * in.row + (h0 + i) * in.head + c, x[i]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
  float wv[8], sn[4], cs[4];
#pragma unroll
  for (int j = 0; j < 8; ++j) wv[j] = on && w ? w[c + j] : 1.f;
  Turns(a.axes, a.freq, c, on).at(a.coords + t * a.axes.width, sn, cs);
#pragma unroll
  for (int i = 0; i < HC; ++i) {
    if (i >= nh) break;
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(x[i][j], x[i][j], s);
    const float r = 1.f / sqrtf(group_sum<LP>(s) / (float)a.D + a.eps);
    float y[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float u = x[i][2 * j] * r * wv[2 * j], v = x[i][2 * j + 1] * r * wv[2 * j + 1];
      y[2 * j] = u * cs[j] - v * sn[j];
      y[2 * j + 1] = u * sn[j] + v * cs[j];
    }
    if (on) store8<NS>(out.p + t * out.row + (h0 + i) * out.head + c, y);
  }
}

// The same for the gradients.  Blocks take rows in turn and keep their share of dw
// in registers; the shares are summed within the block and written to `part`, and
// norm_dw_kernel sums the blocks' in order.
template <int NS, int LP, int HC>
__global__ void __launch_bounds__(NT) norm_rotate_bwd_kernel(NormArgs<NS> a) {
  __shared__ float red[NT / 64][LP * 8];
  const bool isq = (int)blockIdx.y < a.cq;
  const int h0 = ((int)blockIdx.y - (isq ? 0 : a.cq)) * HC;
  const int nh = min(HC, (isq ? a.Hq : a.Hk) - h0);
  const int c = (threadIdx.x % LP) * 8;
  const bool on = c < a.D;
  const auto& in = isq ? a.q : a.k;
  const auto& dy = isq ? a.dqr : a.dkr;
  const auto& out = isq ? a.oq : a.ok;
  const float* const w = isq ? a.wq : a.wk;
  float wv[8], dw[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    wv[j] = on && w ? w[c + j] : 1.f;
    dw[j] = 0.f;
  }
  const Turns turns(a.axes, a.freq, c, on);
  // whole groups of LP lanes run the loop together
  for (int64_t t = (int64_t)blockIdx.x * (NT / LP) + threadIdx.x / LP; t < a.n;
       t += (int64_t)gridDim.x * (NT / LP)) {
    float x[HC][8], g[HC][8];
#pragma unroll
    for (int i = 0; i < HC; ++i)
      if (on && i < nh) {
        load8<NS>(in.p + t * in.row + (h0 + i) * in.head + c, x[i]);
        load8<NS>(dy.p + t * dy.row + (h0 + i) * dy.head + c, g[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = g[i][j] = 0.f;
      }
    float sn[4], cs[4];
    turns.at(a.coords + t * a.axes.width, sn, cs);
#pragma unroll
    for (int i = 0; i < HC; ++i) {
      if (i >= nh) break;
      float s = 0.f, m = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float u = g[i][2 * j], v = g[i][2 * j + 1];
        g[i][2 * j] = u * cs[j] + v * sn[j];
        g[i][2 * j + 1] = v * cs[j] - u * sn[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s = fmaf(x[i][j], x[i][j], s);
        m = fmaf(g[i][j] * wv[j], x[i][j], m);
      }
      const float r = 1.f / sqrtf(group_sum<LP>(s) / (float)a.D + a.eps);
      const float z = r * r * r * (group_sum<LP>(m) / (float)a.D);
      float d[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        d[j] = r * (g[i][j] * wv[j]) - z * x[i][j];
        dw[j] = fmaf(g[i][j], x[i][j] * r, dw[j]);
      }
      if (on) store8<NS>(out.p + t * out.row + (h0 + i) * out.head + c, d);
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int d = LP; d < 64; d <<= 1) dw[j] += __shfl_xor(dw[j], d);
    if ((threadIdx.x & 63) < LP) red[threadIdx.x >> 6][c + j] = dw[j];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.D; i += NT) {
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NT / 64; ++v) s += red[v][i];
    a.part[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * a.D + i] = s;
  }
}

// dw: the blocks' shares, part[rows][D], in a fixed order; blockIdx.x 0 is wq's (the
// first nq rows), 1 wk's
__global__ void __launch_bounds__(1024) norm_dw_kernel(const float* part, int64_t nq, int64_t nk,
                                                       int D, float* dwq, float* dwk) {
  __shared__ float red[1024];
  float* const out = blockIdx.x ? dwk : dwq;
  if (!out) return;
  const int64_t lo = blockIdx.x ? nq : 0, hi = blockIdx.x ? nq + nk : nq;
  const int slices = 1024 / D, s = threadIdx.x / D, c = threadIdx.x % D;
  float v = 0.f;
  if (s < slices)
    for (int64_t i = lo + s; i < hi; i += slices) v += part[i * D + c];
  red[threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.x < D) {
    for (int i = 1; i < slices; ++i) v += red[i * D + c];
    out[c] = v;
  }
}

// ranges[b] = first row whose sample is b or later
__global__ void __launch_bounds__(NT) site_ranges_kernel(const int32_t* coords, int64_t n,
                                                         int width, int batch, int32_t* ranges) {
  const int64_t b = (int64_t)blockIdx.x * NT + threadIdx.x;
  if (b > batch) return;
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (coords[mid * width] < b) lo = mid + 1;
    else hi = mid;
  }
  ranges[b] = (int32_t)lo;
}

constexpr int BWD_BLOCKS = 1024;  // of a backward, over its chunks of heads

int lanes_per_head(int D) {
  int lp = 1;
  while (lp * 8 < D) lp <<= 1;
  return lp;
}
// Heads that share a row's sines and cosines: four once the rows fill the GPU.
int heads_per_lane(int64_t n, int D, int H) {
  return n * H * lanes_per_head(D) >= 256 * 1024 ? 4 : 1;
}
int bwd_blocks(int64_t n, int D, int chunks) {
  const int64_t need = ceil_div(n * lanes_per_head(D), NT);
  return (int)std::max<int64_t>(1, std::min<int64_t>(need, ceil_div(BWD_BLOCKS, chunks)));
}

template <int NS, int LP, int HC>
void launch(const NormArgs<NS>& a, bool bwd, int blocks, int chunks, hipStream_t st) {
  if (bwd)
    hipLaunchKernelGGL((norm_rotate_bwd_kernel<NS, LP, HC>), dim3(blocks, chunks), dim3(NT), 0, st,
                       a);
  else
    hipLaunchKernelGGL((norm_rotate_fwd_kernel<NS, LP, HC>), dim3(blocks, chunks), dim3(NT), 0, st,
                       a);
}
template <int NS, int HC>
void launch_lp(const NormArgs<NS>& a, bool bwd, int blocks, int chunks, hipStream_t st) {
  switch (lanes_per_head(a.D)) {
    case 1: return launch<NS, 1, HC>(a, bwd, blocks, chunks, st);
    case 2: return launch<NS, 2, HC>(a, bwd, blocks, chunks, st);
    case 4: return launch<NS, 4, HC>(a, bwd, blocks, chunks, st);
    case 8: return launch<NS, 8, HC>(a, bwd, blocks, chunks, st);
    default: return launch<NS, 16, HC>(a, bwd, blocks, chunks, st);
  }
}

struct NormCall {
  const char* who;
  int32_t type;
  int64_t n;
  int32_t D, Hq, Hk;
  const scn_heads *q, *k, *dqr, *dkr, *oq, *ok;
  const float *wq, *wk;
  float eps;
  const int32_t* coords;
  int32_t width;
  const float* freq;
  const int32_t* sections;
};

scn_status check(const NormCall& c, bool bwd) {
  if (c.type != SCN_F32 && c.type != SCN_BF16) {
    set_error("%s: unknown type %d", c.who, c.type);
    return SCN_ERR_INVALID;
  }
  if (c.n < 0 || c.Hq < 1 || c.Hk < 0 || c.D < 1 || c.width < 1 || c.width > 1 + MAX_AXES ||
      !(c.eps >= 0.f) || (c.width > 1 && !c.sections) || c.Hq > 65535 || c.Hk > 65535 - c.Hq) {
    set_error("%s: bad size, eps or coordinate width", c.who);
    return SCN_ERR_INVALID;
  }
  if (c.D % 8 != 0 || c.D > ATTN_D) {
    set_error("%s: heads of %d channels (multiples of 8 up to %d are supported)", c.who, c.D,
              ATTN_D);
    return SCN_ERR_UNSUPPORTED;
  }
  if (c.n > ATTN_ROWS) {
    set_error("%s: more than 2^30 rows", c.who);
    return SCN_ERR_OVERFLOW;
  }
  int64_t pairs = 0;
  for (int i = 0; i + 1 < c.width; ++i) {
    if (c.sections[i] < 0) pairs = INT32_MAX;
    pairs += c.sections[i];
  }
  if (pairs > c.D / 2) {
    set_error("%s: sections must be >= 0 and hold at most D/2 pairs", c.who);
    return SCN_ERR_INVALID;
  }
  if (c.n > 0 && (!c.coords || (pairs > 0 && !c.freq))) {
    set_error("%s: coords or freq is null", c.who);
    return SCN_ERR_INVALID;
  }
  if (c.n == 0) return SCN_OK;
  if (scn_status rc = check_heads(c.who, "q", c.q, c.type)) return rc;
  if (scn_status rc = check_heads(c.who, bwd ? "dq" : "qr", c.oq, c.type)) return rc;
  if (bwd)
    if (scn_status rc = check_heads(c.who, "dqr", c.dqr, c.type)) return rc;
  if (c.Hk == 0) return SCN_OK;
  if (scn_status rc = check_heads(c.who, "k", c.k, c.type)) return rc;
  if (scn_status rc = check_heads(c.who, bwd ? "dk" : "kr", c.ok, c.type)) return rc;
  return bwd ? check_heads(c.who, "dkr", c.dkr, c.type) : SCN_OK;
}

template <int NS>
scn_status run(const NormCall& c, bool bwd, float* part, int* rows_q, int* rows_k, hipStream_t st) {
  typedef typename Elem<NS>::T T;
  NormArgs<NS> a;
  a.n = c.n;
  a.D = c.D;
  a.Hq = c.Hq;
  a.Hk = c.Hk;
  a.q = view<const T>(c.q);
  a.k = view<const T>(c.k);
  a.dqr = view<const T>(c.dqr);
  a.dkr = view<const T>(c.dkr);
  a.oq = view<T>(c.oq);
  a.ok = view<T>(c.ok);
  a.wq = c.wq;
  a.wk = c.wk;
  a.eps = c.eps;
  a.coords = c.coords;
  a.freq = c.freq;
  a.axes.width = c.width;
  a.axes.n = c.width - 1;
  for (int i = 0, e = 0; i < MAX_AXES; ++i) {
    if (i + 1 < c.width) e += c.sections[i];
    a.axes.end[i] = e;
  }
  a.part = part;
  const int hc = heads_per_lane(c.n, c.D, c.Hq + c.Hk);
  a.cq = (int)ceil_div(c.Hq, hc);
  const int ck = (int)ceil_div(c.Hk, hc), chunks = a.cq + ck;
  const int blocks = bwd ? bwd_blocks(c.n, c.D, chunks)
                         : (int)ceil_div(c.n * lanes_per_head(c.D), NT);
  if (hc == 4)
    launch_lp<NS, 4>(a, bwd, blocks, chunks, st);
  else
    launch_lp<NS, 1>(a, bwd, blocks, chunks, st);
  SCN_LAUNCH_CHECK();
  *rows_q = a.cq * blocks;
  *rows_k = ck * blocks;
  return SCN_OK;
}

}  // namespace
}  // namespace scn

using namespace scn;

extern "C" {

scn_status scn_site_ranges(const int32_t* coords, int64_t n, int32_t width, int32_t batch,
                           int32_t* ranges, hipStream_t st) {
  clear_error();
  if (n < 0 || width < 1 || batch < 1 || !ranges || (n > 0 && !coords)) {
    set_error("scn_site_ranges: invalid argument");
    return SCN_ERR_INVALID;
  }
  if (n > ATTN_ROWS) {
    set_error("scn_site_ranges: more than 2^30 rows");
    return SCN_ERR_OVERFLOW;
  }
  hipLaunchKernelGGL(site_ranges_kernel, dim3((unsigned)ceil_div((int64_t)batch + 1, NT)), dim3(NT),
                     0, st, coords, n, width, batch, ranges);
  SCN_LAUNCH_CHECK();
  return SCN_OK;
}

scn_status scn_norm_rotate_fwd(int32_t type, int64_t n, int32_t D, int32_t Hq, int32_t Hk,
                               const scn_heads* q, const scn_heads* k, const float* wq,
                               const float* wk, float eps, const int32_t* coords, int32_t width,
                               const float* freq, const int32_t* sections, const scn_heads* qr,
                               const scn_heads* kr, hipStream_t st) {
  clear_error();
  const NormCall c{"scn_norm_rotate_fwd", type, n, D, Hq, Hk, q, k, nullptr, nullptr, qr, kr, wq,
                   wk, eps, coords, width, freq, sections};
  if (scn_status rc = check(c, false)) return rc;
  if (n == 0) return SCN_OK;
  int rq, rk;
  return type == SCN_BF16 ? run<1>(c, false, nullptr, &rq, &rk, st)
                          : run<3>(c, false, nullptr, &rq, &rk, st);
}

size_t scn_norm_rotate_bwd_workspace_bytes(int64_t n, int32_t D, int32_t Hq, int32_t Hk) {
  if (n <= 0 || D < 1 || D > ATTN_D || Hq < 1 || Hk < 0 || n > ATTN_ROWS) return 0;
  const int hc = heads_per_lane(n, D, Hq + Hk);
  const int64_t chunks = ceil_div(Hq, hc) + ceil_div(Hk, hc);
  return (size_t)(chunks * bwd_blocks(n, D, (int)chunks) * D * 4);
}

scn_status scn_norm_rotate_bwd(int32_t type, int64_t n, int32_t D, int32_t Hq, int32_t Hk,
                               const scn_heads* q, const scn_heads* k, const float* wq,
                               const float* wk, float eps, const int32_t* coords, int32_t width,
                               const float* freq, const int32_t* sections, const scn_heads* dqr,
                               const scn_heads* dkr, const scn_heads* dq, const scn_heads* dk,
                               float* dwq, float* dwk, void* ws, size_t ws_bytes, hipStream_t st) {
  clear_error();
  const NormCall c{"scn_norm_rotate_bwd", type, n, D, Hq, Hk, q, k, dqr, dkr, dq, dk, wq,
                   wk, eps, coords, width, freq, sections};
  if (scn_status rc = check(c, true)) return rc;
  const bool want = dwq || dwk;
  if (want && n > 0 && (!ws || ws_bytes < scn_norm_rotate_bwd_workspace_bytes(n, D, Hq, Hk))) {
    set_error("scn_norm_rotate_bwd: workspace missing or too small");
    return SCN_ERR_WORKSPACE;
  }
  int rq = 0, rk = 0;
  float* const part = want ? static_cast<float*>(ws) : nullptr;
  if (n > 0)
    if (scn_status rc = type == SCN_BF16 ? run<1>(c, true, part, &rq, &rk, st)
                                         : run<3>(c, true, part, &rq, &rk, st))
      return rc;
  if (want) {
    hipLaunchKernelGGL(norm_dw_kernel, dim3(2), dim3(1024), 0, st, part, (int64_t)rq, (int64_t)rk,
                       D, dwq, dwk);
    SCN_LAUNCH_CHECK();
  }
  return SCN_OK;
}

}  // extern "C"
