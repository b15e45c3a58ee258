// Norm of queries and keys for each head and their rotation by the site's
// coordinates, forward and backward, and the samples' row ranges.
//
// u = w x / sqrt(mean x^2 + eps), and each channel pair of u turned by its angle.
// With g the gradient turned back, r = 1 / sqrt(mean x^2 + eps) and a = g w:
//   dx = r a - r^3 x mean(a x),   dw = sum over rows and heads of g x r.
// Both passes read and write each row once: memory bounds them.  A lane holds
// eight channels of a row in registers, LP lanes a head; the row's sines and
// cosines are formed once and serve HC heads.  Measured: 300,001 rows of 4 + 4 heads of
// 64 channels, bf16, forward 114 us (5.4 TB/s), backward 219 (4.2: its waves wait for
// memory in 80% of their cycles as the forward's do, with 2.6 of them a SIMD to its 3.7);
// 131,072 rows of 8 + 2 heads of 32, fp32, forward 64 us (5.3).
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
  int D, Hq, Hk, cq, chunks;  // cq: head chunks of q; the following ones are k's
  Heads<const T> q, k, dqr, dkr;
  Heads<T> oq, ok;    // the results, or dq and dk
  const float *wq, *wk;
  float eps, inv;  // inv = 1 / D
  const int32_t* coords;
  const float* freq;
  Axes axes;
  bool quads;   // coords are rows of four, 16-byte aligned
  bool past;    // results past the caches
  float* part;  // [chunks][blocks][D]
};

// The lane's four pairs: their coordinate columns (0: not rotated) and frequencies.
template <int NS>
struct Turns {
  int col[4];
  v4f f;
  __device__ inline Turns(const NormArgs<NS>& a, int c, bool on) {
    f = v4f{0.f, 0.f, 0.f, 0.f};
    if (on && a.freq) f = *reinterpret_cast<const v4f*>(a.freq + (c >> 1));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      col[j] = 0;
      if (on)
        for (int x = a.axes.n - 1; x >= 0; --x)
          if ((c >> 1) + j < a.axes.end[x]) col[j] = 1 + x;
    }
  }
  // The product of a coordinate and a frequency has up to 55 bits and its turns are what
  // counts, so both are formed in 64 bits and reduced before rounding.  The instructions
  // for sine and cosine take turns, and are within 1.3e-7 on half a turn either way (over
  // 2^20 angles).
  __device__ inline void at(const NormArgs<NS>& a, int64_t t, float (&sn)[4], float (&cs)[4]) const {
    int x[4];
    if (a.quads) {  // rows of four: one load
      const v4i r = *reinterpret_cast<const v4i*>(a.coords + t * 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = col[j] == 1 ? r[1] : col[j] == 2 ? r[2] : r[3];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = a.coords[t * a.axes.width + col[j]];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const double u = (double)x[j] * ((double)f[j] * 0.15915494309189535);
      const float v = (float)(u - rint(u));
      sn[j] = col[j] ? __builtin_amdgcn_sinf(v) : 0.f;
      cs[j] = col[j] ? __builtin_amdgcn_cosf(v) : 1.f;
    }
  }
};

template <int NS>
__device__ inline void load_weights(const float* w, int c, bool on, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = 1.f;
  if (on && w) load8<3>(w + c, v);
}

// Rows in turn and HC heads for LP lanes.  The chunks of heads of the same rows follow one
// another, so that what lies together in memory is read together.
template <int NS, int LP, int HC>
__global__ void __launch_bounds__(NT) norm_rotate_fwd_kernel(NormArgs<NS> a) {
  const int chunk = blockIdx.x % a.chunks, block = blockIdx.x / a.chunks;
  const int blocks = gridDim.x / a.chunks;
  const bool isq = chunk < a.cq;
  const int h0 = (chunk - (isq ? 0 : a.cq)) * HC;
  const int nh = min(HC, (isq ? a.Hq : a.Hk) - h0);
  const int c = (threadIdx.x % LP) * 8;
  const bool on = c < a.D;
  const auto& in = isq ? a.q : a.k;
  const auto& out = isq ? a.oq : a.ok;
  float wv[8];
  load_weights<NS>(isq ? a.wq : a.wk, c, on, wv);
  const Turns<NS> turns(a, c, on);
  // whole groups of LP lanes run the loop together
  for (int64_t t = (int64_t)block * (NT / LP) + threadIdx.x / LP; t < a.n;
       t += (int64_t)blocks * (NT / LP)) {
    const auto* const ip = in.p + t * in.row + h0 * in.head + c;
    auto* const op = out.p + t * out.row + h0 * out.head + c;
    float x[HC][8], sn[4], cs[4];
#pragma unroll
    for (int i = 0; i < HC; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
      if (on && i < nh) load8<NS>(ip + i * in.head, x[i]);
    }
    turns.at(a, t, sn, cs);
#pragma unroll
    for (int i = 0; i < HC; ++i) {
      if (i >= nh) break;
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(x[i][j], x[i][j], s);
      const float r = rsqrtf(fmaf(group_sum<LP>(s), a.inv, a.eps));
      float y[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float u = x[i][2 * j] * r * wv[2 * j], v = x[i][2 * j + 1] * r * wv[2 * j + 1];
        y[2 * j] = u * cs[j] - v * sn[j];
        y[2 * j + 1] = u * sn[j] + v * cs[j];
      }
      if (on) store8<NS>(op + i * out.head, y, a.past);
    }
  }
}

// The same for the gradients.  Blocks take rows in turn and keep their share of dw
// in registers; the shares are summed within the block and written to `part`, and
// norm_dw_kernel sums the blocks' in order.
template <int NS, int LP, int HC>
__global__ void __launch_bounds__(NT) norm_rotate_bwd_kernel(NormArgs<NS> a) {
  __shared__ float red[NT / 64][LP * 8];
  const int chunk = blockIdx.x % a.chunks, block = blockIdx.x / a.chunks;
  const int blocks = gridDim.x / a.chunks;
  const bool isq = chunk < a.cq;
  const int h0 = (chunk - (isq ? 0 : a.cq)) * HC;
  const int nh = min(HC, (isq ? a.Hq : a.Hk) - h0);
  const int c = (threadIdx.x % LP) * 8;
  const bool on = c < a.D;
  const auto& in = isq ? a.q : a.k;
  const auto& dy = isq ? a.dqr : a.dkr;
  const auto& out = isq ? a.oq : a.ok;
  float wv[8], dw[8];
  load_weights<NS>(isq ? a.wq : a.wk, c, on, wv);
#pragma unroll
  for (int j = 0; j < 8; ++j) dw[j] = 0.f;
  const Turns<NS> turns(a, c, on);
  for (int64_t t = (int64_t)block * (NT / LP) + threadIdx.x / LP; t < a.n;
       t += (int64_t)blocks * (NT / LP)) {
    float x[HC][8], g[HC][8];
    const auto* const ip = in.p + t * in.row + h0 * in.head + c;
    const auto* const gp = dy.p + t * dy.row + h0 * dy.head + c;
    auto* const op = out.p + t * out.row + h0 * out.head + c;
#pragma unroll
    for (int i = 0; i < HC; ++i)
      if (on && i < nh) {
        load8<NS>(ip + i * in.head, x[i]);
        load8<NS>(gp + i * dy.head, g[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = g[i][j] = 0.f;
      }
    float sn[4], cs[4];
    turns.at(a, t, sn, cs);
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
      const float r = rsqrtf(fmaf(group_sum<LP>(s), a.inv, a.eps));
      // (r^3 would pass fp32's range where its product with x and the mean does not)
      const float z = r * (group_sum<LP>(m) * a.inv);
      float d[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = x[i][j] * r;
        d[j] = r * (g[i][j] * wv[j] - z * n);
        dw[j] = fmaf(g[i][j], n, dw[j]);
      }
      if (on) store8<NS>(op + i * out.head, d, a.past);
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
    a.part[((int64_t)chunk * blocks + block) * a.D + i] = s;
  }
}

// dw: the blocks' shares, part[rows][D], in a fixed order: block (weight, eight
// channels), 128 threads to a channel; weight 0 is wq's (the first nq rows), 1 wk's.
__global__ void __launch_bounds__(1024) norm_dw_kernel(const float* part, int64_t nq, int64_t nk,
                                                       int D, float* dwq, float* dwk) {
  __shared__ float red[16][8];
  float* const out = blockIdx.x & 1 ? dwk : dwq;
  if (!out) return;
  const int64_t lo = blockIdx.x & 1 ? nq : 0, hi = blockIdx.x & 1 ? nq + nk : nq;
  const int c = (blockIdx.x >> 1) * 8 + threadIdx.x % 8;
  float v = 0.f;
#pragma unroll 4
  for (int64_t i = lo + threadIdx.x / 8; i < hi; i += 128) v += part[i * D + c];
#pragma unroll
  for (int d = 8; d < 64; d <<= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) < 8) red[threadIdx.x >> 6][threadIdx.x & 7] = v;
  __syncthreads();
  if (threadIdx.x >= 8) return;
  for (int i = 1; i < 16; ++i) v += red[i][threadIdx.x];
  out[c] = v;
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

constexpr int BLOCKS = 4096;  // of a call, over its chunks of heads (16 a CU)

int lanes_per_head(int D) {
  int lp = 1;
  while (lp * 8 < D) lp <<= 1;
  return lp;
}
// Heads that share a row's sines and cosines: four once the rows fill the GPU.
int heads_per_lane(int64_t n, int D, int H) {
  return n * H * lanes_per_head(D) >= 256 * 1024 ? 4 : 1;
}
int row_blocks(int64_t n, int D, int chunks) {
  const int64_t need = ceil_div(n * lanes_per_head(D), NT);
  return (int)std::max<int64_t>(1, std::min<int64_t>(need, ceil_div(BLOCKS, chunks)));
}

template <int NS, int LP, int HC>
void launch(const NormArgs<NS>& a, bool bwd, int blocks, int chunks, hipStream_t st) {
  if (bwd)
    hipLaunchKernelGGL((norm_rotate_bwd_kernel<NS, LP, HC>), dim3((unsigned)blocks * chunks), dim3(NT),
                       0, st, a);
  else
    hipLaunchKernelGGL((norm_rotate_fwd_kernel<NS, LP, HC>), dim3((unsigned)blocks * chunks), dim3(NT),
                       0, st, a);
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
  if (((reinterpret_cast<uintptr_t>(c.wq) | reinterpret_cast<uintptr_t>(c.wk) |
        reinterpret_cast<uintptr_t>(c.freq)) & 15) != 0) {
    set_error("%s: wq, wk and freq must be 16-byte aligned", c.who);
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
  a.inv = 1.f / (float)c.D;
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
  a.chunks = chunks;
  const int blocks = row_blocks(c.n, c.D, chunks);
  a.quads = c.width == 4 && (reinterpret_cast<uintptr_t>(c.coords) & 15) == 0;
  // Large results of whole 64-byte pieces go past the caches: 131,072 rows of 10 fp32
  // heads of 32 take 61 us that way and 74 through them; pieces of 48 bytes take 14%
  // longer.
  const int64_t row = c.D * (int64_t)sizeof(T);
  a.past = row % 64 == 0 && c.n * (c.Hq + c.Hk) * row >= (int64_t(64) << 20);
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
  return (size_t)(chunks * row_blocks(n, D, (int)chunks) * D * 4);
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
    hipLaunchKernelGGL(norm_dw_kernel, dim3(2 * (D / 8)), dim3(1024), 0, st, part, (int64_t)rq, (int64_t)rk,
                       D, dwq, dwk);
    SCN_LAUNCH_CHECK();
  }
  return SCN_OK;
}

}  // extern "C"
