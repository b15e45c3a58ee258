// The norm of many tensors taken together, and their scaling to a largest norm.
//
//   norm = sqrt(sum over all of t^2),   out = norm > most ? t most / norm : t
// Two kernels: one sums squares, in 64 bits (no square of an fp32 number leaves their
// range, and the sum's rounding is far below fp32's), a number a block; in the other every
// block adds up those numbers in the same order, so that the scale need not be waited for,
// and scales its share, or leaves at once where nothing changes in place.  Memory bounds
// both.  Few elements take one block and one launch.  The tensors' addresses travel in the
// kernels' arguments, up to TABLE of them a launch.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "attn.h"

namespace scn {
namespace {

constexpr int NT = 256;
constexpr int TABLE = 128;       // tensors of a launch (28 bytes each; arguments end at 4 KB)
constexpr int CHUNK = 8192;      // elements that a block takes at a time ...
constexpr int SMALL_CHUNK = 1024;  // ... and a wave of the one block of small calls
constexpr int SMALL = 32768;     // elements of a small call
constexpr int BLOCKS = 2048;     // of all launches together, each at least LEAST
constexpr int LEAST = 64;

struct Table {
  const void* in[TABLE];
  void* out[TABLE];
  int64_t n[TABLE];        // elements; bit 62: bf16
  int32_t start[TABLE];    // chunks of the tensors before
  int32_t count, chunks;
  int32_t moved;           // whether any result is not its gradient's place
};
constexpr int64_t IS_BF16 = int64_t(1) << 62;

typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));

// The chunks first, first + step, ..: what(tensor, first element, elements)
template <int SIZE, class F>
__device__ inline void each_chunk(const Table& t, int first, int step, const F& what) {
  for (int c = first; c < t.chunks; c += step) {
    int lo = 0, hi = t.count;  // the last tensor that starts at c or before
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (t.start[mid] <= c) lo = mid;
      else hi = mid;
    }
    const int64_t n = t.n[lo] & ~IS_BF16, e = (int64_t)(c - t.start[lo]) * SIZE;
    what(lo, e, (int)min((int64_t)SIZE, n - e));
  }
}

template <int THREADS>
__device__ inline double block_sum(double v) {
  __shared__ double red[THREADS / 64];
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) v += red[w];
  return v;
}

// n <= SIZE elements from `first` on of tensor i, for the THREADS threads tid
template <int THREADS, int SIZE>
__device__ inline void add_squares(const Table& t, int i, int64_t first, int n, int tid,
                                   double (&s)[4]) {
  if (t.n[i] & IS_BF16) {
    const uint16_t* const p = static_cast<const uint16_t*>(t.in[i]) + first;
    constexpr int N = SIZE / THREADS / 8;
    v4u x[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int e = (u * THREADS + tid) * 8;
      x[u] = v4u{0, 0, 0, 0};
      if (e + 8 <= n) x[u] = *reinterpret_cast<const v4u_any*>(p + e);
    }
    if (tid < (n & 7)) {
      const double v = Elem<1>::get(p[(n & ~7) + tid]);
      s[0] = fma(v, v, s[0]);
    }
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const double a = __uint_as_float(x[u][j] << 16), b = __uint_as_float(x[u][j] & 0xffff0000u);
        s[j] = fma(a, a, s[j]);
        s[j] = fma(b, b, s[j]);
      }
  } else {
    const float* const p = static_cast<const float*>(t.in[i]) + first;
    constexpr int N = SIZE / THREADS / 4;
    v4f x[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int e = (u * THREADS + tid) * 4;
      x[u] = v4f{0.f, 0.f, 0.f, 0.f};
      if (e + 4 <= n) x[u] = *reinterpret_cast<const v4f_any*>(p + e);
    }
    if (tid < (n & 3)) {
      const double v = p[(n & ~3) + tid];
      s[0] = fma(v, v, s[0]);
    }
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = fma((double)x[u][j], (double)x[u][j], s[j]);
  }
}

// what the norm `all` makes of the tensors (a norm that the caller sees as not finite leaves all
// as it is)
struct Scale {
  bool clip;
  double by;
  __device__ inline Scale(double all, double most)
      : clip(all > most && (float)all < INFINITY), by(clip ? most / all : 1.) {}
};
template <int THREADS, int SIZE>
__device__ inline void scale_to(const Table& t, int i, int64_t first, int n, int tid, Scale z) {
  if (!z.clip && t.in[i] == t.out[i]) return;
  // (products in 64 bits: the scale itself may leave fp32's range)
  auto by = [&](float v) { return (float)(v * z.by); };
  if (t.n[i] & IS_BF16) {
    const uint16_t* const p = static_cast<const uint16_t*>(t.in[i]) + first;
    uint16_t* const o = static_cast<uint16_t*>(t.out[i]) + first;
    constexpr int N = SIZE / THREADS / 8;
    v4u x[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int e = (u * THREADS + tid) * 8;
      if (e + 8 <= n) x[u] = *reinterpret_cast<const v4u_any*>(p + e);
    }
    if (tid < (n & 7)) {
      const int e = (n & ~7) + tid;
      o[e] = z.clip ? Elem<1>::put(by(Elem<1>::get(p[e]))) : p[e];
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int e = (u * THREADS + tid) * 8;
      if (e + 8 > n) continue;
      if (z.clip)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[u][j] = cvt2_bf16(by(__uint_as_float(x[u][j] << 16)),
                              by(__uint_as_float(x[u][j] & 0xffff0000u)));
      *reinterpret_cast<v4u_any*>(o + e) = x[u];
    }
  } else {
    const float* const p = static_cast<const float*>(t.in[i]) + first;
    float* const o = static_cast<float*>(t.out[i]) + first;
    constexpr int N = SIZE / THREADS / 4;
    v4f x[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int e = (u * THREADS + tid) * 4;
      if (e + 4 <= n) x[u] = *reinterpret_cast<const v4f_any*>(p + e);
    }
    if (tid < (n & 3)) {
      const int e = (n & ~3) + tid;
      o[e] = by(p[e]);
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int e = (u * THREADS + tid) * 4;
      if (e + 4 > n) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[u][j] = by(x[u][j]);
      *reinterpret_cast<v4f_any*>(o + e) = x[u];
    }
  }
}

__global__ void __launch_bounds__(NT) grad_squares_kernel(Table t, double* part) {
  double s[4] = {0., 0., 0., 0.};
  each_chunk<CHUNK>(t, blockIdx.x, gridDim.x, [&](int i, int64_t first, int n) {
    add_squares<NT, CHUNK>(t, i, first, n, threadIdx.x, s);
  });
  const double v = block_sum<NT>((s[0] + s[1]) + (s[2] + s[3]));
  if (threadIdx.x == 0) part[blockIdx.x] = v;
}

// `norm` (of the first launch alone) gets the norm.
__global__ void __launch_bounds__(NT) grad_scale_kernel(Table t, const double* part, int parts,
                                                        double most, float* norm) {
  double s = 0.;
#pragma unroll 4
  for (int i = threadIdx.x; i < parts; i += NT) s += part[i];
  const double all = sqrt(block_sum<NT>(s));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)all;
  const Scale z(all, most);
  if (!z.clip && !t.moved) return;
  each_chunk<CHUNK>(t, blockIdx.x, gridDim.x, [&](int i, int64_t first, int n) {
    scale_to<NT, CHUNK>(t, i, first, n, threadIdx.x, z);
  });
}

// Small calls, in one block: a chunk a wave.  20,608 elements in 8 tensors: 3.8 and 4.9 us in two
// kernels.
__global__ void __launch_bounds__(1024) grad_small_kernel(Table t, double most, float* norm) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  double s[4] = {0., 0., 0., 0.};
  each_chunk<SMALL_CHUNK>(t, wave, 16, [&](int i, int64_t first, int n) {
    add_squares<64, SMALL_CHUNK>(t, i, first, n, lane, s);
  });
  const double all = sqrt(block_sum<1024>((s[0] + s[1]) + (s[2] + s[3])));
  if (threadIdx.x == 0) *norm = (float)all;
  const Scale z(all, most);
  if (!z.clip && !t.moved) return;
  each_chunk<SMALL_CHUNK>(t, wave, 16, [&](int i, int64_t first, int n) {
    scale_to<64, SMALL_CHUNK>(t, i, first, n, lane, z);
  });
}

int launches(int64_t count) { return (int)std::max<int64_t>(1, ceil_div(count, TABLE)); }
int blocks_each(int n) { return std::max(LEAST, BLOCKS / n); }
bool small(int64_t count, int64_t elements) { return count <= TABLE && elements <= SMALL; }

int64_t size_of(const scn_tensor& t) { return t.type == SCN_BF16 ? 2 : 4; }

// Results must lie apart from each other and from all gradients but their own.
bool apart(int64_t count, const scn_tensor* grads, void* const* out) {
  struct Piece {
    uintptr_t lo, hi;
    bool result;
  };
  std::vector<Piece> all;
  all.reserve(2 * count);
  for (int64_t i = 0; i < count; ++i) {
    if (grads[i].n == 0) continue;
    const uintptr_t in = reinterpret_cast<uintptr_t>(grads[i].p), size = grads[i].n * size_of(grads[i]);
    const uintptr_t to = out ? reinterpret_cast<uintptr_t>(out[i]) : in;
    all.push_back({to, to + size, true});
    if (to != in) all.push_back({in, in + size, false});
  }
  std::sort(all.begin(), all.end(), [](const Piece& a, const Piece& b) { return a.lo < b.lo; });
  uintptr_t any = 0, result = 0;  // ends of the pieces so far, and of the results among them
  for (const Piece& p : all) {
    if (p.lo < (p.result ? any : result)) return false;
    any = std::max(any, p.hi);
    if (p.result) result = std::max(result, p.hi);
  }
  return true;
}

}  // namespace
}  // namespace scn

using namespace scn;

extern "C" {

size_t scn_grad_clip_workspace_bytes(int64_t count, int64_t elements) {
  if (count < 0 || elements < 0 || small(count, elements)) return 0;
  const int n = launches(count);
  return (size_t)n * blocks_each(n) * sizeof(double);
}

scn_status scn_grad_clip(int64_t count, const scn_tensor* grads, void* const* out, double most,
                         float* norm, void* ws, size_t ws_bytes, hipStream_t st) {
  clear_error();
  const char* const who = "scn_grad_clip";
  if (count < 0 || (count > 0 && !grads) || !norm || !(most >= 0.)) {
    set_error("%s: bad count, no gradients, no norm, or a largest norm that is negative or NaN", who);
    return SCN_ERR_INVALID;
  }
  if (count > (1 << 20)) {
    set_error("%s: more than 2^20 tensors", who);
    return SCN_ERR_OVERFLOW;
  }
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) {
    const scn_tensor& t = grads[i];
    if ((t.type != SCN_F32 && t.type != SCN_BF16) || t.n < 0) {
      set_error("%s: tensor %lld has an unknown type or a negative size", who, (long long)i);
      return SCN_ERR_INVALID;
    }
    const void* const o = out ? out[i] : t.p;
    if (t.n > 0 && (!t.p || !o || (reinterpret_cast<uintptr_t>(t.p) | reinterpret_cast<uintptr_t>(o)) %
                                          size_of(t) != 0)) {
      set_error("%s: tensor %lld or its result is null or misaligned", who, (long long)i);
      return SCN_ERR_INVALID;
    }
    if (t.n > (int64_t(1) << 40) - total) {
      set_error("%s: more than 2^40 elements", who);
      return SCN_ERR_OVERFLOW;
    }
    total += t.n;
  }
  const size_t need = scn_grad_clip_workspace_bytes(count, total);
  if (need && (!ws || reinterpret_cast<uintptr_t>(ws) % 8 != 0 || ws_bytes < need)) {
    set_error("%s: workspace missing, misaligned or too small", who);
    return SCN_ERR_WORKSPACE;
  }
  try {
    if (!apart(count, grads, out)) {
      set_error("%s: results overlap each other or another gradient", who);
      return SCN_ERR_INVALID;
    }
  } catch (const std::bad_alloc&) {
    set_error("%s: no host memory", who);
    return SCN_ERR_NOMEM;
  }
  int64_t i = 0;
  // the next tensors, as many as a launch takes
  auto next = [&](int size) {
    Table t;
    t.count = t.chunks = t.moved = 0;
    for (; i < count && t.count < TABLE; ++i) {
      if (grads[i].n == 0) continue;
      t.in[t.count] = grads[i].p;
      t.out[t.count] = out ? out[i] : grads[i].p;
      t.n[t.count] = grads[i].n | (grads[i].type == SCN_BF16 ? IS_BF16 : 0);
      t.moved |= t.in[t.count] != t.out[t.count];
      t.start[t.count++] = t.chunks;
      t.chunks += (int32_t)ceil_div(grads[i].n, size);
    }
    return t;
  };
  if (need == 0) {
    hipLaunchKernelGGL(grad_small_kernel, dim3(1), dim3(1024), 0, st, next(SMALL_CHUNK), most, norm);
    SCN_LAUNCH_CHECK();
    return SCN_OK;
  }
  double* const part = static_cast<double*>(ws);
  const int each = blocks_each(launches(count));
  auto blocks = [&](const Table& t) { return std::max(1, std::min(t.chunks, each)); };
  int parts = 0;
  do {
    const Table t = next(CHUNK);
    hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)blocks(t)), dim3(NT), 0, st, t,
                       part + parts);
    SCN_LAUNCH_CHECK();
    parts += blocks(t);
  } while (i < count);
  i = 0;
  do {
    const bool first = i == 0;
    const Table t = next(CHUNK);
    hipLaunchKernelGGL(grad_scale_kernel, dim3((unsigned)blocks(t)), dim3(NT), 0, st, t, part, parts,
                       most, first ? norm : nullptr);
    SCN_LAUNCH_CHECK();
  } while (i < count);
  return SCN_OK;
}

}  // extern "C"
