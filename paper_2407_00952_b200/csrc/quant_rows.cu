// Rows in 8 bits: the kernels around the int8 products of a layer whose frozen weight is held as codes.
//   quantize     v = x f (column factors f or 1),  a = max_c |v|,  code = rint(v * (127 / a)),  scale = a / 127
//   norm         s = x + resid,  rstd = (mean s^2 + eps)^-1/2,  v = s g,  code = rint(v * (127 / max|v|)),  scale = max|v| rstd / 127
//   norm, gradient   w = dy g,  dx = resid + rstd (w - h rstd^2 mean(w h)),  dg_c = sum_m dy h rstd
//   dequantize   y = code * scale
// The codes of a normalised row do not depend on rstd: it scales the row and its maximum alike, so one pass over the row
// collects sum s^2 and max |s g| together and every rounding decision is one of fp32 products and one fp32 division, whatever
// the order of the sum.  All arithmetic is fp32; h and y are rounded once to the buffers' type, the norm sees s before that.
// Bounded by HBM: a row lives in registers between its reduction and its output (4 accesses of 16 bytes per thread; 1 to 32 lanes
// per row up to 128 accesses, else whole warps, up to 1024 threads), so it is read once.  Maxima are taken on the bits of |v| as
// unsigned integers: a NaN or infinity is larger than every finite value.
// FRAME: rows that do not start on 16-byte boundaries (odd widths in contiguous rows).  A row is then the whole 16-byte vectors in
// it, position q = column + shift, and the elements around them, which are taken one by one; the gain and the factors, which start
// at column 0, are read as words and shifted, and the codes turn back to column 0 through shared memory.
#include <algorithm>

#include "common.cuh"
#include "host_common.h"
#include "kernels.h"
#include "launch.cuh"

namespace sl {
namespace {

constexpr float TINY_ROW = 1e-36f;       // below this 127 / max overflows: the row is held as zero
constexpr int NV = 4;                    // accesses of 16 bytes per thread

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// rint(v * inv) for |v * inv| < 128 in the low byte of the result: the product is rounded to fp32 first, then adding 1.5 * 2^23
// leaves the nearest integer (ties to even) in the low bits of the sum.
__device__ __forceinline__ uint32_t code_bits(float v, float inv) { return __float_as_uint(__fadd_rn(__fmul_rn(v, inv), 12582912.0f)); }
// W codes as W / 4 words
template <int W> __device__ __forceinline__ void code_words(uint32_t* w, const float* v, float inv, bool live) {
#pragma unroll
  for (int i = 0; i < W / 4; ++i) {
    const uint32_t lo = __byte_perm(code_bits(v[4 * i], inv), code_bits(v[4 * i + 1], inv), 0x0040);
    const uint32_t hi = __byte_perm(code_bits(v[4 * i + 2], inv), code_bits(v[4 * i + 3], inv), 0x0040);
    w[i] = live ? __byte_perm(lo, hi, 0x5410) : 0u;
  }
}
template <int W> __device__ __forceinline__ void store_words(void* p, const uint32_t* w) {
  if constexpr (W == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(p) = w[0];
}

// The largest magnitude's bits -> what a row's codes and scale need.  `unit` is what one unit of the maximum stands for
// (rstd for a norm, 1 for plain rows).
struct RowScale { float inv, scale; bool live; };
__device__ __forceinline__ RowScale row_scale(uint32_t top_bits, float unit) {
  RowScale r;
  const float a = __uint_as_float(top_bits);
  const bool finite = top_bits < 0x7f800000u;
  r.live = finite && a >= TINY_ROW;
  r.inv = r.live ? __fdiv_rn(127.0f, a) : 0.f;
  r.scale = r.live ? __fdiv_rn(__fmul_rn(a, unit), 127.0f) : finite ? 0.f : __uint_as_float(0x7fffffffu);
  return r;
}

// The row a thread works on: `n` threads per row (1-32 lanes of a warp, or whole warps), this one the t-th of them.
struct Place {
  int64_t row; int t, n, group;
  __device__ __forceinline__ explicit Place(int threads) {
    n = threads;
    group = threadIdx.x / threads;
    t = threadIdx.x - group * threads;
    row = (int64_t)blockIdx.x * (blockDim.x / threads) + group;
  }
};

// Sums and maximum over the threads of a row.  With whole warps per row every thread of the block takes part, in step; two sets of
// shared memory in turn make one barrier per call enough.
struct RowShared { float sum[2][32]; uint32_t top[32]; };
template <int NS, bool MAX> __device__ __forceinline__ void reduce_row(float* s, uint32_t& top, const Place& at, RowShared* sh) {
  const int lanes = at.n < 32 ? at.n : 32;
  for (int o = lanes >> 1; o > 0; o >>= 1) {
#pragma unroll
    for (int k = 0; k < NS; ++k) s[k] += __shfl_xor_sync(0xffffffffu, s[k], o);
    if constexpr (MAX) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  }
  if (at.n > 32) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = (at.group * at.n) >> 5, nw = at.n >> 5;
    if (lane == 0) {
#pragma unroll
      for (int k = 0; k < NS; ++k) sh->sum[k][warp] = s[k];
      if constexpr (MAX) sh->top[warp] = top;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NS; ++k) s[k] = warp_sum(lane < nw ? sh->sum[k][first + lane] : 0.f);
    if constexpr (MAX) top = __reduce_max_sync(0xffffffffu, lane < nw ? sh->top[first + lane] : 0u);
  }
}

// A row of d elements at positions s .. s + d: whole vectors [v0, v1), and `edges` elements around them.  (The last vector before the
// row's end counts as edges: reading the gain of a whole vector may take in the element behind it.)
template <typename T, bool FRAME> struct Span {
  static constexpr int W = Vec16<T>::N;
  int s, d, v0, v1, head, edges;
  __device__ __forceinline__ Span(const T* row, int width) : s(0), d(width), v0(0), v1(width / W), head(0), edges(0) {
    if constexpr (FRAME) {
      s = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
      v0 = s > 0 ? 1 : 0;
      v1 = max((s + d - 1) / W, v0);
      head = min(v0 * W, s + d) - s;
      if (v0 == 0) head = 0;
      edges = head + max(s + d - v1 * W, 0);
    }
  }
  __device__ __forceinline__ int edge(int e) const { return e < head ? e : v1 * W + (e - head) - s; }     // column of the e-th
  __device__ __forceinline__ int column(int v) const { return v * W - s; }
  __device__ __forceinline__ bool fits(const T* row) const { return !FRAME || ((reinterpret_cast<uintptr_t>(row - s) & 15u) == 0); }
};

// Vector v of a row that has whole vectors there; fits: its vectors are 16-byte aligned as those of the span's row are.
template <typename T, bool FRAME> __device__ __forceinline__ void load_row(Vec16<T>& r, const T* row, const Span<T, FRAME>& f, int v, bool fits) {
  const T* p = row + f.column(v);
  if (!FRAME || fits) r.load(p);
  else {
#pragma unroll
    for (int i = 0; i < Vec16<T>::N; ++i) reinterpret_cast<T*>(&r.raw)[i] = p[i];
  }
}
template <typename T, bool FRAME> __device__ __forceinline__ void store_row(T* row, const Span<T, FRAME>& f, int v, bool fits, const float* x) {
  constexpr int W = Vec16<T>::N;
  Vec16<T> r;
#pragma unroll
  for (int i = 0; i < W; ++i) r.set(i, x[i]);
  T* p = row + f.column(v);
  if (!FRAME || fits) r.store(p);
  else {
#pragma unroll
    for (int i = 0; i < W; ++i) p[i] = reinterpret_cast<const T*>(&r.raw)[i];
  }
}
// The gain at the columns of vector v.  Shifted bf16 pairs: words from the even element at or before the first, joined by twos.
template <typename T, bool FRAME> __device__ __forceinline__ void load_gain(Vec16<T>& r, const T* g, const Span<T, FRAME>& f, int v) {
  constexpr int W = Vec16<T>::N;
  const int c = f.column(v);
  if constexpr (!FRAME) r.load(g + c);
  else if constexpr (W == 8) {
    const T* p0 = g + c;
    const uint32_t odd = (uint32_t)(reinterpret_cast<uintptr_t>(p0) & 2u);
    const uint32_t* p = reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(p0) - odd);
    uint32_t* out = reinterpret_cast<uint32_t*>(&r.raw);
    uint32_t w[5];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __ldg(p + i);
    w[4] = odd ? __ldg(p + 4) : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = __funnelshift_r(w[i], w[i + 1], odd * 8);
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) r.set(i, __ldg(g + c + i));
  }
}
// x times the column factors of vector v (factor may be null)
template <typename T, bool FRAME> __device__ __forceinline__ void scaled(float* o, const Vec16<T>& r, const float* factor, const Span<T, FRAME>& f, int v) {
  constexpr int W = Vec16<T>::N;
#pragma unroll
  for (int i = 0; i < W; ++i) o[i] = r.get(i);
  if (factor) {
    const int c = f.column(v);
    float w[W + 4];
    if constexpr (!FRAME) {
#pragma unroll
      for (int i = 0; i < W; i += 4) *reinterpret_cast<float4*>(w + i) = __ldg(reinterpret_cast<const float4*>(factor + c + i));
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = __ldg(factor + c + i);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) o[i] = __fmul_rn(o[i], w[i]);
  }
}

// FRAME: the row's codes lie in shared memory at their positions (`mine`: 16-byte aligned, room for a word more); out with
// them, four at a time, to columns from 0.  words: rows of codes start on 4-byte boundaries.
__device__ __forceinline__ void codes_out(const uint8_t* mine, int8_t* cr, int s, int d, const Place& at, bool words) {
  if (at.n > 32) __syncthreads(); else __syncwarp();
  if (words) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(mine) + (s >> 2);
    const int sh = (s & 3) * 8, full = d >> 2;
#pragma unroll 4
    for (int i = at.t; i < full; i += at.n) reinterpret_cast<uint32_t*>(cr)[i] = __funnelshift_r(p[i], p[i + 1], sh);
    for (int c = full * 4 + at.t; c < d; c += at.n) cr[c] = (int8_t)mine[s + c];
  } else {
    for (int c = at.t; c < d; c += at.n) cr[c] = (int8_t)mine[s + c];
  }
}
// Shared memory of a row's codes, for `threads` threads.
template <typename T> __host__ __device__ constexpr int code_bytes(int threads) { return (threads * NV * Vec16<T>::N + 4 * Vec16<T>::N + 31) / 16 * 16; }
__device__ __forceinline__ uint8_t one_code(float v, const RowScale& rs) { return rs.live ? (uint8_t)code_bits(v, rs.inv) : (uint8_t)0; }

template <typename T, bool FRAME>
__global__ void __launch_bounds__(1024)
quantize_kernel(const T* __restrict__ x, const float* __restrict__ factor, int64_t M, int d, int threads, int8_t* __restrict__ codes, int64_t ldc,
                int words, float* __restrict__ scales) {
  overlap_sync();
  constexpr int W = Vec16<T>::N;
  extern __shared__ __align__(16) uint8_t staged[];
  __shared__ RowShared sh;
  const Place at(threads);
  const bool in = at.row < M;              // lanes of a row past the last still take part in the warp's exchanges
  const T* xr = x + (in ? at.row : 0) * d;
  const Span<T, FRAME> f(xr, d);
  const int v1 = in ? f.v1 : 0, edges = in ? f.edges : 0;
  Vec16<T> r[NV];
  uint32_t top = 0u;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) r[k].load(xr + f.column(v));
  }
  auto edge = [&](int c) { return factor ? __fmul_rn(to_f<T>(xr[c]), factor[c]) : to_f<T>(xr[c]); };
  if constexpr (FRAME) {
    for (int e = at.t; e < edges; e += at.n) top = max(top, abs_bits(edge(f.edge(e))));
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      float o[W];
      scaled<T, FRAME>(o, r[k], factor, f, v);
#pragma unroll
      for (int i = 0; i < W; ++i) top = max(top, abs_bits(o[i]));
    }
  }
  reduce_row<0, true>(nullptr, top, at, &sh);
  const RowScale rs = row_scale(top, 1.0f);
  if (at.t == 0 && in) scales[at.row] = rs.scale;
  int8_t* cr = codes + at.row * ldc;
  uint8_t* mine = FRAME ? staged + (size_t)at.group * code_bytes<T>(at.n) : nullptr;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      float o[W];
      uint32_t w[W / 4];
      scaled<T, FRAME>(o, r[k], factor, f, v);
      code_words<W>(w, o, rs.inv, rs.live);
      store_words<W>(FRAME ? (void*)(mine + v * W) : (void*)(cr + v * W), w);
    }
  }
  if constexpr (FRAME) {
    for (int e = at.t; e < edges; e += at.n) mine[f.s + f.edge(e)] = one_code(edge(f.edge(e)), rs);
    codes_out(mine, cr, f.s, in ? d : 0, at, words != 0);
  }
}

// Rows wider than the registers of 1024 threads hold: read twice, the second time from L2.
template <typename T, bool FRAME>
__global__ void __launch_bounds__(1024)
quantize_wide_kernel(const T* __restrict__ x, const float* __restrict__ factor, int d, int8_t* __restrict__ codes, int64_t ldc, float* __restrict__ scales) {
  overlap_sync();
  constexpr int W = Vec16<T>::N;
  __shared__ RowShared sh;
  const Place at(1024);
  const T* xr = x + at.row * d;
  int8_t* cr = codes + at.row * ldc;
  const Span<T, FRAME> f(xr, d);
  auto edge = [&](int c) { return factor ? __fmul_rn(to_f<T>(xr[c]), factor[c]) : to_f<T>(xr[c]); };
  uint32_t top = 0u;
  for (int e = at.t; e < f.edges; e += 1024) top = max(top, abs_bits(edge(f.edge(e))));
  for (int v = f.v0 + at.t; v < f.v1; v += 1024) {
    Vec16<T> r;
    float o[W];
    r.load(xr + f.column(v));
    scaled<T, FRAME>(o, r, factor, f, v);
#pragma unroll
    for (int i = 0; i < W; ++i) top = max(top, abs_bits(o[i]));
  }
  reduce_row<0, true>(nullptr, top, at, &sh);
  const RowScale rs = row_scale(top, 1.0f);
  if (at.t == 0) scales[at.row] = rs.scale;
  for (int e = at.t; e < f.edges; e += 1024) cr[f.edge(e)] = (int8_t)one_code(edge(f.edge(e)), rs);
  for (int v = f.v0 + at.t; v < f.v1; v += 1024) {
    Vec16<T> r;
    float o[W];
    uint32_t w[W / 4];
    r.load(xr + f.column(v));
    scaled<T, FRAME>(o, r, factor, f, v);
    code_words<W>(w, o, rs.inv, rs.live);
    if constexpr (!FRAME) store_words<W>(cr + v * W, w);
    else {
#pragma unroll
      for (int i = 0; i < W; ++i) cr[f.column(v) + i] = (int8_t)((w[i / 4] >> (8 * (i & 3))) & 0xffu);
    }
  }
}

template <typename T, bool FRAME>
__global__ void __launch_bounds__(1024)
dequantize_kernel(const int8_t* __restrict__ codes, int64_t ldc, const float* __restrict__ scales, int64_t M, int d, int threads, T* __restrict__ y) {
  overlap_sync();
  constexpr int W = Vec16<T>::N;
  const Place at(threads);
  if (at.row >= M) return;
  T* yr = y + at.row * d;
  const int8_t* cr = codes + at.row * ldc;
  const float s = scales[at.row];
  const Span<T, FRAME> f(yr, d);
  if constexpr (FRAME) {
    for (int e = at.t; e < f.edges; e += at.n) yr[f.edge(e)] = from_f<T>(__fmul_rn((float)cr[f.edge(e)], s));
  }
  for (int first = f.v0 + at.t; first < f.v1; first += NV * at.n) {
    uint32_t w[NV][W / 4];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + k * at.n, c = f.column(v);
      if (v >= f.v1) continue;
      if constexpr (!FRAME) {
        if constexpr (W == 8) { const uint2 q = *reinterpret_cast<const uint2*>(cr + c); w[k][0] = q.x; w[k][W / 4 - 1] = q.y; }
        else w[k][0] = *reinterpret_cast<const uint32_t*>(cr + c);
      } else {
        // words that hold the codes, joined; near the row's end the word behind the last code may lie outside the buffer
        const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(cr + c) & 3u);
        const uint32_t* p = reinterpret_cast<const uint32_t*>(cr + c - off);
        if (c + W + 4 <= d) {
          uint32_t u[W / 4 + 1];
#pragma unroll
          for (int i = 0; i <= W / 4; ++i) u[i] = __ldg(p + i);
#pragma unroll
          for (int i = 0; i < W / 4; ++i) w[k][i] = __funnelshift_r(u[i], u[i + 1], off * 8);
        } else {
#pragma unroll
          for (int i = 0; i < W / 4; ++i) w[k][i] = 0u;
#pragma unroll
          for (int i = 0; i < W; ++i) w[k][i / 4] |= (uint32_t)(uint8_t)cr[c + i] << (8 * (i & 3));
        }
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + k * at.n;
      if (v >= f.v1) continue;
      float o[W];
#pragma unroll
      for (int i = 0; i < W; ++i) o[i] = __fmul_rn((float)(int8_t)(w[k][i / 4] >> (8 * (i & 3))), s);
      store_row<T, FRAME>(yr, f, v, true, o);
    }
  }
}

template <typename T, bool FRAME>
__global__ void __launch_bounds__(1024)
rmsnorm_quantize_kernel(const T* __restrict__ x, const T* __restrict__ resid, const T* __restrict__ g, int64_t M, int d, int threads, float eps,
                        T* __restrict__ h, T* __restrict__ y, int8_t* __restrict__ codes, int64_t ldc, int words, float* __restrict__ scales) {
  overlap_sync();
  constexpr int W = Vec16<T>::N;
  extern __shared__ __align__(16) uint8_t staged[];
  __shared__ RowShared sh;
  const Place at(threads);
  const bool in = at.row < M;
  const int64_t row0 = (in ? at.row : 0) * d;
  const T* xr = x + row0;
  const T* rr = resid ? resid + row0 : nullptr;
  const Span<T, FRAME> f(xr, d);
  const int v1 = in ? f.v1 : 0, edges = in ? f.edges : 0;
  const bool fit_r = f.fits(rr), fit_h = f.fits(h + row0), fit_y = f.fits(y + row0);
  // every load of the row before the first use
  Vec16<T> xv[NV], rv[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      xv[k].load(xr + f.column(v));
      if (resid) load_row<T, FRAME>(rv[k], rr, f, v, fit_r);
    }
  }
  float sum = 0.f;
  uint32_t top = 0u;
  auto edge = [&](int c) { return resid ? __fadd_rn(to_f<T>(xr[c]), to_f<T>(rr[c])) : to_f<T>(xr[c]); };
  if constexpr (FRAME) {
    for (int e = at.t; e < edges; e += at.n) {
      const float t = edge(f.edge(e));
      sum = fmaf(t, t, sum);
      top = max(top, abs_bits(__fmul_rn(t, to_f<T>(g[f.edge(e)]))));
    }
  }
  float o[NV][W];                          // s g: all that the outputs but h need
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      Vec16<T> gv;
      load_gain<T, FRAME>(gv, g, f, v);
      float s[W];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        s[i] = resid ? __fadd_rn(xv[k].get(i), rv[k].get(i)) : xv[k].get(i);
        sum = fmaf(s[i], s[i], sum);
        o[k][i] = __fmul_rn(s[i], gv.get(i));
        top = max(top, abs_bits(o[k][i]));
      }
      if (h) store_row<T, FRAME>(h + row0, f, v, fit_h, s);
    }
  }
  reduce_row<1, true>(&sum, top, at, &sh);
  const float rstd = rsqrtf(sum / d + eps);
  const RowScale rs = row_scale(top, rstd);
  if (at.t == 0 && in) scales[at.row] = rs.scale;
  int8_t* cr = codes + at.row * ldc;
  uint8_t* mine = FRAME ? staged + (size_t)at.group * code_bytes<T>(at.n) : nullptr;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      uint32_t w[W / 4];
      code_words<W>(w, o[k], rs.inv, rs.live);
      store_words<W>(FRAME ? (void*)(mine + v * W) : (void*)(cr + v * W), w);
      if (y) {
#pragma unroll
        for (int i = 0; i < W; ++i) o[k][i] *= rstd;
        store_row<T, FRAME>(y + row0, f, v, fit_y, o[k]);
      }
    }
  }
  if constexpr (FRAME) {
    for (int e = at.t; e < edges; e += at.n) {           // read again: h, which may be x or residual, is written here only
      const int c = f.edge(e);
      const float s = edge(c), v = __fmul_rn(s, to_f<T>(g[c]));
      mine[f.s + c] = one_code(v, rs);
      if (h) h[row0 + c] = from_f<T>(s);
      if (y) y[row0 + c] = from_f<T>(v * rstd);
    }
    codes_out(mine, cr, f.s, in ? d : 0, at, words != 0);
  }
}

// The gradient of one row whose vectors are in registers; acc, acc_edge (DG): this thread's columns of the gain's gradient (DG: a
// thread has one edge at most).  Contractions are spelled out: dx does not depend on whether dg is asked for.
template <typename T, bool FRAME, bool DG>
__device__ __forceinline__ void norm_row_bwd(const Vec16<T>* hv, const Vec16<T>* dv, const Vec16<T>* rv, const T* g, const T* hr, const T* dr, const T* rr,
                                             const Span<T, FRAME>& f, int v1, int edges, const Place& at, RowShared* sh, float eps, T* dx,
                                             bool fit_dx, float (*acc)[Vec16<T>::N], float* acc_edge) {
  constexpr int W = Vec16<T>::N;
  float s[2] = {0.f, 0.f};
  if constexpr (FRAME) {
    for (int e = at.t; e < edges; e += at.n) {
      const int c = f.edge(e);
      const float hh = to_f<T>(hr[c]);
      s[0] = fmaf(hh, hh, s[0]);
      s[1] = fmaf(__fmul_rn(to_f<T>(dr[c]), to_f<T>(g[c])), hh, s[1]);
    }
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      Vec16<T> gv;
      load_gain<T, FRAME>(gv, g, f, v);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float hh = hv[k].get(i);
        s[0] = fmaf(hh, hh, s[0]);
        s[1] = fmaf(__fmul_rn(dv[k].get(i), gv.get(i)), hh, s[1]);
      }
    }
  }
  uint32_t none = 0u;
  reduce_row<2, false>(s, none, at, sh);
  const float rstd = rsqrtf(s[0] / f.d + eps);
  const float c = rstd * rstd * (s[1] / f.d);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      Vec16<T> gv;
      load_gain<T, FRAME>(gv, g, f, v);
      float o[W];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float hh = hv[k].get(i), dd = dv[k].get(i);
        const float t = fmaf(-hh, c, __fmul_rn(dd, gv.get(i)));
        o[i] = rr ? fmaf(rstd, t, rv[k].get(i)) : __fmul_rn(rstd, t);
        if constexpr (DG) acc[k][i] = fmaf(dd, __fmul_rn(hh, rstd), acc[k][i]);
      }
      store_row<T, FRAME>(dx, f, v, fit_dx, o);
    }
  }
  if constexpr (FRAME)
    for (int e = at.t; e < edges; e += at.n) {           // read again: dx, which may be dy or residual, is written here only
      const int q = f.edge(e);
      const float hh = to_f<T>(hr[q]), dd = to_f<T>(dr[q]);
      const float t = fmaf(-hh, c, __fmul_rn(dd, to_f<T>(g[q])));
      dx[q] = from_f<T>(rr ? fmaf(rstd, t, to_f<T>(rr[q])) : __fmul_rn(rstd, t));
      if constexpr (DG) *acc_edge = fmaf(dd, __fmul_rn(hh, rstd), *acc_edge);
    }
}

template <typename T, bool FRAME>
__global__ void __launch_bounds__(1024)
rmsnorm_bwd_kernel(const T* __restrict__ dy, const T* __restrict__ h, const T* __restrict__ g, const T* __restrict__ resid, int64_t M, int d, int threads,
                   float eps, T* __restrict__ dx) {
  overlap_sync();
  __shared__ RowShared sh;
  const Place at(threads);
  const bool in = at.row < M;
  const int64_t row0 = (in ? at.row : 0) * d;
  const T *hr = h + row0, *dr = dy + row0, *rr = resid ? resid + row0 : nullptr;
  const Span<T, FRAME> f(hr, d);
  const int v1 = in ? f.v1 : 0;
  const bool fit_d = f.fits(dr), fit_r = f.fits(rr);
  Vec16<T> hv[NV], dv[NV], rv[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      hv[k].load(hr + f.column(v));
      load_row<T, FRAME>(dv[k], dr, f, v, fit_d);
      if (rr) load_row<T, FRAME>(rv[k], rr, f, v, fit_r);
    }
  }
  norm_row_bwd<T, FRAME, false>(hv, dv, rv, g, hr, dr, rr, f, v1, in ? f.edges : 0, at, &sh, eps, dx + row0, f.fits(dx + row0), nullptr, nullptr);
}

// With the gain's gradient: the blocks walk the rows, each group of threads every (groups of the grid)-th one, and keep their
// columns' sums in registers; the groups of a block add theirs up in order, and each block leaves one row of partial
// sums [gridDim.x, d] that dg_reduce_kernel adds up in order: the result does not depend on scheduling.  A group with more than one
// row has a stride of a multiple of 8 rows, so its rows all have the same shift.
// MAXT 512: a thread copies its share of the next row into shared memory while it works on this one; rows that need more threads
// leave no room for that.
template <typename T, bool FRAME, int MAXT>
__global__ void __launch_bounds__(MAXT, 1)
rmsnorm_bwd_gain_kernel(const T* __restrict__ dy, const T* __restrict__ h, const T* __restrict__ g, const T* __restrict__ resid, int64_t M, int d,
                        int threads, float eps, T* __restrict__ dx, float* __restrict__ partial) {
  overlap_sync();
  constexpr int W = Vec16<T>::N;
  constexpr bool AHEAD = MAXT <= 512;
  extern __shared__ __align__(16) uint8_t staged[];      // AHEAD: [2][array][k][thread] vectors of 16 bytes; in the end sums
  __shared__ RowShared sh[2];
  const Place at(threads);
  const int per = blockDim.x / threads;
  const int64_t groups = (int64_t)gridDim.x * per;
  const int narr = resid ? 3 : 2;
  const Span<T, FRAME> f(h + at.row * d, d);
  const bool fit_d = f.fits(dy + at.row * d), fit_r = f.fits(resid + at.row * d), fit_dx = f.fits(dx + at.row * d);
  auto slot = [&](int stage, int a, int k) { return staged + ((size_t)((stage * narr + a) * NV + k) * blockDim.x + threadIdx.x) * 16; };
  auto fetch = [&](int64_t row, int stage) {
    if (AHEAD && row < M) {
#pragma unroll
      for (int a = 0; a < 3; ++a) {
        if ((a == 1 && !fit_d) || (a == 2 && (!resid || !fit_r))) continue;
        const T* p = (a == 0 ? h : a == 1 ? dy : resid) + row * d;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int v = f.v0 + k * at.n + at.t;
          if (v < f.v1)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(slot(stage, a, k))), "l"(p + f.column(v)) : "memory");
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto take = [&](Vec16<T>& r, int stage, int a, int k, const T* p, bool fits) {
    if (AHEAD && fits) r.raw = *reinterpret_cast<const decltype(r.raw)*>(slot(stage, a, k));
    else load_row<T, FRAME>(r, p, f, f.v0 + k * at.n + at.t, fits);
  };
  float acc[NV][W], acc_edge = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < W; ++i) acc[k][i] = 0.f;
  fetch(at.row, 0);
  int stage = 0;
  // every thread of the block goes through the same number of rows
  for (int64_t row = at.row, lead = (int64_t)blockIdx.x * per; lead < M; row += groups, lead += groups, stage ^= 1) {
    const bool in = row < M;
    const int64_t row0 = (in ? row : 0) * d;
    const T *hr = h + row0, *dr = dy + row0, *rr = resid ? resid + row0 : nullptr;
    Vec16<T> hv[NV], dv[NV], rv[NV];
    fetch(row + groups, stage ^ 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (in && f.v0 + k * at.n + at.t < f.v1) {
        take(hv[k], stage, 0, k, hr, true);
        take(dv[k], stage, 1, k, dr, fit_d);
        if (rr) take(rv[k], stage, 2, k, rr, fit_r);
      }
    }
    norm_row_bwd<T, FRAME, true>(hv, dv, rv, g, hr, dr, rr, f, in ? f.v1 : 0, in ? f.edges : 0, at, &sh[stage], eps, dx + row0, fit_dx, acc, &acc_edge);
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  float* sums = reinterpret_cast<float*>(staged);
  for (int c = threadIdx.x; c < d; c += blockDim.x) sums[c] = 0.f;
  __syncthreads();
  for (int gr = 0; gr < per; ++gr) {
    if (at.group == gr) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int v = f.v0 + k * at.n + at.t;
#pragma unroll
        for (int i = 0; i < W; ++i) if (v < f.v1) sums[f.column(v) + i] += acc[k][i];
      }
      if (FRAME && at.t < f.edges) sums[f.edge(at.t)] += acc_edge;
    }
    __syncthreads();
  }
  float* out = partial + (int64_t)blockIdx.x * d;
  for (int c = threadIdx.x; c < d; c += blockDim.x) out[c] = sums[c];
}

// 32 columns per block, 8 threads per column, each adding every eighth partial row in order.
__global__ void __launch_bounds__(256) dg_reduce_kernel(const float* __restrict__ partial, int rows, int d, float* __restrict__ dg) {
  overlap_sync();
  __shared__ float sh[8][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
  float s = 0.f;
  if (c < d)
#pragma unroll 4
    for (int r = part; r < rows; r += 8) s += partial[(int64_t)r * d + c];
  sh[part][threadIdx.x & 31] = s;
  __syncthreads();
  if (part == 0 && c < d) {
#pragma unroll
    for (int p = 1; p < 8; ++p) s += sh[p][threadIdx.x];
    dg[c] = s;
  }
}

bool al(const void* p, int a) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(a - 1)) == 0; }

// Threads per row: as many as give each NV accesses, a power of two up to a warp, else whole warps; at least `least`.
template <typename T> int row_threads(int d, int least = 1) {
  const int nv = (d + Vec16<T>::N - 1) / Vec16<T>::N, need = (nv + NV - 1) / NV;
  if (need > 32) return (need + 31) / 32 * 32;
  int n = least;
  while (n < need) n *= 2;
  return n;
}
// Blocks of 256 threads where a row takes a warp or less, else a block per row.
struct Shape { int threads, block; int64_t blocks; };
Shape shape_of(int64_t M, int threads) {
  Shape s;
  s.threads = threads;
  s.block = threads <= 32 ? 256 : threads;
  const int per = s.block / threads;
  s.blocks = (M + per - 1) / per;
  return s;
}

}  // namespace

cudaError_t quantize_rows(int dt, const void* x, const float* factor, int64_t M, int d, int8_t* codes, int64_t ldc, float* scales, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int W = Vec16<T>::N;
    const bool frame = d % W != 0 || ldc % W != 0 || !al(x, 16) || !al(factor, 16) || !al(codes, W);
    const int threads = row_threads<T>(d);
    if (threads > 1024)
      return frame ? launch_overlapped(quantize_wide_kernel<T, true>, dim3((unsigned)M), dim3(1024), 0, st, (const T*)x, factor, d, codes, ldc, scales)
                   : launch_overlapped(quantize_wide_kernel<T, false>, dim3((unsigned)M), dim3(1024), 0, st, (const T*)x, factor, d, codes, ldc, scales);
    const Shape s = shape_of(M, threads);
    const int words = ldc % 4 == 0 && al(codes, 4);
    const size_t smem = frame ? (size_t)(s.block / threads) * code_bytes<T>(threads) : 0;
    auto go = [&](auto kernel) {
      return launch_overlapped(kernel, dim3((unsigned)s.blocks), dim3(s.block), smem, st, (const T*)x, factor, M, d, threads, codes, ldc, words, scales);
    };
    return frame ? go(quantize_kernel<T, true>) : go(quantize_kernel<T, false>);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

cudaError_t dequantize_rows(int dt, const int8_t* codes, int64_t ldc, const float* scales, int64_t M, int d, void* y, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int W = Vec16<T>::N;
    const bool frame = d % W != 0 || ldc % W != 0 || !al(y, 16) || !al(codes, W);
    int threads = row_threads<T>(d);
    if (threads > 1024) threads = 1024;
    const Shape s = shape_of(M, threads);
    return launch_overlapped(frame ? dequantize_kernel<T, true> : dequantize_kernel<T, false>, dim3((unsigned)s.blocks), dim3(s.block), 0, st, codes, ldc,
                             scales, M, d, threads, (T*)y);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

cudaError_t rmsnorm_quantize(int dt, const void* x, const void* resid, const void* g, int64_t M, int d, float eps, void* h, void* y, int8_t* codes,
                             int64_t ldc, float* scales, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int W = Vec16<T>::N;
    const bool frame = d % W != 0 || ldc % W != 0 || !al(x, 16) || !al(g, 16) || !al(resid, 16) || !al(h, 16) || !al(y, 16) || !al(codes, W);
    const int threads = row_threads<T>(d);
    const Shape s = shape_of(M, threads);
    const int words = ldc % 4 == 0 && al(codes, 4);
    const size_t smem = frame ? (size_t)(s.block / threads) * code_bytes<T>(threads) : 0;
    auto go = [&](auto kernel) {
      return launch_overlapped(kernel, dim3((unsigned)s.blocks), dim3(s.block), smem, st, (const T*)x, (const T*)resid, (const T*)g, M, d, threads, eps,
                               (T*)h, (T*)y, codes, ldc, words, scales);
    };
    return frame ? go(rmsnorm_quantize_kernel<T, true>) : go(rmsnorm_quantize_kernel<T, false>);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

namespace {
template <typename T, bool FRAME, int MAXT>
cudaError_t launch_gain(const void* dy, const void* h, const void* g, const void* resid, int64_t M, int d, int threads, int block, int64_t blocks,
                        float eps, void* dx, float* partial, cudaStream_t st) {
  constexpr int MOST = MAXT <= 512 ? 2 * 3 * NV * 512 * 16 : ROWS_MAX_WIDTH * 4;
  static_assert(MOST >= ROWS_MAX_WIDTH * 4 && MOST <= 230000, "");
  const auto kernel = rmsnorm_bwd_gain_kernel<T, FRAME, MAXT>;
  static PerDeviceOnce once;
  const int dev = current_device();
  if (once.needed(dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST);
    if (e != cudaSuccess) return e;
    once.done(dev);
  }
  size_t smem = (size_t)d * 4;
  if constexpr (MAXT <= 512) smem = std::max(smem, (size_t)2 * (resid ? 3 : 2) * NV * block * 16);
  return launch_overlapped(kernel, dim3((unsigned)blocks), dim3(block), smem, st, (const T*)dy, (const T*)h, (const T*)g,
                           (const T*)resid, M, d, threads, eps, (T*)dx, partial);
}
}  // namespace

size_t rmsnorm_dg_scratch_floats(int64_t M, int d) { return (size_t)(M < DG_PARTIAL_ROWS ? M : DG_PARTIAL_ROWS) * d; }

cudaError_t rmsnorm_gain_bwd(int dt, const void* dy, const void* h, const void* g, const void* resid, int64_t M, int d, float eps, void* dx, float* dg,
                             float* partial, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int W = Vec16<T>::N;
    const bool frame = d % W != 0 || !al(dy, 16) || !al(h, 16) || !al(g, 16) || !al(resid, 16) || !al(dx, 16);
    const int threads = row_threads<T>(d, frame ? 2 * W : 1);       // an edge per thread
    if (!dg) {
      const Shape s = shape_of(M, threads);
      auto go = [&](auto kernel) {
        return launch_overlapped(kernel, dim3((unsigned)s.blocks), dim3(s.block), 0, st, (const T*)dy, (const T*)h, (const T*)g, (const T*)resid, M, d,
                                 threads, eps, (T*)dx);
      };
        return frame ? go(rmsnorm_bwd_kernel<T, true>) : go(rmsnorm_bwd_kernel<T, false>);
    }
    const int per = threads > 512 ? 1 : 512 / threads, block = per * threads;
    int64_t blocks = num_sms() < DG_PARTIAL_ROWS ? num_sms() : DG_PARTIAL_ROWS;
    if (blocks * per >= M) blocks = (M + per - 1) / per;
    else if (blocks >= 8) blocks = blocks / 8 * 8;
    else if (frame) blocks = M < 8 ? M : 8;
    const cudaError_t e = threads > 512 ? (frame ? launch_gain<T, true, 1024>(dy, h, g, resid, M, d, threads, block, blocks, eps, dx, partial, st)
                                                 : launch_gain<T, false, 1024>(dy, h, g, resid, M, d, threads, block, blocks, eps, dx, partial, st))
                                        : (frame ? launch_gain<T, true, 512>(dy, h, g, resid, M, d, threads, block, blocks, eps, dx, partial, st)
                                                 : launch_gain<T, false, 512>(dy, h, g, resid, M, d, threads, block, blocks, eps, dx, partial, st));
    if (e != cudaSuccess) return e;
    return launch_overlapped(dg_reduce_kernel, dim3((unsigned)((d + 31) / 32)), dim3(256), 0, st, (const float*)partial, (int)blocks, d, dg);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

}  // namespace sl
