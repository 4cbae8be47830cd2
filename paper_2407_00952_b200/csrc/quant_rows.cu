// Rows in 8 bits: the kernels around the int8 products of a layer whose frozen weight is held as codes.
//   quantize     v = x f (column factors f or 1),  a = max_c |v|,  code = rint(v * (127 / a)),  scale = a / 127
//   norm         s = x + resid,  rstd = (mean s^2 + eps)^-1/2,  v = s g,  code = rint(v * (127 / max|v|)),  scale = max|v| rstd / 127
//   norm, gradient   w = dy g,  dx = resid + rstd (w - h rstd^2 mean(w h)),  dg_c = sum_m dy h rstd
//   dequantize   y = code * scale
// The codes of a normalised row do not depend on rstd: it scales the row and its maximum alike, so one pass over the row
// collects sum s^2 and max |s g| together and every rounding decision is one of fp32 products and one fp32 division, whatever
// the order of the sum.  All arithmetic is fp32; h and y are rounded once to the buffers' type, the norm sees s before that.
// Bounded by HBM: a row lives in registers between its reduction and its output (4 accesses of 16 bytes per thread, up to 1024
// threads per row; a warp per row up to 128 accesses), so it is read once.  Maxima are taken on the bits of |v| as
// unsigned integers: one instruction per value and per warp, and a NaN or infinity is larger than every finite value.
#include "common.cuh"
#include "host_common.h"
#include "kernels.h"
#include "launch.cuh"

namespace sl {
namespace {

constexpr float TINY_ROW = 1e-36f;       // below this 127 / max overflows: the row is held as zero
constexpr int NV_VEC = 4, NV_ONE = 16;   // accesses per thread: of 16 bytes, of one element

// W consecutive elements of type T as floats: W = 16 / sizeof(T) with aligned 16-byte accesses, or W = 1.
template <typename T, int W> struct Acc {
  T raw[W];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (W > 1) *reinterpret_cast<uint4*>(raw) = *reinterpret_cast<const uint4*>(p);
    else raw[0] = p[0];
  }
  __device__ __forceinline__ float get(int i) const { return to_f<T>(raw[i]); }
};
template <typename T, int W> __device__ __forceinline__ void store_acc(T* p, const float* v) {
  if constexpr (W > 1) {
    Vec16<T> o;
#pragma unroll
    for (int i = 0; i < W; ++i) o.set(i, v[i]);
    o.store(p);
  } else {
    p[0] = from_f<T>(v[0]);
  }
}
template <int W> __device__ __forceinline__ void load_f32(float* v, const float* p) {
  if constexpr (W == 1) v[0] = p[0];
  else {
#pragma unroll
    for (int i = 0; i < W; i += 4) *reinterpret_cast<float4*>(v + i) = *reinterpret_cast<const float4*>(p + i);
  }
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// rint(v * inv) for |v * inv| < 128 in the low byte of the result: the product is rounded to fp32 first, then adding 1.5 * 2^23
// leaves the nearest integer (ties to even) in the low bits of the sum.
__device__ __forceinline__ uint32_t code_bits(float v, float inv) { return __float_as_uint(__fadd_rn(__fmul_rn(v, inv), 12582912.0f)); }
template <int W> __device__ __forceinline__ void store_codes(int8_t* p, const float* v, float inv, bool live) {
  if constexpr (W == 1) {
    p[0] = live ? (int8_t)(code_bits(v[0], inv) & 0xffu) : (int8_t)0;
  } else {
    uint32_t w[W / 4];
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const uint32_t lo = __byte_perm(code_bits(v[4 * i], inv), code_bits(v[4 * i + 1], inv), 0x0040);
      const uint32_t hi = __byte_perm(code_bits(v[4 * i + 2], inv), code_bits(v[4 * i + 3], inv), 0x0040);
      w[i] = live ? __byte_perm(lo, hi, 0x5410) : 0u;
    }
    if constexpr (W == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(p) = w[0];
  }
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

// Sums and maxima over the threads of a row: a warp, or all warps of the block.
struct RowShared { float sum[2][32]; uint32_t top[32]; };
template <bool WARP, int NS, bool MAX> __device__ __forceinline__ void reduce_row(float* s, uint32_t& top, RowShared* sh) {
#pragma unroll
  for (int k = 0; k < NS; ++k) s[k] = warp_sum(s[k]);
  if constexpr (MAX) top = __reduce_max_sync(0xffffffffu, top);
  if constexpr (!WARP) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = blockDim.x >> 5;
    if (lane == 0) {
#pragma unroll
      for (int k = 0; k < NS; ++k) sh->sum[k][warp] = s[k];
      if constexpr (MAX) sh->top[warp] = top;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NS; ++k) s[k] = warp_sum(lane < nw ? sh->sum[k][lane] : 0.f);
    if constexpr (MAX) top = __reduce_max_sync(0xffffffffu, lane < nw ? sh->top[lane] : 0u);
  }
}

// Which row, which thread of it, how many: a warp per row (eight rows per block), or a block per row.
template <bool WARP> struct Place {
  int64_t row; int t, n;
  __device__ __forceinline__ Place() {
    row = WARP ? (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
    t = WARP ? threadIdx.x & 31 : threadIdx.x;
    n = WARP ? 32 : blockDim.x;
  }
};

// NV == 0: any width, the row is read twice (the second time from L1 or L2).
template <typename T, int W, int NV, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : 1024)
quantize_kernel(const T* __restrict__ x, const float* __restrict__ factor, int64_t M, int d, int8_t* __restrict__ codes, int64_t ldc,
                float* __restrict__ scales) {
  overlap_sync();
  __shared__ RowShared sh;
  const Place<WARP> at;
  if (at.row >= M) return;                 // whole warps; a block per row has no row to spare
  const T* xr = x + at.row * d;
  int8_t* cr = codes + at.row * ldc;
  const int nacc = d / W;
  uint32_t top = 0u;
  auto values = [&](int a, float* v) {
    Acc<T, W> r; r.load(xr + (int64_t)a * W);
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = r.get(i);
    if (factor) {
      float f[W];
      load_f32<W>(f, factor + (int64_t)a * W);
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] = __fmul_rn(v[i], f[i]);
    }
  };
  if constexpr (NV > 0) {
    float v[NV][W];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int a = k * at.n + at.t;
      if (a < nacc) {
        values(a, v[k]);
#pragma unroll
        for (int i = 0; i < W; ++i) top = max(top, abs_bits(v[k][i]));
      }
    }
    reduce_row<WARP, 0, true>(nullptr, top, &sh);
    const RowScale rs = row_scale(top, 1.0f);
    if (at.t == 0) scales[at.row] = rs.scale;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int a = k * at.n + at.t;
      if (a < nacc) store_codes<W>(cr + (int64_t)a * W, v[k], rs.inv, rs.live);
    }
  } else {
    for (int a = at.t; a < nacc; a += at.n) {
      float v[W];
      values(a, v);
#pragma unroll
      for (int i = 0; i < W; ++i) top = max(top, abs_bits(v[i]));
    }
    reduce_row<WARP, 0, true>(nullptr, top, &sh);
    const RowScale rs = row_scale(top, 1.0f);
    if (at.t == 0) scales[at.row] = rs.scale;
    for (int a = at.t; a < nacc; a += at.n) {
      float v[W];
      values(a, v);
      store_codes<W>(cr + (int64_t)a * W, v, rs.inv, rs.live);
    }
  }
}

template <typename T, int W>
__global__ void __launch_bounds__(256)
dequantize_kernel(const int8_t* __restrict__ codes, int64_t ldc, const float* __restrict__ scales, int64_t M, int d, T* __restrict__ y) {
  overlap_sync();
  const int nacc = d / W;
  const int64_t total = M * nacc, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t k = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; k < total; k += step) {
    const int64_t row = k / nacc;
    const int64_t c = (k - row * nacc) * W;
    const float s = scales[row];
    const int8_t* p = codes + row * ldc + c;
    int8_t q[W];
    if constexpr (W == 8) *reinterpret_cast<uint2*>(q) = *reinterpret_cast<const uint2*>(p);
    else if constexpr (W == 4) *reinterpret_cast<uint32_t*>(q) = *reinterpret_cast<const uint32_t*>(p);
    else q[0] = p[0];
    float v[W];
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = __fmul_rn((float)q[i], s);
    store_acc<T, W>(y + row * d + c, v);
  }
}

template <typename T, int W, int NV, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : 1024)
rmsnorm_quantize_kernel(const T* __restrict__ x, const T* __restrict__ resid, const T* __restrict__ g, int64_t M, int d, float eps,
                        T* __restrict__ h, T* __restrict__ y, int8_t* __restrict__ codes, int64_t ldc, float* __restrict__ scales) {
  overlap_sync();
  __shared__ RowShared sh;
  const Place<WARP> at;
  if (at.row >= M) return;
  const int nacc = d / W;
  const int64_t row0 = at.row * d;
  float s[NV][W];
  float sum = 0.f;
  uint32_t top = 0u;
  // every load of the row before the first use
  Acc<T, W> xv[NV], rv[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int a = k * at.n + at.t;
    if (a < nacc) {
      xv[k].load(x + row0 + (int64_t)a * W);
      if (resid) rv[k].load(resid + row0 + (int64_t)a * W);
    }
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int a = k * at.n + at.t;
    if (a < nacc) {
      Acc<T, W> gv; gv.load(g + (int64_t)a * W);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float t = resid ? __fadd_rn(xv[k].get(i), rv[k].get(i)) : xv[k].get(i);
        sum += t * t;
        s[k][i] = t;
        top = max(top, abs_bits(__fmul_rn(t, gv.get(i))));
      }
      if (h) store_acc<T, W>(h + row0 + (int64_t)a * W, s[k]);
    }
  }
  reduce_row<WARP, 1, true>(&sum, top, &sh);
  const float rstd = rsqrtf(sum / d + eps);
  const RowScale rs = row_scale(top, rstd);
  if (at.t == 0) scales[at.row] = rs.scale;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int a = k * at.n + at.t;
    if (a < nacc) {
      Acc<T, W> gv; gv.load(g + (int64_t)a * W);
      float v[W];
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] = __fmul_rn(s[k][i], gv.get(i));
      store_codes<W>(codes + at.row * ldc + (int64_t)a * W, v, rs.inv, rs.live);
      if (y) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] *= rstd;
        store_acc<T, W>(y + row0 + (int64_t)a * W, v);
      }
    }
  }
}

// DG: the gain's gradient too.  The blocks walk the rows and keep their columns' sums in registers; each leaves one row of
// partial sums [gridDim.x, d] that dg_reduce_kernel adds up in order, so the result does not depend on scheduling.
template <typename T, int W, int NV, bool WARP, bool DG>
__global__ void __launch_bounds__(WARP ? 256 : 1024)
rmsnorm_bwd_kernel(const T* __restrict__ dy, const T* __restrict__ h, const T* __restrict__ g, const T* __restrict__ resid, int64_t M, int d,
                   float eps, T* __restrict__ dx, float* __restrict__ partial) {
  static_assert(!(WARP && DG), "the gain's gradient takes a block per row");
  overlap_sync();
  __shared__ RowShared sh[2];
  const Place<WARP> at;
  const int nacc = d / W;
  float acc[DG ? NV : 1][W];
  if constexpr (DG) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < W; ++i) acc[k][i] = 0.f;
  }
  int flip = 0;                            // consecutive rows reduce through different shared memory: one barrier per row
  for (int64_t row = at.row; row < M; row += WARP ? M : (int64_t)gridDim.x, flip ^= 1) {
    const int64_t row0 = row * d;
    Acc<T, W> hv[NV], dv[NV], rv[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int a = k * at.n + at.t;
      if (a < nacc) {
        hv[k].load(h + row0 + (int64_t)a * W);
        dv[k].load(dy + row0 + (int64_t)a * W);
        if (resid) rv[k].load(resid + row0 + (int64_t)a * W);
      }
    }
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int a = k * at.n + at.t;
      if (a < nacc) {
        Acc<T, W> gv; gv.load(g + (int64_t)a * W);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float hh = hv[k].get(i);
          s[0] = fmaf(hh, hh, s[0]);
          s[1] = fmaf(__fmul_rn(dv[k].get(i), gv.get(i)), hh, s[1]);
        }
      }
    }
    uint32_t none = 0u;
    reduce_row<WARP, 2, false>(s, none, &sh[flip]);
    const float rstd = rsqrtf(s[0] / d + eps);
    const float c = rstd * rstd * (s[1] / d);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int a = k * at.n + at.t;
      if (a < nacc) {
        Acc<T, W> gv; gv.load(g + (int64_t)a * W);
        float v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float hh = hv[k].get(i), dd = dv[k].get(i);
          // (contractions spelled out: dx does not depend on whether dg is asked for)
          const float t = fmaf(-hh, c, __fmul_rn(dd, gv.get(i)));
          v[i] = resid ? fmaf(rstd, t, rv[k].get(i)) : __fmul_rn(rstd, t);
          if constexpr (DG) acc[k][i] = fmaf(dd, __fmul_rn(hh, rstd), acc[k][i]);
        }
        store_acc<T, W>(dx + row0 + (int64_t)a * W, v);
      }
    }
  }
  if constexpr (DG) {
    float* out = partial + (int64_t)blockIdx.x * d;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int a = k * at.n + at.t;
      if (a < nacc) {
#pragma unroll
        for (int i = 0; i < W; ++i) out[(int64_t)a * W + i] = acc[k][i];
      }
    }
  }
}

// 32 columns per block, 8 threads per column, each adding every eighth partial row in order.
__global__ void __launch_bounds__(256) dg_reduce_kernel(const float* __restrict__ partial, int rows, int d, float* __restrict__ dg) {
  overlap_sync();
  __shared__ float sh[8][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
  float s = 0.f;
  if (c < d)
    for (int r = part; r < rows; r += 8) s += partial[(int64_t)r * d + c];
  sh[part][threadIdx.x & 31] = s;
  __syncthreads();
  if (part == 0 && c < d) {
#pragma unroll
    for (int p = 1; p < 8; ++p) s += sh[p][threadIdx.x];
    dg[c] = s;
  }
}

bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Threads per row where each takes nv accesses: 32 for up to 32 * nv (a warp per row), else whole warps of a block of its own.
int row_threads(int nacc, int nv) { return (nacc + 32 * nv - 1) / (32 * nv) * 32; }

}  // namespace

cudaError_t quantize_rows(int dt, const void* x, const float* factor, int64_t M, int d, int8_t* codes, int64_t ldc, float* scales, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int N = Vec16<T>::N;
    const bool vec = d % N == 0 && ldc % N == 0 && al16(x) && (!factor || al16(factor)) && (reinterpret_cast<uintptr_t>(codes) % N) == 0;
    auto go = [&](auto kernel, int threads, bool warp) -> cudaError_t {
      const int64_t blocks = warp ? (M + 7) / 8 : M;
      return launch_overlapped(kernel, dim3((unsigned)blocks), dim3(warp ? 256 : threads), 0, st, (const T*)x, factor, M, d, codes, ldc, scales);
    };
    const int nacc = vec ? d / N : d, threads = row_threads(nacc, vec ? NV_VEC : NV_ONE);
    if (vec) {
      if (threads == 32) return go(quantize_kernel<T, N, NV_VEC, true>, 32, true);
      if (threads <= 1024) return go(quantize_kernel<T, N, NV_VEC, false>, threads, false);
      return go(quantize_kernel<T, N, 0, false>, 1024, false);
    }
    if (threads == 32) return go(quantize_kernel<T, 1, NV_ONE, true>, 32, true);
    if (threads <= 1024) return go(quantize_kernel<T, 1, NV_ONE, false>, threads, false);
    return go(quantize_kernel<T, 1, 0, false>, 1024, false);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

cudaError_t dequantize_rows(int dt, const int8_t* codes, int64_t ldc, const float* scales, int64_t M, int d, void* y, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int N = Vec16<T>::N;
    const bool vec = d % N == 0 && ldc % N == 0 && al16(y) && (reinterpret_cast<uintptr_t>(codes) % N) == 0;
    const int64_t total = M * (vec ? d / N : d), most = (int64_t)num_sms() * 8 * 4;
    const int64_t blocks = (total + 255) / 256;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    if (vec) return launch_overlapped(dequantize_kernel<T, N>, dim3(grid), dim3(256), 0, st, codes, ldc, scales, M, d, (T*)y);
    return launch_overlapped(dequantize_kernel<T, 1>, dim3(grid), dim3(256), 0, st, codes, ldc, scales, M, d, (T*)y);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

cudaError_t rmsnorm_quantize(int dt, const void* x, const void* resid, const void* g, int64_t M, int d, float eps, void* h, void* y, int8_t* codes,
                             int64_t ldc, float* scales, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int N = Vec16<T>::N;
    const bool vec = d % N == 0 && ldc % N == 0 && al16(x) && al16(g) && al16(resid) && al16(h) && al16(y) && (reinterpret_cast<uintptr_t>(codes) % N) == 0;
    auto go = [&](auto kernel, int threads, bool warp) -> cudaError_t {
      const int64_t blocks = warp ? (M + 7) / 8 : M;
      return launch_overlapped(kernel, dim3((unsigned)blocks), dim3(warp ? 256 : threads), 0, st, (const T*)x, (const T*)resid, (const T*)g, M, d, eps,
                               (T*)h, (T*)y, codes, ldc, scales);
    };
    const int nacc = vec ? d / N : d, threads = row_threads(nacc, vec ? NV_VEC : NV_ONE);
    if (vec) return threads == 32 ? go(rmsnorm_quantize_kernel<T, N, NV_VEC, true>, 32, true) : go(rmsnorm_quantize_kernel<T, N, NV_VEC, false>, threads, false);
    return threads == 32 ? go(rmsnorm_quantize_kernel<T, 1, NV_ONE, true>, 32, true) : go(rmsnorm_quantize_kernel<T, 1, NV_ONE, false>, threads, false);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

// Partial rows of the gain's gradient: blocks that walk the rows.
static int dg_blocks(int64_t M) { return (int)(M < DG_PARTIAL_ROWS ? M : DG_PARTIAL_ROWS); }
size_t rmsnorm_dg_scratch_floats(int64_t M, int d) { return (size_t)dg_blocks(M) * d; }

cudaError_t rmsnorm_gain_bwd(int dt, const void* dy, const void* h, const void* g, const void* resid, int64_t M, int d, float eps, void* dx, float* dg,
                             float* partial, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int N = Vec16<T>::N;
    const bool vec = d % N == 0 && al16(dy) && al16(h) && al16(g) && al16(resid) && al16(dx);
    const int nacc = vec ? d / N : d, threads = row_threads(nacc, vec ? NV_VEC : NV_ONE);
    auto go = [&](auto kernel, int64_t blocks, int block) -> cudaError_t {
      return launch_overlapped(kernel, dim3((unsigned)blocks), dim3(block), 0, st, (const T*)dy, (const T*)h, (const T*)g, (const T*)resid, M, d, eps,
                               (T*)dx, partial);
    };
    if (dg) {
      const int blocks = dg_blocks(M);
      const cudaError_t e = vec ? go(rmsnorm_bwd_kernel<T, N, NV_VEC, false, true>, blocks, threads) : go(rmsnorm_bwd_kernel<T, 1, NV_ONE, false, true>, blocks, threads);
      if (e != cudaSuccess) return e;
      return launch_overlapped(dg_reduce_kernel, dim3((unsigned)((d + 31) / 32)), dim3(256), 0, st, (const float*)partial, blocks, d, dg);
    }
    if (threads == 32) return vec ? go(rmsnorm_bwd_kernel<T, N, NV_VEC, true, false>, (M + 7) / 8, 256) : go(rmsnorm_bwd_kernel<T, 1, NV_ONE, true, false>, (M + 7) / 8, 256);
    return vec ? go(rmsnorm_bwd_kernel<T, N, NV_VEC, false, false>, M, threads) : go(rmsnorm_bwd_kernel<T, 1, NV_ONE, false, false>, M, threads);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

}  // namespace sl
