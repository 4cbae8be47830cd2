// Rows in 8 bits: the kernels around the int8 products of a layer whose frozen weight is held as codes.
//   quantize     v = x f (column factors f or 1),  a = max_c |v|,  code = rint(v * (127 / a)),  scale = a / 127
//   norm         s = x + resid,  rstd = (mean s^2 + eps)^-1/2,  v = s g,  code = rint(v * (127 / max|v|)),  scale = max|v| rstd / 127
//   norm, gradient   w = dy g,  dx = resid + rstd (w - h rstd^2 mean(w h)),  dg_c = sum_m dy h rstd
//   dequantize   y = code * scale
// The codes of a normalised row do not depend on rstd: it scales the row and its maximum alike, so one pass over the row
// collects sum s^2 and max |s g| together and every rounding decision is one of fp32 products and one fp32 division, whatever
// the order of the sum.  All arithmetic is fp32; h and y are rounded once to the buffers' type, the norm sees s before that.
// Bounded by HBM: a row lives in registers between its reduction and its output (4 or 8 accesses of 16 bytes per thread; 1 to 32
// lanes per row where a warp holds it, else whole warps, up to 1024 threads), so it is read once.  Rows are many and short-lived: a
// block each (walking the rows with copies one row ahead was 10-20 % slower where no sums are carried from row to row).
// 8192 x 4096 bf16, and the time of the traffic alone at the chip's measured copy rate: quantize 18.6 us (15.4), dequantize 16.5
// (15.4), norm with residual, h and codes 41.3 (35.9), with y too 51 (46.2), gradient 35.2 (30.8), with residual 45.3 (41.1), with
// residual and gain gradient 66 (41.1).
// An output may be one of the inputs where the call allows it (h one of x and the residual, dx one of dy and the residual): a thread writes
// only elements that it alone has read, and these pointers promise the compiler nothing (no __restrict__).
// FRAME: rows that do not start on 16-byte boundaries (odd widths in contiguous rows).  A row is then the whole 16-byte vectors in
// it, position q = column + shift, and the elements around them, which are taken one by one; the gain and the factors, which start
// at column 0, are read as words and shifted, and the codes turn back to column 0 through shared memory.
#include "common.cuh"
#include "host_common.h"
#include "kernels.h"
#include "launch.cuh"
#include "tc_common.cuh"

namespace sl {
namespace {

constexpr float TINY_ROW = 1e-36f;       // below this 127 / max overflows: the row is held as zero
constexpr int NV = 4;                    // accesses of 16 bytes per thread
constexpr int NV_CODES = 8, NV_SCALED = 4;       // of a thread that only quantises, without and with column factors
// Rows on 16-byte boundaries; at any place, but all arrays of activations at the same place of a 16-byte vector; at any place.
enum { FRAME_NONE = 0, FRAME_SAME = 1, FRAME_ANY = 2 };

using tc::add2; using tc::fma2; using tc::mul2; using tc::pack2; using tc::unpack2;

// The values of a 16-byte vector as pairs of floats: the arithmetic runs on the packed fp32 instructions, which halve its
// instructions (a norm is bound by instruction issue as much as by HBM: 35 instructions per element of one value at a time, 57 us for
// 8192 x 4096 bf16 with residual and both outputs).
template <typename T> struct Pairs { uint64_t v[Vec16<T>::N / 2]; };
__device__ __forceinline__ Pairs<bf16> pairs_of(const Vec16<bf16>& r) {
  const uint32_t w[4] = {r.raw.x, r.raw.y, r.raw.z, r.raw.w};
  Pairs<bf16> p;
#pragma unroll
  for (int i = 0; i < 4; ++i) p.v[i] = tc::bf16x2_to_f32x2(w[i]);
  return p;
}
__device__ __forceinline__ Pairs<float> pairs_of(const Vec16<float>& r) {
  Pairs<float> p;
  p.v[0] = pack2(r.raw.x, r.raw.y);
  p.v[1] = pack2(r.raw.z, r.raw.w);
  return p;
}
__device__ __forceinline__ Vec16<bf16> vector_of(const Pairs<bf16>& p) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    unpack2(p.v[i], a, b);
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  Vec16<bf16> r;
  r.raw = make_uint4(w[0], w[1], w[2], w[3]);
  return r;
}
__device__ __forceinline__ Vec16<float> vector_of(const Pairs<float>& p) {
  Vec16<float> r;
  unpack2(p.v[0], r.raw.x, r.raw.y);
  unpack2(p.v[1], r.raw.z, r.raw.w);
  return r;
}

// The larger of `top` and both magnitudes of a pair; a NaN stays.
__device__ __forceinline__ float max_abs(float top, uint64_t pair) {
  float a, b, r;
  unpack2(pair, a, b);
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(top), "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_abs(float top, float v) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(top), "f"(fabsf(v)));
  return r;
}

// rint(v * inv) for |v * inv| < 128 in the low byte of the result: the product is rounded to fp32 first, then adding 1.5 * 2^23
// leaves the nearest integer (ties to even) in the low bits of the sum.
constexpr float ROUNDER = 12582912.0f;
__device__ __forceinline__ uint32_t code_bits(float v, float inv) { return __float_as_uint(__fadd_rn(__fmul_rn(v, inv), ROUNDER)); }
// Four of them.  The sums are scalar: a packed product and a packed sum are contracted into one rounding, .rn or not.
__device__ __forceinline__ uint32_t code_word(uint64_t v01, uint64_t v23, uint64_t inv2, bool live) {
  float a, b, c, d;
  unpack2(mul2(v01, inv2), a, b);
  unpack2(mul2(v23, inv2), c, d);
  const uint32_t lo = __byte_perm(__float_as_uint(__fadd_rn(a, ROUNDER)), __float_as_uint(__fadd_rn(b, ROUNDER)), 0x0040);
  const uint32_t hi = __byte_perm(__float_as_uint(__fadd_rn(c, ROUNDER)), __float_as_uint(__fadd_rn(d, ROUNDER)), 0x0040);
  return live ? __byte_perm(lo, hi, 0x5410) : 0u;
}
// the W codes of a vector as W / 4 words
template <typename T> __device__ __forceinline__ void code_words(uint32_t* w, const Pairs<T>& v, float inv, bool live) {
  const uint64_t inv2 = pack2(inv, inv);
#pragma unroll
  for (int i = 0; i < Vec16<T>::N / 4; ++i) w[i] = code_word(v.v[2 * i], v.v[2 * i + 1], inv2, live);
}
template <int W> __device__ __forceinline__ void store_words(void* p, const uint32_t* w) {
  if constexpr (W == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(p) = w[0];
}

// The largest magnitude -> what a row's codes and scale need.  `unit` is what one unit of the maximum stands for (rstd for a norm,
// 1 for plain rows).
struct RowScale { float inv, scale; bool live; };
__device__ __forceinline__ RowScale row_scale(float a, float unit) {
  RowScale r;
  const bool finite = a < INFINITY;        // neither infinity nor NaN
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

// Sums and maximum over the threads of a row.  With whole warps per row every thread of the block takes part, in step; where a block walks
// several rows, two sets of shared memory in turn make one barrier per call enough.
struct RowShared { float sum[2][32]; uint32_t top[32]; };
template <int NS, bool MAX> __device__ __forceinline__ void reduce_row(float* s, float& largest, const Place& at, RowShared* sh) {
  uint32_t top = MAX ? __float_as_uint(largest) : 0u;    // no negative values: the order of the bits, NaN above all
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
  if constexpr (MAX) largest = __uint_as_float(top);
}

// A row of d elements at positions s .. s + d: whole vectors [v0, v1), and `edges` elements around them.  (The last vector before the
// row's end counts as edges: reading the gain of a whole vector may take in the element behind it.)
template <typename T, int FRAME> struct Span {
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
};

// What a thread reads of a row: its vectors, and its edge (FRAME: one at most).  AHEAD: one row ahead, the vectors through shared memory
// (slots of its own, so nothing but its own copies is waited for; stages: two rows, or one where there is no more room), the edge
// through a register.  Else straight from memory.  FRAME_ANY: arrays whose rows are not 16-byte aligned where the first array's
// are, element by element.
template <typename T, int FRAME, int ARRAYS, bool AHEAD, int EARLY = ARRAYS> struct Feed {
  const T* p[ARRAYS];
  bool fit[ARRAYS];
  T edge[ARRAYS], edge_next[ARRAYS];
  Vec16<T> raw[AHEAD ? 1 : EARLY][AHEAD ? 1 : NV];
  int stages, stage;
  uint8_t* slots;
  __device__ __forceinline__ Feed(int st, uint8_t* smem) : stages(st), stage(0), slots(smem + threadIdx.x * 16) {}
  __device__ __forceinline__ void array(int a, const T* q) {
    p[a] = q;
    fit[a] = FRAME != FRAME_ANY || ((reinterpret_cast<uintptr_t>(q) - reinterpret_cast<uintptr_t>(p[0])) & 15u) == 0;
  }
  __device__ __forceinline__ uint8_t* slot(int st, int a, int k) const { return slots + (size_t)((st * ARRAYS + a) * NV + k) * blockDim.x * 16; }
  __device__ __forceinline__ void fetch(int64_t row, int64_t M, int d, const Place& at, int st) {
    if (row < M) {
      const Span<T, FRAME> f(p[0] + row * d, d);
#pragma unroll
      for (int a = 0; a < ARRAYS; ++a) {
        const T* q = p[a] + row * d;
        if (!AHEAD && a < EARLY) {         // under way before the first use
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            const int v = f.v0 + k * at.n + at.t;
            if (v < f.v1) read(raw[AHEAD || a >= EARLY ? 0 : a][AHEAD ? 0 : k], a, q + f.column(v));
          }
        }
        if (FRAME && at.t < f.edges) edge_next[a] = q[f.edge(at.t)];
        if constexpr (AHEAD) {
          if (!fit[a]) continue;
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            const int v = f.v0 + k * at.n + at.t;
            if (v < f.v1)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(slot(st, a, k))), "l"(q + f.column(v)) : "memory");
          }
        }
      }
    }
    if (AHEAD) asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ __forceinline__ void read(Vec16<T>& r, int a, const T* q) const {
    if (fit[a]) r.load(q);
    else {
#pragma unroll
      for (int i = 0; i < Vec16<T>::N; ++i) reinterpret_cast<T*>(&r.raw)[i] = q[i];
    }
  }
  // before the first row, at the begin of a row (whose successor is `next`), at its end
  __device__ __forceinline__ void start(int64_t row, int64_t M, int d, const Place& at) { if (AHEAD) fetch(row, M, d, at, 0); }
  __device__ __forceinline__ void begin(int64_t row, int64_t next, int64_t M, int d, const Place& at) {
    if (!AHEAD) fetch(row, M, d, at, 0);
#pragma unroll
    for (int a = 0; a < ARRAYS; ++a) edge[a] = edge_next[a];
    if (!AHEAD) return;
    if (stages == 2) {
      fetch(next, M, d, at, stage ^ 1);
      asm volatile("cp.async.wait_group 1;" ::: "memory");
    } else {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
  }
  __device__ __forceinline__ void end(int64_t next, int64_t M, int d, const Place& at) {
    if (!AHEAD) return;
    if (stages == 2) stage ^= 1;
    else fetch(next, M, d, at, 0);
  }
  __device__ __forceinline__ void finish() const { if (AHEAD) asm volatile("cp.async.wait_group 0;" ::: "memory"); }
  // vector v = k-th of this thread, of array a, in the row at q = p[a] + row * d
  __device__ __forceinline__ void take(Vec16<T>& r, int a, int k, const T* q, int column) const {
    if constexpr (!AHEAD) r = raw[a][k];
    else if (fit[a]) r.raw = *reinterpret_cast<const decltype(r.raw)*>(slot(stage, a, k));
    else read(r, a, q + column);
  }
};
template <typename T, int FRAME> __device__ __forceinline__ void store_row(T* row, const Span<T, FRAME>& f, int v, bool fits, const Pairs<T>& x) {
  const Vec16<T> r = vector_of(x);
  T* p = row + f.column(v);
  if (FRAME != FRAME_ANY || fits) r.store(p);
  else {
#pragma unroll
    for (int i = 0; i < Vec16<T>::N; ++i) p[i] = reinterpret_cast<const T*>(&r.raw)[i];
  }
}
// The gain at the columns of vector v.  Shifted bf16 pairs: words from the even element at or before the first, joined by twos.
template <typename T, int FRAME> __device__ __forceinline__ void load_gain(Vec16<T>& r, const T* g, const Span<T, FRAME>& f, int v) {
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
// x times the column factors of vector v (factor may be null).  Shifted factors: whole float4s around them, by the shift.
template <typename T, int FRAME> __device__ __forceinline__ Pairs<T> scaled(const Vec16<T>& r, const float* factor, const Span<T, FRAME>& f, int v) {
  constexpr int W = Vec16<T>::N;
  Pairs<T> p = pairs_of(r);
  if (factor) {
    const float* q = factor + f.column(v);
    const int off = FRAME ? (int)((reinterpret_cast<uintptr_t>(q) >> 2) & 3u) : 0;
    auto times = [&](const float* w) {
#pragma unroll
      for (int i = 0; i < W / 2; ++i) p.v[i] = mul2(p.v[i], pack2(w[2 * i], w[2 * i + 1]));
    };
    float w[W + 4];
    if (off == 0) {
#pragma unroll
      for (int i = 0; i < W; i += 4) *reinterpret_cast<float4*>(w + i) = __ldg(reinterpret_cast<const float4*>(q + i));
      times(w);
    } else if (f.column(v) + W + 4 <= f.d && f.column(v) >= 4) {
#pragma unroll
      for (int i = 0; i <= W; i += 4) *reinterpret_cast<float4*>(w + i) = __ldg(reinterpret_cast<const float4*>(q - off + i));
      if (off == 1) times(w + 1);
      else if (off == 2) times(w + 2);
      else times(w + 3);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = __ldg(q + i);
      times(w);
    }
  }
  return p;
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
template <typename T> __host__ __device__ constexpr int code_bytes(int threads, int nv = NV) { return (threads * nv * Vec16<T>::N + 4 * Vec16<T>::N + 31) / 16 * 16; }
__device__ __forceinline__ uint8_t one_code(float v, const RowScale& rs) { return rs.live ? (uint8_t)code_bits(v, rs.inv) : (uint8_t)0; }

// The rows of a thread that adds up over rows (the gain's gradient): its group's, every (groups of the grid)-th.  `lead`: the row of the
// block's first group, by which all its threads go through the same number of rows.
struct Walk {
  int64_t row, lead, step;
  __device__ __forceinline__ explicit Walk(const Place& at) {
    const int per = blockDim.x / at.n;
    lead = (int64_t)blockIdx.x * per;
    row = lead + at.group;
    step = (int64_t)gridDim.x * per;
  }
};

// Past the first-level cache, which is left to the column factors.
template <typename T> __device__ __forceinline__ void load_past(Vec16<T>& r, const T* p) {
  uint32_t* w = reinterpret_cast<uint32_t*>(&r.raw);
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
}

// COL: with column factors, whose products stay in registers, for which a thread takes fewer accesses: 8192 x 4096 bf16 23.3 us, 4096 x
// 11008 38.9 (18.6 and 25 without factors, where four accesses took 24.7 and 35).  Factors read twice with eight accesses: 33 and 45; a
// thread's vector in two halves, so that the factors of neighbours lie side by side: 24.7 and 40.8.
template <typename T, int FRAME, bool COL>
__global__ void __launch_bounds__(1024)
quantize_kernel(const T* __restrict__ x, const float* __restrict__ factor, int64_t M, int d, int threads, int8_t* __restrict__ codes, int64_t ldc,
                int words, float* __restrict__ scales) {
  overlap_sync();
  constexpr int W = Vec16<T>::N, NV = COL ? NV_SCALED : NV_CODES;
  extern __shared__ __align__(16) uint8_t smem[];        // FRAME: codes
  __shared__ RowShared sh;
  const Place at(threads);
  const bool in = at.row < M;              // lanes of a row past the last still take part in the warp's exchanges
  const T* xr = x + (in ? at.row : 0) * d;
  const Span<T, FRAME> f(xr, d);
  const int v1 = in ? f.v1 : 0;
  Vec16<T> raw[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {           // everything the row needs is under way before the first use
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      if constexpr (COL) load_past(raw[k], xr + f.column(v));
      else raw[k].load(xr + f.column(v));
    }
  }
  const bool has_edge = FRAME && in && at.t < f.edges;
  const int ec = f.edge(at.t);
  float top = 0.f, ev = 0.f;
  if (has_edge) {
    ev = to_f<T>(xr[ec]);
    if (COL) ev = __fmul_rn(ev, factor[ec]);
    top = max_abs(top, ev);
  }
  Pairs<T> kept[COL ? NV : 1];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      Pairs<T>& o = kept[COL ? k : 0];
      if constexpr (COL) o = scaled<T, FRAME>(raw[k], factor, f, v);
      else o = pairs_of(raw[k]);
#pragma unroll
      for (int i = 0; i < W / 2; ++i) top = max_abs(top, o.v[i]);
    }
  }
  reduce_row<0, true>(nullptr, top, at, &sh);
  const RowScale rs = row_scale(top, 1.0f);
  if (at.t == 0 && in) scales[at.row] = rs.scale;
  int8_t* cr = codes + at.row * ldc;
  uint8_t* mine = FRAME ? smem + (size_t)at.group * code_bytes<T>(at.n, NV) : nullptr;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      uint32_t q[W / 4];
      if constexpr (COL) code_words<T>(q, kept[k], rs.inv, rs.live);
      else code_words<T>(q, pairs_of(raw[k]), rs.inv, rs.live);
      store_words<W>(FRAME ? (void*)(mine + v * W) : (void*)(cr + v * W), q);
    }
  }
  if constexpr (FRAME) {
    if (has_edge) mine[f.s + ec] = one_code(ev, rs);
    codes_out(mine, cr, f.s, in ? d : 0, at, words != 0);
  }
}

// Rows wider than the registers of 1024 threads (FRAME: 48 KB of codes) hold: read twice, the second time from L2.
template <typename T, int FRAME>
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
  float top = 0.f;
  for (int e = at.t; e < f.edges; e += 1024) top = max_abs(top, edge(f.edge(e)));
  for (int v = f.v0 + at.t; v < f.v1; v += 1024) {
    Vec16<T> r;
    r.load(xr + f.column(v));
    const Pairs<T> o = scaled<T, FRAME>(r, factor, f, v);
#pragma unroll
    for (int i = 0; i < W / 2; ++i) top = max_abs(top, o.v[i]);
  }
  reduce_row<0, true>(nullptr, top, at, &sh);
  const RowScale rs = row_scale(top, 1.0f);
  if (at.t == 0) scales[at.row] = rs.scale;
  for (int e = at.t; e < f.edges; e += 1024) cr[f.edge(e)] = (int8_t)one_code(edge(f.edge(e)), rs);
  for (int v = f.v0 + at.t; v < f.v1; v += 1024) {
    Vec16<T> r;
    uint32_t w[W / 4];
    r.load(xr + f.column(v));
    code_words<T>(w, scaled<T, FRAME>(r, factor, f, v), rs.inv, rs.live);
    if constexpr (!FRAME) store_words<W>(cr + v * W, w);
    else {
#pragma unroll
      for (int i = 0; i < W; ++i) cr[f.column(v) + i] = (int8_t)((w[i / 4] >> (8 * (i & 3))) & 0xffu);
    }
  }
}

template <typename T, int FRAME>
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
      Pairs<T> o;
#pragma unroll
      for (int i = 0; i < W; i += 2)
        o.v[i / 2] = mul2(pack2((float)(int8_t)(w[k][i / 4] >> (8 * (i & 3))), (float)(int8_t)(w[k][i / 4] >> (8 * (i & 3) + 8))), pack2(s, s));
      store_row<T, FRAME>(yr, f, v, true, o);
    }
  }
}

template <typename T, int FRAME, bool RES>
__global__ void __launch_bounds__(1024)
rmsnorm_quantize_kernel(const T* x, const T* resid, const T* __restrict__ g, int64_t M, int d, int threads, float eps,
                        T* h, T* __restrict__ y, int8_t* __restrict__ codes, int64_t ldc, int words, float* __restrict__ scales) {
  overlap_sync();
  constexpr int W = Vec16<T>::N;
  extern __shared__ __align__(16) uint8_t smem[];        // FRAME: codes
  __shared__ RowShared sh;
  const Place at(threads);
  Feed<T, FRAME, RES ? 2 : 1, false> feed(0, smem);
  feed.array(0, x);
  if constexpr (RES) feed.array(1, resid);
  uint8_t* mine = smem + (size_t)at.group * code_bytes<T>(at.n);
  const bool fit_h = ((reinterpret_cast<uintptr_t>(h) - reinterpret_cast<uintptr_t>(x)) & 15u) == 0;
  const bool fit_y = ((reinterpret_cast<uintptr_t>(y) - reinterpret_cast<uintptr_t>(x)) & 15u) == 0;
  const bool in = at.row < M;              // lanes of a row past the last still take part in the warp's exchanges
  const int64_t row0 = (in ? at.row : 0) * d;
  const Span<T, FRAME> f(x + row0, d);
  const int v1 = in ? f.v1 : 0, ec = f.edge(at.t);
  const bool has_edge = FRAME && in && at.t < f.edges;
  feed.begin(at.row, M, M, d, at);
  uint64_t sum2 = 0ull;
  float es = 0.f, ev = 0.f, top = 0.f;
  // x + residual, from the vectors as they came: formed twice, which costs less than the registers that would keep it
  auto sum_of = [&](int k) {
    Pairs<T> s = pairs_of(feed.raw[0][k]);
    if constexpr (RES) {
      const Pairs<T> rp = pairs_of(feed.raw[1][k]);
#pragma unroll
      for (int i = 0; i < W / 2; ++i) s.v[i] = add2(s.v[i], rp.v[i]);
    }
    return s;
  };
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      Vec16<T> gv;
      load_gain<T, FRAME>(gv, g, f, v);
      const Pairs<T> s = sum_of(k), gain = pairs_of(gv);
#pragma unroll
      for (int i = 0; i < W / 2; ++i) {
        sum2 = fma2(s.v[i], s.v[i], sum2);
        top = max_abs(top, mul2(s.v[i], gain.v[i]));
      }
      if (h) store_row<T, FRAME>(h + row0, f, v, fit_h, s);
    }
  }
  float sum;
  {
    float a, b;
    unpack2(sum2, a, b);
    sum = a + b;
  }
  if (has_edge) {
    es = to_f<T>(feed.edge[0]);
    if constexpr (RES) es = __fadd_rn(es, to_f<T>(feed.edge[1]));
    ev = __fmul_rn(es, to_f<T>(g[ec]));
    sum = fmaf(es, es, sum);
    top = max_abs(top, ev);
    if (h) h[row0 + ec] = from_f<T>(es);
  }
  reduce_row<1, true>(&sum, top, at, &sh);
  const float rstd = rsqrtf(sum / d + eps);
  const RowScale rs = row_scale(top, rstd);
  if (at.t == 0 && in) scales[at.row] = rs.scale;
  int8_t* cr = codes + at.row * ldc;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = f.v0 + k * at.n + at.t;
    if (v < v1) {
      Vec16<T> gv;
      load_gain<T, FRAME>(gv, g, f, v);
      Pairs<T> o = sum_of(k);
      const Pairs<T> gain = pairs_of(gv);
#pragma unroll
      for (int i = 0; i < W / 2; ++i) o.v[i] = mul2(o.v[i], gain.v[i]);
      uint32_t q[W / 4];
      code_words<T>(q, o, rs.inv, rs.live);
      store_words<W>(FRAME ? (void*)(mine + v * W) : (void*)(cr + v * W), q);
      if (y) {
        const uint64_t rstd2 = pack2(rstd, rstd);
#pragma unroll
        for (int i = 0; i < W / 2; ++i) o.v[i] = mul2(o.v[i], rstd2);
        store_row<T, FRAME>(y + row0, f, v, fit_y, o);
      }
    }
  }
  if constexpr (FRAME) {
    if (has_edge) {
      mine[f.s + ec] = one_code(ev, rs);
      if (y) y[row0 + ec] = from_f<T>(ev * rstd);
    }
    codes_out(mine, cr, f.s, in ? d : 0, at, words != 0);
  }
}

// The gradient.  Contractions are spelled out: dx does not depend on whether dg is asked for.
// DG: the gain's gradient too.  A group keeps its columns' sums in registers; the groups of a block add theirs up in order, and each
// block leaves one row of partial sums [gridDim.x, d] that dg_reduce_kernel adds up in order: the result does not depend on
// scheduling.  The number of groups is then a multiple of 8 (or each has one row), so a group's rows all have the same shift and
// its threads the same columns.
template <typename T, int FRAME, bool DG, bool RES, int MAXT>
__global__ void __launch_bounds__(MAXT)
rmsnorm_bwd_kernel(const T* dy, const T* __restrict__ h, const T* __restrict__ g, const T* resid, int64_t M, int d, int threads, int stages, float eps,
                   T* dx, float* __restrict__ partial) {
  overlap_sync();
  constexpr int W = Vec16<T>::N;
  extern __shared__ __align__(16) uint8_t smem[];        // the feed's slots; in the end (DG) sums
  __shared__ RowShared sh[2];
  const Place at(threads);
  Feed<T, FRAME, RES ? 3 : 2, DG, 2> feed(stages, smem);
  feed.array(0, h);
  feed.array(1, dy);
  if constexpr (RES) feed.array(2, resid);
  const bool fit_dx = ((reinterpret_cast<uintptr_t>(dx) - reinterpret_cast<uintptr_t>(h)) & 15u) == 0;
  Pairs<T> acc[DG ? NV : 1];
  float acc_edge = 0.f;
  if constexpr (DG) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < W / 2; ++i) acc[k].v[i] = 0ull;
  }
  Walk w(at);
  const Span<T, FRAME> own(h + w.row * d, d);            // of all rows of this group (DG)
  feed.start(w.row, M, d, at);
  for (int flip = 0; w.lead < M; w.row += w.step, w.lead += w.step, flip ^= 1) {
    const bool in = w.row < M;
    const int64_t row0 = (in ? w.row : 0) * d;
    const Span<T, FRAME> f(h + row0, d);
    const int v1 = in ? f.v1 : 0, ec = f.edge(at.t);
    const bool has_edge = FRAME && in && at.t < f.edges;
    feed.begin(w.row, w.row + w.step, M, d, at);
    Vec16<T> kept[2][DG ? NV : 1];          // AHEAD: out of the slots, once
    auto vec = [&](int a, int k) -> const Vec16<T>& { if constexpr (DG) return kept[a][k]; else return feed.raw[a][k]; };
    uint64_t hh2 = 0ull, wh2 = 0ull;
    float eh = 0.f, ed = 0.f, eg = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = f.v0 + k * at.n + at.t;
      if (v < v1) {
        Vec16<T> gv;
        if constexpr (DG) {
          feed.take(kept[0][k], 0, k, h + row0, f.column(v));
          feed.take(kept[1][k], 1, k, dy + row0, f.column(v));
        }
        load_gain<T, FRAME>(gv, g, f, v);
        const Pairs<T> hp = pairs_of(vec(0, k)), dp = pairs_of(vec(1, k)), gp = pairs_of(gv);
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
          hh2 = fma2(hp.v[i], hp.v[i], hh2);
          wh2 = fma2(mul2(dp.v[i], gp.v[i]), hp.v[i], wh2);
        }
      }
    }
    float s[2];
    {
      float a, b;
      unpack2(hh2, a, b); s[0] = a + b;
      unpack2(wh2, a, b); s[1] = a + b;
    }
    if (has_edge) {
      eh = to_f<T>(feed.edge[0]); ed = to_f<T>(feed.edge[1]); eg = to_f<T>(g[ec]);
      s[0] = fmaf(eh, eh, s[0]);
      s[1] = fmaf(__fmul_rn(ed, eg), eh, s[1]);
    }
    // the residual's vectors: under way during the reduction, where registers are free for them (not with edges or sums to keep)
    constexpr bool SOON = RES && !DG && FRAME == FRAME_NONE;
    Vec16<T> rv[SOON ? NV : 1];
    if constexpr (SOON) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int v = f.v0 + k * at.n + at.t;
        if (v < v1) rv[k].load(resid + row0 + f.column(v));
      }
    }
    float none = 0.f;
    reduce_row<2, false>(s, none, at, &sh[flip]);
    const float rstd = rsqrtf(s[0] / d + eps);
    const float c = rstd * rstd * (s[1] / d);
    const uint64_t rstd2 = pack2(rstd, rstd), c2 = pack2(-c, -c);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = f.v0 + k * at.n + at.t;
      if (v < v1) {
        Vec16<T> gv;
        load_gain<T, FRAME>(gv, g, f, v);
        const Pairs<T> hp = pairs_of(vec(0, k)), dp = pairs_of(vec(1, k)), gp = pairs_of(gv);
        Pairs<T> o;
#pragma unroll
        for (int i = 0; i < W / 2; ++i) o.v[i] = fma2(hp.v[i], c2, mul2(dp.v[i], gp.v[i]));
        if constexpr (RES) {
          if constexpr (DG) feed.take(rv[0], 2, k, resid + row0, f.column(v));
          else if constexpr (!SOON) feed.read(rv[0], 2, resid + row0 + f.column(v));
          const Pairs<T> rp = pairs_of(rv[SOON ? k : 0]);
#pragma unroll
          for (int i = 0; i < W / 2; ++i) o.v[i] = fma2(rstd2, o.v[i], rp.v[i]);
        } else {
#pragma unroll
          for (int i = 0; i < W / 2; ++i) o.v[i] = mul2(rstd2, o.v[i]);
        }
        if constexpr (DG) {
#pragma unroll
          for (int i = 0; i < W / 2; ++i) acc[k].v[i] = fma2(dp.v[i], mul2(hp.v[i], rstd2), acc[k].v[i]);
        }
        store_row<T, FRAME>(dx + row0, f, v, fit_dx, o);
      }
    }
    if (has_edge) {
      const float t = fmaf(-eh, c, __fmul_rn(ed, eg));
      if constexpr (RES) dx[row0 + ec] = from_f<T>(fmaf(rstd, t, to_f<T>(feed.edge[2])));
      else dx[row0 + ec] = from_f<T>(__fmul_rn(rstd, t));
      if constexpr (DG) acc_edge = fmaf(ed, __fmul_rn(eh, rstd), acc_edge);
    }
    if constexpr (!DG) break;              // a group per row
    feed.end(w.row + w.step, M, d, at);
  }
  feed.finish();
  if constexpr (DG) {
    __syncthreads();
    float* sums = reinterpret_cast<float*>(smem);
    for (int c = threadIdx.x; c < d; c += blockDim.x) sums[c] = 0.f;
    __syncthreads();
    // several rows per warp with the same columns per lane: added up in the warp first, which then takes one turn
    const int lane = threadIdx.x & 31, mates = FRAME == FRAME_NONE && at.n < 32 ? 32 / at.n : 1;
    for (int o = at.n; o < at.n * mates; o <<= 1) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < W / 2; ++i) acc[k].v[i] = add2(acc[k].v[i], __shfl_xor_sync(0xffffffffu, acc[k].v[i], o));
    }
    for (int turn = 0; turn < (int)blockDim.x / (threads * mates); ++turn) {
      if (at.group / mates == turn && (mates == 1 || lane < at.n)) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int v = own.v0 + k * at.n + at.t;
          if (v < own.v1) {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
              float a, b;
              unpack2(acc[k].v[i], a, b);
              sums[own.column(v) + 2 * i] += a;
              sums[own.column(v) + 2 * i + 1] += b;
            }
          }
        }
        if (FRAME && at.t < own.edges) sums[own.edge(at.t)] += acc_edge;
      }
      __syncthreads();
    }
    float* out = partial + (int64_t)blockIdx.x * d;
    for (int c = threadIdx.x; c < d; c += blockDim.x) out[c] = sums[c];
  }
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

// Threads per row: as many as give each `nv_each` accesses, a power of two up to a warp, else whole warps.  frame: an edge per thread.
template <typename T> int row_threads(int d, bool frame, int nv_each = NV) {
  const int nv = (d + Vec16<T>::N - 1) / Vec16<T>::N, need = (nv + nv_each - 1) / nv_each;
  if (need > 32) return (need + 31) / 32 * 32;
  int n = frame ? 2 * Vec16<T>::N : 1;
  while (n < need) n *= 2;
  return n;
}

// Blocks of 256 threads where a row takes a warp or less, else a block per row.
struct Shape { int block, per; int64_t blocks; };
Shape shape_of(int64_t M, int threads) {
  Shape s;
  s.block = threads <= 32 ? 256 : threads;
  s.per = s.block / threads;
  s.blocks = (M + s.per - 1) / s.per;
  return s;
}

template <typename T, int FRAME, bool COL>
cudaError_t quantize_t(const T* x, const float* factor, int64_t M, int d, int8_t* codes, int64_t ldc, float* scales, cudaStream_t st) {
  constexpr int nv = COL ? NV_SCALED : NV_CODES;
  const int threads = row_threads<T>(d, FRAME != 0, nv);
  if (threads > 1024 || (FRAME && code_bytes<T>(threads, nv) > 48 * 1024))         // wider than registers, or shared memory, take
    return launch_overlapped(quantize_wide_kernel<T, FRAME>, dim3((unsigned)M), dim3(1024), 0, st, x, factor, d, codes, ldc, scales);
  const Shape s = shape_of(M, threads);
  const int words = ldc % 4 == 0 && al(codes, 4);
  return launch_overlapped(quantize_kernel<T, FRAME, COL>, dim3((unsigned)s.blocks), dim3(s.block), FRAME ? (size_t)s.per * code_bytes<T>(threads, nv) : 0, st,
                           x, factor, M, d, threads, codes, ldc, words, scales);
}
template <typename T, int FRAME>
cudaError_t norm_t(const T* x, const T* resid, const T* g, int64_t M, int d, float eps, T* h, T* y, int8_t* codes, int64_t ldc, float* scales, cudaStream_t st) {
  const int threads = row_threads<T>(d, FRAME != 0);
  const Shape s = shape_of(M, threads);
  const int words = ldc % 4 == 0 && al(codes, 4);
  return launch_overlapped(resid ? rmsnorm_quantize_kernel<T, FRAME, true> : rmsnorm_quantize_kernel<T, FRAME, false>, dim3((unsigned)s.blocks), dim3(s.block),
                           FRAME ? (size_t)s.per * code_bytes<T>(threads) : 0, st, x, resid, g, M, d, threads, eps, h, y, codes, ldc, words, scales);
}
template <typename T, int FRAME>
cudaError_t norm_bwd_t(const T* dy, const T* h, const T* g, const T* resid, int64_t M, int d, int threads, float eps, T* dx, cudaStream_t st) {
  const Shape s = shape_of(M, threads);
  return launch_overlapped(resid ? rmsnorm_bwd_kernel<T, FRAME, false, true, 1024> : rmsnorm_bwd_kernel<T, FRAME, false, false, 1024>, dim3((unsigned)s.blocks),
                           dim3(s.block), 0, st, dy, h, g, resid, M, d, threads, 0, eps, dx, (float*)nullptr);
}
// With dg: as many rows per block as 512 threads take, a block per SM (128 registers per thread, up to 192 KB of copies ahead).
template <typename T, int FRAME, int MAXT>
cudaError_t norm_gain_t(const T* dy, const T* h, const T* g, const T* resid, int64_t M, int d, int threads, float eps, T* dx, float* partial, int* rows,
                        cudaStream_t st) {
  constexpr size_t MOST = 230000;
  const auto kernel = resid ? rmsnorm_bwd_kernel<T, FRAME, true, true, MAXT> : rmsnorm_bwd_kernel<T, FRAME, true, false, MAXT>;
  static PerDeviceOnce once[2];
  const int dev = current_device();
  if (once[resid ? 1 : 0].needed(dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MOST);
    if (e != cudaSuccess) return e;
    once[resid ? 1 : 0].done(dev);
  }
  const int per = threads > 512 ? 1 : 512 / threads, block = per * threads;
  const size_t one = (size_t)(resid ? 3 : 2) * NV * block * 16;
  const int stages = 2 * one <= MOST ? 2 : 1;
  const size_t smem = stages * one < (size_t)d * 4 ? (size_t)d * 4 : stages * one;
  const int64_t all = (M + per - 1) / per;
  int64_t blocks = num_sms() < DG_PARTIAL_ROWS ? num_sms() : DG_PARTIAL_ROWS;
  if (blocks >= all) blocks = all;
  else blocks = blocks >= 8 ? blocks / 8 * 8 : 8;
  *rows = (int)blocks;
  return launch_overlapped(kernel, dim3((unsigned)blocks), dim3(block), smem, st, dy, h, g, resid, M, d, threads, stages, eps, dx, partial);
}
// Arrays at the same place of a 16-byte vector as the first one.
bool same_place(const void* p, const void* first) { return !p || ((reinterpret_cast<uintptr_t>(p) - reinterpret_cast<uintptr_t>(first)) & 15u) == 0; }

}  // namespace

cudaError_t quantize_rows(int dt, const void* x, const float* factor, int64_t M, int d, int8_t* codes, int64_t ldc, float* scales, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int W = Vec16<T>::N;
    const bool frame = d % W != 0 || ldc % W != 0 || !al(x, 16) || !al(factor, 16) || !al(codes, W);
    auto go = [&](auto launch) { return launch((const T*)x, factor, M, d, codes, ldc, scales, st); };
    if (factor) return frame ? go(quantize_t<T, FRAME_SAME, true>) : go(quantize_t<T, FRAME_NONE, true>);
    return frame ? go(quantize_t<T, FRAME_SAME, false>) : go(quantize_t<T, FRAME_NONE, false>);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

cudaError_t dequantize_rows(int dt, const int8_t* codes, int64_t ldc, const float* scales, int64_t M, int d, void* y, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int W = Vec16<T>::N;
    const bool frame = d % W != 0 || ldc % W != 0 || !al(y, 16) || !al(codes, W);
    int threads = row_threads<T>(d, frame);
    if (threads > 1024) threads = 1024;
    const int block = threads <= 32 ? 256 : threads, per = block / threads;
    return launch_overlapped(frame ? dequantize_kernel<T, FRAME_SAME> : dequantize_kernel<T, FRAME_NONE>, dim3((unsigned)((M + per - 1) / per)), dim3(block), 0, st,
                             codes, ldc, scales, M, d, threads, (T*)y);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

cudaError_t rmsnorm_quantize(int dt, const void* x, const void* resid, const void* g, int64_t M, int d, float eps, void* h, void* y, int8_t* codes,
                             int64_t ldc, float* scales, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int W = Vec16<T>::N;
    const bool frame = d % W != 0 || ldc % W != 0 || !al(x, 16) || !al(g, 16) || !al(resid, 16) || !al(h, 16) || !al(y, 16) || !al(codes, W);
    auto go = [&](auto launch) { return launch((const T*)x, (const T*)resid, (const T*)g, M, d, eps, (T*)h, (T*)y, codes, ldc, scales, st); };
    if (!frame) return go(norm_t<T, FRAME_NONE>);
    return same_place(resid, x) && same_place(h, x) && same_place(y, x) ? go(norm_t<T, FRAME_SAME>) : go(norm_t<T, FRAME_ANY>);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

size_t rmsnorm_dg_scratch_floats(int64_t M, int d) { return (size_t)(M < DG_PARTIAL_ROWS ? M : DG_PARTIAL_ROWS) * d; }

cudaError_t rmsnorm_gain_bwd(int dt, const void* dy, const void* h, const void* g, const void* resid, int64_t M, int d, float eps, void* dx, float* dg,
                             float* partial, cudaStream_t st) {
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    const bool frame = d % Vec16<T>::N != 0 || !al(dy, 16) || !al(h, 16) || !al(g, 16) || !al(resid, 16) || !al(dx, 16);
    const int threads = row_threads<T>(d, frame);
    const bool same = same_place(dy, h) && same_place(resid, h) && same_place(dx, h);
    if (!dg) {
      auto go = [&](auto launch) { return launch((const T*)dy, (const T*)h, (const T*)g, (const T*)resid, M, d, threads, eps, (T*)dx, st); };
      if (!frame) return go(norm_bwd_t<T, FRAME_NONE>);
      return same ? go(norm_bwd_t<T, FRAME_SAME>) : go(norm_bwd_t<T, FRAME_ANY>);
    }
    int rows = 0;
    auto go = [&](auto launch) { return launch((const T*)dy, (const T*)h, (const T*)g, (const T*)resid, M, d, threads, eps, (T*)dx, partial, &rows, st); };
    cudaError_t e = cudaSuccess;
    if (threads <= 512) e = !frame ? go(norm_gain_t<T, FRAME_NONE, 512>) : same ? go(norm_gain_t<T, FRAME_SAME, 512>) : go(norm_gain_t<T, FRAME_ANY, 512>);
    else if constexpr (sizeof(T) == 4)
      e = !frame ? go(norm_gain_t<T, FRAME_NONE, 1024>) : same ? go(norm_gain_t<T, FRAME_SAME, 1024>) : go(norm_gain_t<T, FRAME_ANY, 1024>);
    if (e != cudaSuccess) return e;
    return launch_overlapped(dg_reduce_kernel, dim3((unsigned)((d + 31) / 32)), dim3(256), 0, st, (const float*)partial, rows, d, dg);
  };
  return dt == DT_BF16 ? run(bf16()) : run(float());
}

}  // namespace sl
