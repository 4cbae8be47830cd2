// Loss over the vocabulary against a teacher's top logits and the labels, with its gradient.  Per row m with logits z (V of
// them), temperature T, the teacher's k entries (idx_j, t_j) and the label y:
//   q = softmax_j(t_j / T) over the row's entries,  p1 = softmax(z),  pT = softmax(z / T)
//   row  = wc (-log p1[y])  +  wk T^2 sum_j q_j (log q_j - log pT[idx_j])
//   dz_v = ( wc (p1_v - [v = y])  +  wk T (pT_v - sum_{j: idx_j = v} q_j) ) / n
// Both softmaxes share the row's maximum.  Between their one read and one write narrow rows are held in a warp's registers
// (distill_warp_kernel), rows of up to 114 thousand bf16 or 57 thousand fp32 logits in shared memory (distill_ring_kernel); wider
// ones are read twice (distill_kernel).  In all of them the at most k + 1 entries that carry a target are written again from their saved logits, with all of a repeated index's weights summed by the first
// of its entries in order: one rounding per output, no atomics.  Exponents are formed as (z - max) * log2(e) / T: for the entries
// that matter z - max is small, so the fp32 rounding of the product stays near 2^-24 of the probability.
// 4096 x 50257 bf16, k = 32, both terms: 173 us at T = 2, 177 at T = 4, 226 at T = 1.3; the traffic alone takes 126.
// The gradient may be written over the logits: every element is read before it is written, and written by the thread that read it or
// behind a barrier.
#include <type_traits>

#include "common.cuh"
#include "host_common.h"
#include "kernels.h"
#include "launch.cuh"
#include "tc_common.cuh"

namespace sl {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// How the two exponentials of a logit come about.
enum { EXP_ONE = 0,       // one temperature is enough (T = 1, or one of the two terms has no weight): the second is not used
       EXP_TWO = 1 };     // both

struct DistillArgs {
  const int32_t* labels; const int32_t* idx; const float* t;
  int64_t ld, ldo;
  int V, k;
  float temp, wc, wk;
  float c1, cT;            // log2(e) / temperature of the first and second exponential
  float inv_t;
  float* rows; int* n_valid; int n_fixed;
  int same;                // rows of logits and gradient start at the same place of a 16-byte vector
  int count_here;          // the kernel that holds the rows counts the labels and leaves the count in n_valid
};

// Running maximum and sums of exponentials relative to it.
struct Online { float m, s1, sT; };
template <int MODE> __device__ __forceinline__ void online_merge(Online& a, const Online& b, float c1, float cT) {
  const float m = fmaxf(a.m, b.m);
  const float base = m == -INFINITY ? 0.f : m;           // nothing but -inf so far: every factor is ex2(-inf) = 0
  const float da = a.m - base, db = b.m - base;
  a.s1 = a.s1 * ex2(da * c1) + b.s1 * ex2(db * c1);
  if constexpr (MODE == EXP_TWO) a.sT = a.sT * ex2(da * cT) + b.sT * ex2(db * cT);
  a.m = m;
}

// Rows wider than shared memory, one block each: a pass for the maximum and the running sums of exponentials, a pass that writes the
// gradient from the logits' second read (L1 or L2).  4 exponentials per logit with two temperatures: bound by the exponential unit and
// instruction issue as much as by traffic: 1024 x 128256 bf16 at T 2 182 us, where the traffic takes 80 (4096 x 50257 took 467 us with it,
// where the ring kernel takes 173).
template <typename T, int W, int MODE>
__global__ void __launch_bounds__(512)
distill_kernel(const T* logits, T* grad, DistillArgs p) {
  overlap_sync();
  __shared__ Online sh_on[16];
  __shared__ float sh_red[16];
  __shared__ int sh_idx[DISTILL_MAX_K];
  __shared__ float sh_q[DISTILL_MAX_K], sh_z[DISTILL_MAX_K];
  __shared__ float sh_zy;
  const int64_t row = blockIdx.x;
  const T* z = logits + row * p.ld;
  T* out = grad + row * p.ldo;
  const int V = p.V, k = p.k, tid = threadIdx.x, nt = blockDim.x, warp = tid >> 5, lane = tid & 31, nw = nt >> 5;
  const int y = p.labels ? p.labels[row] : -1;
  const bool valid = p.labels == nullptr || (y >= 0 && y < V);
  const int n = p.n_valid ? *p.n_valid : p.n_fixed;
  const int nacc = V / W;
  if (!valid) {                            // the row takes no part: zeros
    if (tid == 0) p.rows[row] = 0.f;
    const int all = (int)(p.ldo / W);
    T none[W];
#pragma unroll
    for (int i = 0; i < W; ++i) none[i] = from_f<T>(0.f);
    for (int a = tid; a < all; a += nt) {
      if constexpr (W > 1) *reinterpret_cast<uint4*>(out + (int64_t)a * W) = make_uint4(0u, 0u, 0u, 0u);
      else out[a] = none[0];
    }
    for (int c = all * W + tid; c < p.ldo; c += nt) out[c] = none[0];
    return;
  }

  // ---- the teacher's distribution and the logits of its entries
  const float inv_t = 1.0f / p.temp;
  float tmax = -INFINITY;
  for (int j = tid; j < k; j += nt) {
    const int v = p.idx[row * k + j];
    const bool ok = v >= 0 && v < V;
    const float t = ok ? p.t[row * k + j] : -INFINITY;
    sh_idx[j] = ok ? v : -1;
    sh_q[j] = t;
    sh_z[j] = ok ? to_f<T>(z[v]) : 0.f;
    tmax = t != t ? t : fmaxf(tmax, t);
  }
  if (tid == 0 && p.labels) sh_zy = to_f<T>(z[y]);

  // ---- maximum and sums of the student's row
  Online on{-INFINITY, 0.f, 0.f};
  auto take = [&](const float* v, int count) {
    float m = on.m;
#pragma unroll
    for (int i = 0; i < W; ++i) if (i < count) m = fmaxf(m, v[i]);
    const float base = m == -INFINITY ? 0.f : m;
    float a1 = 0.f, aT = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < count) {
        const float dd = v[i] - base;
        a1 += ex2(dd * p.c1);
        if constexpr (MODE == EXP_TWO) aT += ex2(dd * p.cT);
      }
    const float dm = on.m - base;
    on.s1 = on.s1 * ex2(dm * p.c1) + a1;
    if constexpr (MODE == EXP_TWO) on.sT = on.sT * ex2(dm * p.cT) + aT;
    on.m = m;
  };
  for (int a = tid; a < nacc; a += nt) {
    float v[W];
    if constexpr (W > 1) {
      Vec16<T> r; r.load(z + (int64_t)a * W);
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] = r.get(i);
    } else {
      v[0] = to_f<T>(z[a]);
    }
    take(v, W);
  }
  if (W > 1 && tid < V - nacc * W) {
    float v[W];
    v[0] = to_f<T>(z[nacc * W + tid]);
    take(v, 1);
  }
  // a NaN among the logits is in the sums; one that every maximum has passed over stays there
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Online b;
    b.m = __shfl_xor_sync(0xffffffffu, on.m, o); b.s1 = __shfl_xor_sync(0xffffffffu, on.s1, o); b.sT = __shfl_xor_sync(0xffffffffu, on.sT, o);
    const float other = __shfl_xor_sync(0xffffffffu, tmax, o);
    online_merge<MODE>(on, b, p.c1, p.cT);
    tmax = tmax != tmax ? tmax : other != other ? other : fmaxf(tmax, other);
  }
  if (lane == 0) { sh_on[warp] = on; sh_red[warp] = tmax; }
  __syncthreads();
  on = sh_on[0];
  tmax = sh_red[0];
  for (int w = 1; w < nw; ++w) {           // every thread in the same order
    online_merge<MODE>(on, sh_on[w], p.c1, p.cT);
    const float other = sh_red[w];
    tmax = tmax != tmax ? tmax : other != other ? other : fmaxf(tmax, other);
  }
  __syncthreads();
  const bool some = tmax != -INFINITY && p.wk != 0.f;      // else the teacher says nothing about this row
  // teacher: sum of exponentials, then q and the row's divergence
  float tsum = 0.f;
  for (int j = tid; j < k; j += nt) tsum += some ? expf((sh_q[j] - tmax) * inv_t) : 0.f;
  tsum = warp_sum(tsum);
  if (lane == 0) sh_red[warp] = tsum;
  __syncthreads();
  tsum = 0.f;
  for (int w = 0; w < nw; ++w) tsum += sh_red[w];
  __syncthreads();
  const float base = on.m == -INFINITY ? 0.f : on.m;
  const float sT = MODE == EXP_TWO ? on.sT : on.s1;
  const float log_s1 = logf(on.s1), log_sT = logf(sT), log_ts = logf(tsum);
  float kl = 0.f;
  for (int j = tid; j < k; j += nt) {
    const float lq = (sh_q[j] - tmax) * inv_t - log_ts;
    const float q = some ? expf(lq) : 0.f;
    if (q != 0.f) kl += q * fmaf(p.temp, lq + log_sT, base - sh_z[j]);      // T times the divergence: (z - base) / T could overflow
    sh_q[j] = q;
  }
  kl = warp_sum(kl);
  if (lane == 0) sh_red[warp] = kl;
  __syncthreads();
  kl = 0.f;
  for (int w = 0; w < nw; ++w) kl += sh_red[w];
  const float wk = some ? p.wk : 0.f;
  if (tid == 0) {
    float r = wk != 0.f ? wk * p.temp * kl : 0.f;
    if (p.wc != 0.f) r += p.wc * (log_s1 - (sh_zy - base));
    p.rows[row] = r;
  }

  // ---- gradient
  const float inv_n = 1.0f / (float)(n > 0 ? n : 1);
  // EXP_ONE: one exponential carries both terms
  const float f1 = MODE == EXP_TWO ? p.wc / on.s1 * inv_n : (p.wc + wk * p.temp) / on.s1 * inv_n;
  const float fT = MODE == EXP_TWO ? wk * p.temp / sT * inv_n : 0.f;
  auto value = [&](float v) {
    const float dd = v - base;
    float r = f1 * ex2(dd * p.c1);
    if constexpr (MODE == EXP_TWO) r += fT * ex2(dd * p.cT);
    return r;
  };
  for (int a = tid; a < nacc; a += nt) {
    if constexpr (W > 1) {
      Vec16<T> r, o; r.load(z + (int64_t)a * W);
#pragma unroll
      for (int i = 0; i < W; ++i) o.set(i, value(r.get(i)));
      o.store(out + (int64_t)a * W);
    } else {
      out[a] = from_f<T>(value(to_f<T>(z[a])));
    }
  }
  for (int64_t c = (int64_t)nacc * W + tid; c < p.ldo; c += nt) out[c] = from_f<T>(c < V ? value(to_f<T>(z[c])) : 0.f);
  __syncthreads();
  // the entries with a target: the first entry of an index writes for all of them
  for (int j = tid; j < k; j += nt) {
    const int v = sh_idx[j];
    if (v < 0) continue;
    bool first = true;
    float q = 0.f;
    for (int i = 0; i < k; ++i) {
      if (sh_idx[i] != v) continue;
      if (i < j) first = false;
      q += sh_q[i];
    }
    if (!first) continue;
    float r = value(sh_z[j]) - (wk * p.temp * inv_n) * q;
    if (v == y) r -= p.wc * inv_n;
    out[v] = from_f<T>(r);
  }
  if (tid == 0 && p.labels) {
    bool taken = false;
    for (int i = 0; i < k; ++i) taken |= sh_idx[i] == y;
    if (!taken) out[y] = from_f<T>(value(sh_zy) - p.wc * inv_n);
  }
}

// ------------------------------------------------------------------------------------------
// rows in shared memory
// ------------------------------------------------------------------------------------------
// Persistent blocks walk the rows.  One thread copies the next rows into a ring of one or two buffers with bulk copies; a row's
// logits are read from there three times (maximum, sums, gradient; keeping the exponentials in registers between the last two took 280 us
// where this takes 174: fewer rows per SM), and the gradient leaves from there: a logit costs HBM one read and one write, and
// two exponentials where one temperature is enough or the two are 1 and 2, 3 or 4 (then e^z = (e^(z/2))^2 and so on), else four.
// Bounded by shared memory's reads, issue and HBM alike; fp32, twice the bytes for the same exponentials, by HBM.
// Rows may start anywhere (a vocabulary of 50257 entries in contiguous rows): a row is held as the 16-byte vectors that cover it, its
// first and last vector patched by the threads that own them; the copies take whole vectors inside the buffer and plain
// loads the ragged ends of the first and last row.
// Modes from 2 on: temperatures 1 and `mode` (2, 3 or 4): e^z is that power of e^(z / mode).
enum { EXP_POWERS = 2 };
template <int MODE> __device__ __forceinline__ float power(float x) { return MODE == 2 ? x * x : MODE == 3 ? x * x * x : (x * x) * (x * x); }
template <int MODE> __device__ __forceinline__ uint64_t power2(uint64_t x) {
  const uint64_t s = tc::mul2(x, x);
  return MODE == 2 ? s : MODE == 3 ? tc::mul2(s, x) : tc::mul2(s, s);
}

__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// the W values of a 16-byte vector as W / 2 packed pairs
__device__ __forceinline__ uint64_t pair_of(const Vec16<bf16>& r, int i) { return tc::bf16x2_to_f32x2(reinterpret_cast<const uint32_t*>(&r.raw)[i]); }
__device__ __forceinline__ uint64_t pair_of(const Vec16<float>& r, int i) { return tc::pack2(r.get(2 * i), r.get(2 * i + 1)); }

__device__ __forceinline__ uint64_t exp_pair(uint64_t x) {
  float a, c;
  tc::unpack2(x, a, c);
  return tc::pack2(ex2(a), ex2(c));
}

// The same on the fp32 units, for x <= 0: 2^x = 2^n 2^f with n = rint(x), f in [-1/2, 1/2] and 2^f by a polynomial of degree 5 (fitted for
// the least relative error with p(0) = 1, each coefficient rounded to fp32 before the next was fitted): 9.3e-8, with the roundings
// 1.6e-7, where ex2.approx is allowed 2^-22 = 2.4e-7.  -inf gives 0 (its n of -127 becomes a factor of 0), NaN stays.
__device__ __forceinline__ uint64_t exp_pair_poly(uint64_t x) {
  float a, c;
  tc::unpack2(x, a, c);
  asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(a));      // -127
  asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(c));
  auto both = [](float v) { return tc::pack2(v, v); };
  const uint64_t xs = tc::pack2(a, c), t = tc::add2(xs, both(12582912.0f));      // n in the low bits
  const uint64_t f = tc::add2(xs, tc::fma2(t, both(-1.0f), both(12582912.0f)));
  uint64_t p = tc::fma2(f, both(0x1.5bda36p-10f), both(0x1.3ce8aap-7f));
  p = tc::fma2(p, f, both(0x1.c6b6d8p-5f));
  p = tc::fma2(p, f, both(0x1.ebf9c2p-3f));
  p = tc::fma2(p, f, both(0x1.62e42ap-1f));
  p = tc::fma2(p, f, both(1.0f));
  tc::unpack2(t, a, c);
  return tc::mul2(p, tc::pack2(__uint_as_float((__float_as_uint(a) << 23) + 0x3f800000u), __uint_as_float((__float_as_uint(c) << 23) + 0x3f800000u)));
}

// EXP_TWO: every second pair's second exponential goes there, a quarter of all (4096 x 50257 bf16 at T 1.3: none 261 us, a quarter 228,
// three eighths 243).
__device__ __forceinline__ uint64_t exp_second(int i, uint64_t x) { return i % 2 == 1 ? exp_pair_poly(x) : exp_pair(x); }

// A pair's share of the sums of exponentials (dd: logits less the maximum; i: its number in the vector), and its gradient
// f1 e^(c1 dd) + fT e^(cT dd).
template <int MODE> __device__ __forceinline__ void add_exps(uint64_t dd, int i, uint64_t cT2, uint64_t c12, uint64_t& sT2, uint64_t& s12) {
  const uint64_t e = exp_pair(tc::mul2(dd, cT2));
  sT2 = tc::add2(sT2, e);
  if constexpr (MODE == 2) s12 = tc::fma2(e, e, s12);
  if constexpr (MODE > 2) s12 = tc::add2(s12, power2<MODE>(e));
  if constexpr (MODE == EXP_TWO) s12 = tc::add2(s12, exp_second(i, tc::mul2(dd, c12)));
}
template <int MODE> __device__ __forceinline__ uint64_t slopes(uint64_t dd, int i, uint64_t cT2, uint64_t c12, uint64_t f12, uint64_t fT2) {
  const uint64_t e = exp_pair(tc::mul2(dd, cT2));
  if constexpr (MODE == EXP_ONE) return tc::mul2(e, f12);
  else if constexpr (MODE == 2) return tc::mul2(e, tc::fma2(e, f12, fT2));
  else if constexpr (MODE > 2) return tc::fma2(power2<MODE>(e), f12, tc::mul2(e, fT2));
  else return tc::fma2(e, fT2, tc::mul2(f12, exp_second(i, tc::mul2(dd, c12))));
}
template <int MODE> __device__ __forceinline__ float slope(float dd, float cT, float c1, float f1, float fT) {
  const float x = ex2(dd * cT);
  if constexpr (MODE == EXP_ONE) return f1 * x;
  else if constexpr (MODE == EXP_TWO) return fmaf(f1, ex2(dd * c1), fT * x);
  else return fmaf(f1, power<MODE>(x), fT * x);
}
// a vector's gradient, rounded
template <int MODE, typename T> __device__ __forceinline__ Vec16<T> slopes_of(const Vec16<T>& r, uint64_t neg2, uint64_t cT2, uint64_t c12, uint64_t f12, uint64_t fT2) {
  Vec16<T> o;
#pragma unroll
  for (int i = 0; i < Vec16<T>::N / 2; ++i) {
    float a, c;
    tc::unpack2(slopes<MODE>(tc::add2(pair_of(r, i), neg2), i, cT2, c12, f12, fT2), a, c);
    if constexpr (Vec16<T>::N == 8) reinterpret_cast<__nv_bfloat162*>(&o.raw)[i] = __floats2bfloat162_rn(a, c);
    else { o.set(2 * i, a); o.set(2 * i + 1, c); }
  }
  return o;
}

// maximum over a warp in one instruction, on integers in the order of the floats (no NaN comes here)
__device__ __forceinline__ float warp_max_redux(float v) {
  const int i = __float_as_int(v), o = i ^ ((i >> 31) & 0x7fffffff), m = __reduce_max_sync(0xffffffffu, o);
  return __int_as_float(m ^ ((m >> 31) & 0x7fffffff));
}

// Positions [from, to) of a row of the gradient (position 0: a 16-byte boundary of the logits) become zero; thread t of n.
template <typename T> __device__ __forceinline__ void zero_span(T* out, int from, int to, int t, int n, bool whole) {
  constexpr int W = Vec16<T>::N;
  for (int v = from / W + t; v * W < to; v += n) {
    if (whole && v * W >= from && (v + 1) * W <= to) *reinterpret_cast<uint4*>(out + (int64_t)v * W) = make_uint4(0u, 0u, 0u, 0u);
    else
      for (int i = 0; i < W; ++i)
        if (v * W + i >= from && v * W + i < to) out[v * W + i] = from_f<T>(0.f);
  }
}

// One warp: a row's teacher entries, q holding their logits: q_j = softmax(t / T) in place, log q_j = (t_j - top) / T - lts; absent entries
// and the room up to a multiple of four get index -1.
struct Teacher { float top, lts; bool some; };
__device__ __forceinline__ Teacher teacher_of(int* idx, float* q, const DistillArgs& p, int lane) {
  const int k = p.k, k4 = (k + 3) / 4 * 4;
  float tmax = -INFINITY, tsum = 0.f;
  for (int j = lane; j < k; j += 32) {
    const int v = idx[j];
    const bool ok = v >= 0 && v < p.V;
    const float t = ok ? q[j] : -INFINITY;
    if (!ok) { idx[j] = -1; q[j] = t; }
    tmax = t != t || tmax != tmax ? __uint_as_float(0x7fffffffu) : fmaxf(tmax, t);
  }
  for (int j = k + lane; j < k4; j += 32) idx[j] = -1;
  const bool nan = __any_sync(0xffffffffu, tmax != tmax);
  tmax = warp_max_redux(nan ? 0.f : tmax);
  if (nan) tmax = __uint_as_float(0x7fffffffu);
  const bool some = tmax != -INFINITY && p.wk != 0.f;      // else the teacher says nothing about this row
  for (int j = lane; j < k; j += 32) tsum += some ? expf((q[j] - tmax) * p.inv_t) : 0.f;
  tsum = warp_sum(tsum);
  for (int j = lane; j < k; j += 32) q[j] = some ? expf((q[j] - tmax) * p.inv_t) / tsum : 0.f;
  return {tmax, logf(tsum), some};
}
// The entries of a row that carry a target, entries j0, j0 + step ...: the first entry of an index writes for all of them.  zt: their logits.
struct Slope { float base, f1, fT, fq, fy; };              // gradient = slope(z) - fq sum of q - fy at the label
template <int MODE, typename T>
__device__ __forceinline__ void targets(T* out, const Slope& f, const DistillArgs& p, int j0, int step, const int* idx, const float* q, const float* zt, int y, float zy) {
  const int k = p.k;
  for (int j = j0; j <= k; j += step) {
    const int v = j < k ? idx[j] : p.labels ? y : -1;      // entry k: the label
    if (v < 0) continue;
    bool first = true;
    float sum = 0.f;
    for (int i = 0; i < k; i += 4) {
      const int4 w = *reinterpret_cast<const int4*>(&idx[i]);
      if (w.x == v) { if (i < j) first = false; sum += q[i]; }
      if (w.y == v) { if (i + 1 < j) first = false; sum += q[i + 1]; }
      if (w.z == v) { if (i + 2 < j) first = false; sum += q[i + 2]; }
      if (w.w == v) { if (i + 3 < j) first = false; sum += q[i + 3]; }
    }
    if (!first) continue;
    float r = slope<MODE>((j < k ? zt[j] : zy) - f.base, p.cT, p.c1, f.f1, f.fT) - f.fq * sum;
    if (p.labels && v == y) r -= f.fy;
    out[v] = from_f<T>(r);
  }
}

constexpr int SLOTS = 4;     // rows whose tables are in use at once: two ahead, this one, the one whose targets are being written
constexpr int BATCH = 128;   // rows of a block that are looked at together for those that take part

// MINB: blocks per SM.  One barrier per row (two with one buffer).  Behind it every sum is there, and the previous row's gradient
// has been written but for the entries with a target, which follow then.  What a row needs besides its logits is spread over the
// warps: 0 the row's loss, 1 the ragged ends and the teacher's distribution of the next row, the others the previous row's targets.
template <typename T, int THREADS, int MINB, int MODE>
__global__ void __launch_bounds__(THREADS, MINB)
distill_ring_kernel(const T* logits, T* grad, DistillArgs p, int M, int nbuf, int buf_bytes, int* status) {
  constexpr int W = Vec16<T>::N, NW = THREADS / 32, ISSUER = THREADS - 32;
  constexpr int UNROLL = THREADS > 128 ? 4 : 2;          // many blocks in different places of their rows: the code has to stay cached
  extern __shared__ __align__(128) uint8_t smem[];       // nbuf rows, then the tables of the teacher's entries
  const int k4 = (p.k + 3) / 4 * 4;
  int* tables = reinterpret_cast<int*>(smem + (size_t)nbuf * buf_bytes);
  auto sh_idx = [&](int slot) { return tables + slot * k4; };
  auto sh_q = [&](int slot) { return reinterpret_cast<float*>(tables + (SLOTS + slot) * k4); };
  auto sh_z = [&](int par) { return reinterpret_cast<float*>(tables + (2 * SLOTS + par) * k4); };
  __shared__ float sh_m[2][NW], sh_sT[2][NW], sh_s1[2][NW];
  __shared__ T sh_edge[2][2][W];                         // logits of the row's ragged first and last vector
  __shared__ float sh_zy[2], sh_f1[2], sh_fT[2], sh_base[2], sh_fq[2];
  __shared__ float sh_tmax[SLOTS], sh_lts[SLOTS];        // log q_j = (t_j - tmax) / T - lts
  __shared__ int sh_teach[SLOTS], sh_rows[BATCH], sh_ys[BATCH], sh_cnt[NW], sh_abort;
  __shared__ __align__(8) uint64_t bars[2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int V = p.V, k = p.k;
  const uint32_t smem_base = tc::smem_u32(smem);
  if (tid == 0) {
    tc::mbar_init(tc::smem_u32(&bars[0]), 1);
    tc::mbar_init(tc::smem_u32(&bars[1]), 1);
    sh_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  overlap_sync();

  auto takes_part = [&](int y) { return y >= 0 && y < V; };
  int n = p.n_fixed;
  if (p.n_valid && !p.count_here) n = *p.n_valid;
  if (p.count_here) {                      // few labels: every block counts them itself
    int c = 0;
    for (int i = tid; i < M; i += THREADS) c += takes_part(p.labels[i]) ? 1 : 0;
    c = __reduce_add_sync(0xffffffffu, c);
    if (lane == 0) sh_cnt[warp] = c;
    __syncthreads();
    n = 0;
    for (int w = 0; w < NW; ++w) n += sh_cnt[w];
    if (blockIdx.x == 0 && tid == 0) *p.n_valid = n;
  }
  const float inv_n = 1.0f / (float)(n > 0 ? n : 1);

  // thread ISSUER: logits of a row into a buffer
  auto issue = [&](int row, int b) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(logits + row * p.ld), a1 = a0 + (uintptr_t)V * sizeof(T), f0 = a0 & ~(uintptr_t)15;
    const uintptr_t lo = row == 0 && f0 < a0 ? f0 + 16 : f0, hi = row == M - 1 ? a1 & ~(uintptr_t)15 : (a1 + 15) & ~(uintptr_t)15;
    const uint32_t bytes = hi > lo ? (uint32_t)(hi - lo) : 0u, bar = tc::smem_u32(&bars[b]);
    tc::mbar_expect_tx(bar, bytes);
    if (bytes)
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                   ::"r"(smem_base + (uint32_t)(b * buf_bytes) + (uint32_t)(lo - f0)), "l"(lo), "r"(bytes), "r"(bar) : "memory");
  };
  // warp 1: a row's teacher entries into the tables; lane j % 32 copies entry j and is the one that reads it
  auto fetch_teacher = [&](int row, int slot) {
    for (int j = lane; j < k; j += 32) {
      cp_async4(tc::smem_u32(&sh_idx(slot)[j]), p.idx + (int64_t)row * k + j);
      cp_async4(tc::smem_u32(&sh_q(slot)[j]), p.t + (int64_t)row * k + j);
    }
  };
  auto teacher = [&](int slot) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    const Teacher t = teacher_of(sh_idx(slot), sh_q(slot), p, lane);
    if (lane == 0) { sh_teach[slot] = t.some; sh_tmax[slot] = t.top; sh_lts[slot] = t.lts; }
  };
  // from warp 2 on
  auto write_targets = [&](int row, int y, int slot, int par) {
    const Slope f{sh_base[par], sh_f1[par], sh_fT[par], sh_fq[par], p.wc * inv_n};
    targets<MODE>(grad + row * p.ldo, f, p, tid - 64, THREADS - 64, sh_idx(slot), sh_q(slot), sh_z(par), y, sh_zy[par]);
  };
  auto zeros = [&](T* out, int from, int to) { zero_span(out, from, to, tid, THREADS, p.same != 0); };
  auto shift_of = [&](int row) { return (int)((reinterpret_cast<uintptr_t>(logits + row * p.ld) & 15u) / sizeof(T)); };

  const uint64_t cT2 = tc::pack2(p.cT, p.cT), c12 = tc::pack2(p.c1, p.c1);
  int used = 0;                            // rows copied so far: buffer used % nbuf, phase used / nbuf
  for (int64_t row0 = blockIdx.x; row0 < M; row0 += (int64_t)BATCH * gridDim.x) {
    // ---- which of the next rows take part
    __syncthreads();                       // the previous batch's lists and tables
    int count = 0;
    for (int i0 = 0; i0 < BATCH; i0 += 32) {             // (every warp for itself; warp 0 writes the list)
      const int64_t r = row0 + (int64_t)(i0 + lane) * gridDim.x;
      const int y = r < M && p.labels ? p.labels[r] : 0;
      const bool in = r < M && takes_part(y);
      const uint32_t mask = __ballot_sync(0xffffffffu, in);
      if (warp == 0 && in) {
        const int at = count + __popc(mask & ((1u << lane) - 1u));
        sh_rows[at] = (int)r;
        sh_ys[at] = y;
      }
      uint32_t out_mask = __ballot_sync(0xffffffffu, r < M && !in);
      while (out_mask) {                   // a row that takes no part: zeros
        const int l = __ffs(out_mask) - 1;
        out_mask &= out_mask - 1;
        const int row = (int)(row0 + (int64_t)(i0 + l) * gridDim.x), s = shift_of(row);
        if (tid == 0) p.rows[row] = 0.f;
        zeros(grad + row * p.ldo - s, s, s + (int)p.ldo);
      }
      count += __popc(mask);
    }
    __syncthreads();
    if (tid == ISSUER)
      for (int b = 0; b < nbuf && b < count; ++b) issue(sh_rows[b], (used + b) % nbuf);
    if (warp == 1 && count > 0) {
      fetch_teacher(sh_rows[0], 0);
      teacher(0);
      if (count > 1) fetch_teacher(sh_rows[1], 1);
    }
    for (int at = 0; at < count; ++at, ++used) {
      const int row = sh_rows[at], y = sh_ys[at], slot = at % SLOTS, par = at & 1, b = used % nbuf, s = shift_of(row);
      T* out = grad + row * p.ldo - s;     // position q = s + column
      const int end = s + V, nvec = (end + W - 1) / W, last = nvec - 1;
      const bool arrived = tc::mbar_wait(tc::smem_u32(&bars[b]), (uint32_t)(used / nbuf) & 1u, &sh_abort, status, 81);
      T* zs = reinterpret_cast<T*>(smem + (size_t)b * buf_bytes);
      // A ragged first or last vector (in the first and last row of all the copies left it out): the thread that owns it keeps its
      // logits for the gradient and puts -inf around them.
      const bool ragged_first = s > 0 || (last == 0 && end % W != 0), ragged_last = end % W != 0;
      if ((tid == 0 && ragged_first) || (tid == last % THREADS && ragged_last)) {
        const T* z = logits + row * p.ld - s;
        const bool left = row == 0 || row == M - 1;
        for (int which = tid == 0 && ragged_first ? 0 : 1; which < (tid == last % THREADS && ragged_last ? 2 : 1); ++which)
          for (int i = 0; i < W; ++i) {
            const int q = (which ? last * W : 0) + i;
            const T v = q < s || q >= end ? from_f<T>(-INFINITY) : left ? z[q] : zs[q];
            zs[q] = v;
            sh_edge[par][which][i] = v;
          }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // before a copy takes the buffer again
      }
      // ---- this thread's maximum, then its exponentials relative to it
      float m = -INFINITY;
      if constexpr (W == 8) {
        __nv_bfloat162 m2 = __floats2bfloat162_rn(-INFINITY, -INFINITY);
#pragma unroll UNROLL
        for (int v = tid; v < nvec; v += THREADS) {
          Vec16<T> r; r.load(zs + (size_t)v * W);
          const __nv_bfloat162* h2 = reinterpret_cast<const __nv_bfloat162*>(&r.raw);
          m2 = __hmax2(m2, __hmax2(__hmax2(h2[0], h2[1]), __hmax2(h2[2], h2[3])));
        }
        m = fmaxf(__low2float(m2), __high2float(m2));
      } else {
#pragma unroll UNROLL
        for (int v = tid; v < nvec; v += THREADS) {
          Vec16<T> r; r.load(zs + (size_t)v * W);
#pragma unroll
          for (int i = 0; i < W; ++i) m = fmaxf(m, r.get(i));
        }
      }
      const float mine = m == -INFINITY ? 0.f : m;
      uint64_t sT2 = 0ull, s12 = 0ull;
      {
        const uint64_t neg2 = tc::pack2(-mine, -mine);
#pragma unroll UNROLL
        for (int v = tid; v < nvec; v += THREADS) {
          Vec16<T> r; r.load(zs + (size_t)v * W);
#pragma unroll
          for (int i = 0; i < W / 2; ++i) {
            add_exps<MODE>(tc::add2(pair_of(r, i), neg2), i, cT2, c12, sT2, s12);
          }
        }
      }
      float sT, s1;
      {
        float a, c;
        tc::unpack2(sT2, a, c); sT = a + c;
        tc::unpack2(s12, a, c); s1 = a + c;
      }
      // ---- the row's maximum and sums.  Without a maximum the sums are 0 or, from NaN, NaN: no factor
      auto factor = [&](float from, float to, float c) { return from == -INFINITY ? 1.f : ex2((from - to) * c); };
      const float wm = warp_max_redux(m), wbase = wm == -INFINITY ? 0.f : wm;
      {
        const float f = factor(m, wbase, p.cT);
        sT = warp_sum(sT * f);
        if constexpr (MODE >= EXP_POWERS) s1 = warp_sum(s1 * power<MODE>(f));
        if constexpr (MODE == EXP_TWO) s1 = warp_sum(s1 * factor(m, wbase, p.c1));
      }
      if (lane == 0) {
        sh_m[par][warp] = wm; sh_sT[par][warp] = sT;
        if constexpr (MODE != EXP_ONE) sh_s1[par][warp] = s1;
      }
      if (__syncthreads_or(!arrived)) {
        // A row that did not arrive: `status` holds the code, neither this row nor a later one of the block is written, no copy follows.
        // Those under way (this row's; before the first row's barrier the second row's too) land, or 2 ms pass, before the shared
        // memory becomes another block's.
        auto landed = [&](int u) { return tc::mbar_test(tc::smem_u32(&bars[u % nbuf]), (uint32_t)(u / nbuf) & 1u); };
        const bool second = nbuf > 1 && at == 0 && count > 1;
        for (int i = 0; i < 2000 && !(landed(used) && (!second || landed(used + 1))); ++i) __nanosleep(1000);
        return;
      }
      if (tid == ISSUER && nbuf > 1 && at > 0 && at + 1 < count) issue(sh_rows[at + 1], (used + 1) % nbuf);    // nobody reads the previous row's logits any more
      float base;
      {
        float rm = sh_m[par][lane % NW];
        sT = sh_sT[par][lane % NW];
        s1 = MODE == EXP_ONE ? 0.f : sh_s1[par][lane % NW];
        m = warp_max_redux(rm);
        base = m == -INFINITY ? 0.f : m;
        const float f = factor(rm, base, p.cT);
        sT *= f;
        if constexpr (MODE >= EXP_POWERS) s1 *= power<MODE>(f);
        if constexpr (MODE == EXP_TWO) s1 *= factor(rm, base, p.c1);
#pragma unroll
        for (int o = NW / 2; o > 0; o >>= 1) {
          sT += __shfl_xor_sync(0xffffffffu, sT, o);
          if constexpr (MODE != EXP_ONE) s1 += __shfl_xor_sync(0xffffffffu, s1, o);
        }
        if constexpr (MODE == EXP_ONE) s1 = sT;
      }
      const float wkT = sh_teach[slot] ? p.wk * p.temp : 0.f;
      const float f1 = MODE == EXP_ONE ? (p.wc + wkT) / s1 * inv_n : p.wc / s1 * inv_n, fT = MODE == EXP_ONE ? 0.f : wkT / sT * inv_n;
      if (warp == 0) {                     // the divergence, the row's loss, and what its targets need
        const float log_sT = logf(sT), tmax = sh_tmax[slot], lts = sh_lts[slot], *t = p.t + (int64_t)row * k;
        float kl = 0.f;
        for (int j = lane; j < k; j += 32) {
          const int v = sh_idx(slot)[j];
          const float q = sh_q(slot)[j], z = v >= 0 ? to_f<T>(zs[s + v]) : 0.f;
          sh_z(par)[j] = z;
          // T times the divergence: (z - base) / T could overflow
          if (q != 0.f) kl += q * fmaf(p.temp, ((t[j] - tmax) * p.inv_t - lts) + log_sT, base - z);
        }
        kl = warp_sum(kl);
        if (lane == 0) {
          const float zy = p.labels ? to_f<T>(zs[s + y]) : 0.f;
          float r = wkT != 0.f ? p.wk * p.temp * kl : 0.f;
          if (p.wc != 0.f) r += p.wc * (logf(s1) - (zy - base));
          p.rows[row] = r;
          sh_zy[par] = zy; sh_f1[par] = f1; sh_fT[par] = fT; sh_base[par] = base; sh_fq[par] = wkT * inv_n;
        }
      } else if (warp == 1) {
        if (lane < 2 * W) {                // the ragged ends, one logit per lane
          const int which = lane / W, i = lane % W, q = (which ? last * W : 0) + i;
          if ((which ? ragged_last : ragged_first && !(last == 0 && ragged_last)) && q >= s && q < end) {
            out[q] = from_f<T>(slope<MODE>(to_f<T>(sh_edge[par][which][i]) - base, p.cT, p.c1, f1, fT));
          }
        }
        __syncwarp();
        if (at + 1 < count) teacher((at + 1) % SLOTS);
        if (at + 2 < count) fetch_teacher(sh_rows[at + 2], (at + 2) % SLOTS);
      } else if (at > 0) {
        write_targets(sh_rows[at - 1], sh_ys[at - 1], (at - 1) % SLOTS, par ^ 1);
      }
      // ---- gradient
      const uint64_t f12 = tc::pack2(f1, f1), fT2 = tc::pack2(fT, fT), neg2 = tc::pack2(-base, -base);
      const int v_to = ragged_last ? last : nvec;
#pragma unroll UNROLL
      for (int v = tid == 0 && ragged_first ? THREADS : tid; v < v_to; v += THREADS) {
        Vec16<T> r;
        r.load(zs + (size_t)v * W);
        const Vec16<T> o = slopes_of<MODE>(r, neg2, cT2, c12, f12, fT2);
        if (p.same) o.store(out + (int64_t)v * W);
        else
#pragma unroll
          for (int i = 0; i < W; ++i) out[v * W + i] = reinterpret_cast<const T*>(&o.raw)[i];
      }
      if (p.ldo > V) zeros(out, end, s + (int)p.ldo);
      if (nbuf == 1) {
        __syncthreads();
        if (tid == ISSUER && at + 1 < count) issue(sh_rows[at + 1], 0);
      }
    }
    if (count > 0) {
      __syncthreads();
      if (warp >= 2) write_targets(sh_rows[count - 1], sh_ys[count - 1], (count - 1) % SLOTS, (count - 1) & 1);
    }
  }
}

// ------------------------------------------------------------------------------------------
// rows in the registers of a warp
// ------------------------------------------------------------------------------------------
// A warp per row of up to 32 x NVR vectors, eight rows per block: no barriers between a row's steps, and other rows' loads in flight on
// the SM's other warps.  What bounds it is the chain of a row (the teacher's entries, three reductions, the targets), then launches: 300
// x 117 takes 8.3 us, of which the sum over the rows' losses, a launch of its own, is 4.
constexpr int WARP_ROWS = 8;
template <typename T, int NVR, int MODE>
__global__ void __launch_bounds__(32 * WARP_ROWS, NVR == 4 ? 4 : 3)
distill_warp_kernel(const T* logits, T* grad, DistillArgs p, int M) {
  constexpr int W = Vec16<T>::N;
  extern __shared__ __align__(16) int warp_tables[];       // per row: indexes, weights, logits of the teacher's entries
  __shared__ int sh_cnt[WARP_ROWS];
  overlap_sync();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, V = p.V, k = p.k, k4 = (k + 3) / 4 * 4;
  const int64_t row = (int64_t)blockIdx.x * WARP_ROWS + warp;
  const bool in = row < M;
  const int y = in && p.labels ? p.labels[row] : 0;
  const bool valid = in && y >= 0 && y < V;
  const T* z = logits + (in ? row : 0) * p.ld;
  int* idx = warp_tables + warp * 3 * k4;
  float* q = reinterpret_cast<float*>(idx + k4), *zt = q + k4;
  // position = column + s; whole vectors [v0, v1) and up to 14 elements around them, one per lane
  const int s = (int)((reinterpret_cast<uintptr_t>(z) & 15u) / sizeof(T)), end = s + V, v0 = s > 0 ? 1 : 0, v1 = max(end / W, v0);
  const int head = v0 ? min(W, end) - s : 0, edges = head + max(end - v1 * W, 0), ec = lane < head ? lane : v1 * W - s + lane - head;
  const bool has_edge = valid && lane < edges;
  Vec16<T> raw[NVR];
#pragma unroll
  for (int i = 0; i < NVR; ++i) {
    const int v = v0 + i * 32 + lane;
    if (valid && v < v1) raw[i].load(z + v * W - s);
    else
#pragma unroll
      for (int c = 0; c < W; ++c) raw[i].set(c, -INFINITY);
  }
  const float ez = has_edge ? to_f<T>(z[ec]) : -INFINITY, zy = valid && p.labels ? to_f<T>(z[y]) : 0.f;
  if (valid)
    for (int j = lane; j < k; j += 32) {
      const int v = p.idx[row * k + j];
      idx[j] = v;
      q[j] = p.t[row * k + j];
      zt[j] = v >= 0 && v < V ? to_f<T>(z[v]) : 0.f;
    }
  int n = p.n_fixed;
  if (p.n_valid && !p.count_here) n = *p.n_valid;
  if (p.count_here) {
    int c = 0;
    for (int i = tid; i < M; i += 32 * WARP_ROWS) c += p.labels[i] >= 0 && p.labels[i] < V ? 1 : 0;
    c = __reduce_add_sync(0xffffffffu, c);
    if (lane == 0) sh_cnt[warp] = c;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < WARP_ROWS; ++w) n += sh_cnt[w];
    if (blockIdx.x == 0 && tid == 0) *p.n_valid = n;
  }
  if (!in) return;
  const float inv_n = 1.0f / (float)(n > 0 ? n : 1);
  T* out = grad + row * p.ldo;
  zero_span(out - s, valid ? end : s, s + (int)p.ldo, lane, 32, p.same != 0);
  if (!valid) {
    if (lane == 0) p.rows[row] = 0.f;
    return;
  }
  // ---- maximum, sums
  float m = ez != ez ? -INFINITY : ez;
#pragma unroll
  for (int i = 0; i < NVR; ++i)
    if constexpr (W == 8) {
      const __nv_bfloat162* h2 = reinterpret_cast<const __nv_bfloat162*>(&raw[i].raw);
      const __nv_bfloat162 m2 = __hmax2(__hmax2(h2[0], h2[1]), __hmax2(h2[2], h2[3]));
      m = fmaxf(m, fmaxf(__low2float(m2), __high2float(m2)));
    } else {
#pragma unroll
      for (int c = 0; c < W; ++c) m = fmaxf(m, raw[i].get(c));
    }
  m = warp_max_redux(m);
  const float base = m == -INFINITY ? 0.f : m;
  const uint64_t cT2 = tc::pack2(p.cT, p.cT), c12 = tc::pack2(p.c1, p.c1);
  const uint64_t neg2 = tc::pack2(-base, -base);
  uint64_t sT2 = 0ull, s12 = 0ull;
#pragma unroll
  for (int i = 0; i < NVR; ++i)
#pragma unroll
    for (int c = 0; c < W / 2; ++c) add_exps<MODE>(tc::add2(pair_of(raw[i], c), neg2), c, cT2, c12, sT2, s12);
  float sT, s1;
  {
    add_exps<MODE>(tc::pack2(ez - base, -INFINITY), 0, cT2, c12, sT2, s12);
    float a, c;
    tc::unpack2(sT2, a, c); sT = warp_sum(a + c);
    tc::unpack2(s12, a, c); s1 = MODE == EXP_ONE ? sT : warp_sum(a + c);
  }
  // ---- the teacher's distribution, the divergence and the row's loss
  const Teacher te = teacher_of(idx, q, p, lane);
  const float wkT = te.some ? p.wk * p.temp : 0.f, log_sT = logf(sT);
  float kl = 0.f;
  for (int j = lane; j < k; j += 32)
    if (q[j] != 0.f) kl += q[j] * fmaf(p.temp, ((p.t[row * k + j] - te.top) * p.inv_t - te.lts) + log_sT, base - zt[j]);     // T times the divergence
  kl = warp_sum(kl);
  if (lane == 0) {
    float r = wkT != 0.f ? p.wk * p.temp * kl : 0.f;
    if (p.wc != 0.f) r += p.wc * (logf(s1) - (zy - base));
    p.rows[row] = r;
  }
  // ---- gradient
  const float f1 = MODE == EXP_ONE ? (p.wc + wkT) / s1 * inv_n : p.wc / s1 * inv_n, fT = MODE == EXP_ONE ? 0.f : wkT / sT * inv_n;
  const uint64_t f12 = tc::pack2(f1, f1), fT2 = tc::pack2(fT, fT);
  __syncwarp();                            // every lane has read what it needs of the row: the gradient may lie over it
#pragma unroll
  for (int i = 0; i < NVR; ++i) {
    const int v = v0 + i * 32 + lane;
    if (v < v1) {
      // formed from the logits again: the compiler would keep converted logits or exponentials, twice the registers
      uint32_t* w = reinterpret_cast<uint32_t*>(&raw[i].raw);
      asm volatile("" : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3]));
      const Vec16<T> o = slopes_of<MODE>(raw[i], neg2, cT2, c12, f12, fT2);
      T* at = out + v * W - s;
      if (p.same) o.store(at);
      else
#pragma unroll
        for (int c = 0; c < W; ++c) at[c] = reinterpret_cast<const T*>(&o.raw)[c];
    }
  }
  if (has_edge) out[ec] = from_f<T>(slope<MODE>(ez - base, p.cT, p.c1, f1, fT));
  __syncwarp();                            // the tables, and the targets' first values
  targets<MODE>(out, Slope{base, f1, fT, wkT * inv_n, p.wc * inv_n}, p, lane, 32, idx, q, zt, y, zy);
}

// One block each: eight elements per thread under way at a time, added up in an order of their own.
constexpr int TALLY = 1024, TALLY_EACH = 8;
__global__ void __launch_bounds__(TALLY) distill_count_kernel(const int32_t* __restrict__ labels, int M, int V, int* __restrict__ n_valid) {
  overlap_sync();
  __shared__ int sh[32];
  int c = 0;
  for (int i0 = threadIdx.x; i0 < M; i0 += TALLY * TALLY_EACH) {
    int y[TALLY_EACH];
#pragma unroll
    for (int e = 0; e < TALLY_EACH; ++e) y[e] = i0 + e * TALLY < M ? labels[i0 + e * TALLY] : -1;
#pragma unroll
    for (int e = 0; e < TALLY_EACH; ++e) c += y[e] >= 0 && y[e] < V ? 1 : 0;
  }
  c = __reduce_add_sync(0xffffffffu, c);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = c;
  __syncthreads();
  if (threadIdx.x < 32) {
    c = __reduce_add_sync(0xffffffffu, sh[threadIdx.x]);
    if (threadIdx.x == 0) *n_valid = c;
  }
}

__global__ void __launch_bounds__(TALLY) distill_loss_kernel(const float* __restrict__ rows, int M, const int* __restrict__ n_valid, int n_fixed, float* __restrict__ loss) {
  overlap_sync();
  __shared__ double sh[32];
  double s = 0.0;
  for (int i0 = threadIdx.x; i0 < M; i0 += TALLY * TALLY_EACH) {
    float r[TALLY_EACH];
#pragma unroll
    for (int e = 0; e < TALLY_EACH; ++e) r[e] = i0 + e * TALLY < M ? rows[i0 + e * TALLY] : 0.f;
#pragma unroll
    for (int e = 0; e < TALLY_EACH; ++e) s += (double)r[e];
  }
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x < 32) {
    s = sh[threadIdx.x];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int n = n_valid ? *n_valid : n_fixed;
    if (threadIdx.x == 0) *loss = n > 0 ? (float)(s / n) : 0.f;
  }
}

}  // namespace

namespace {

// Up to this many labels are counted by every block of the warp and ring kernels instead of a launch in front of them.
constexpr int COUNT_HERE = 4096;
// Static shared memory of a block with what the system keeps per block, dynamic shared memory of a block, all of an SM's.
constexpr int RING_STATIC = 4096, RING_BYTES = 229376, SM_BYTES = 233472;

template <typename T, int THREADS, int MINB, int MODE>
cudaError_t launch_ring(const T* logits, T* grad, const DistillArgs& p, int M, int buf, int nbuf, int tables, int fit, int* status, cudaStream_t st) {
  const auto kernel = distill_ring_kernel<T, THREADS, MINB, MODE>;
  static PerDeviceOnce once;
  const int dev = current_device();
  if (once.needed(dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, RING_BYTES);
    if (e != cudaSuccess) return e;
    once.done(dev);
  }
  const int64_t most = (int64_t)num_sms() * (fit < MINB ? fit : MINB);
  return launch_overlapped(kernel, dim3((unsigned)(M < most ? M : most)), dim3(THREADS), (size_t)nbuf * buf + tables, st, logits, grad, p, M, nbuf, buf, status);
}

// Rows of up to 8 vectors per lane of a warp.  Warps and rings, bf16 at T 2: 16384 x 128 28 and 55 us, 8192 x 1000 18.6 and 36, 8192 x
// 2000 25 and 41; with 16 vectors 8192 x 4000 49 and 52, but 64 x 4000 11.3 and 10.3.
constexpr int WARP_MOST = 8 * 32;
template <typename T, int MODE>
cudaError_t warp_rows(const T* logits, T* grad, const DistillArgs& p, int M, cudaStream_t st) {
  const int nv = p.V / Vec16<T>::N;
  auto go = [&](auto kernel) -> cudaError_t {
    return launch_overlapped(kernel, dim3((unsigned)((M + (int64_t)WARP_ROWS - 1) / WARP_ROWS)), dim3(32 * WARP_ROWS), (size_t)WARP_ROWS * 3 * ((p.k + 3) / 4 * 4) * 4, st,
                             logits, grad, p, M);
  };
  return nv <= 4 * 32 ? go(distill_warp_kernel<T, 4, MODE>) : go(distill_warp_kernel<T, 8, MODE>);
}

int ring_buffer(int V, size_t es) { return (int)(((size_t)V * es + 15) / 16 * 16 + 16); }         // a row at any alignment
int ring_tables(int k) { return (2 * SLOTS + 2) * ((k + 3) / 4 * 4) * 4; }
bool ring_supported(int V, int k, size_t es) { return (int64_t)V * (int64_t)es + 32 + ring_tables(k) <= RING_BYTES; }

// As many rows per SM as shared memory holds, up to eight; two buffers per row where eight rows have room for them.
template <typename T, int MODE>
cudaError_t ring(const T* logits, T* grad, const DistillArgs& p, int M, int* status, cudaStream_t st) {
  const int buf = ring_buffer(p.V, sizeof(T)), tables = ring_tables(p.k);
  const int one = SM_BYTES / (buf + tables + RING_STATIC), two = SM_BYTES / (2 * buf + tables + RING_STATIC);
  if (two >= 8) return launch_ring<T, 128, 8, MODE>(logits, grad, p, M, buf, 2, tables, two, status, st);
  if (one >= 6) return launch_ring<T, 128, 8, MODE>(logits, grad, p, M, buf, 1, tables, one, status, st);
  if (one >= 4) return launch_ring<T, 256, 4, MODE>(logits, grad, p, M, buf, 1, tables, one, status, st);
  if (one == 3) return launch_ring<T, 256, 3, MODE>(logits, grad, p, M, buf, 1, tables, one, status, st);
  if (one == 2) return launch_ring<T, 256, 2, MODE>(logits, grad, p, M, buf, 1, tables, one, status, st);
  return launch_ring<T, 512, 1, MODE>(logits, grad, p, M, buf, 1, tables, one, status, st);
}

}  // namespace

cudaError_t distill(int dt, const void* logits, int64_t ld, const int32_t* labels, const int32_t* idx, const float* t, int M, int V, int k,
                    float temperature, float wc, float wk, int normalizer, void* grad, int64_t ldo, float* rows, int* n_valid, float* loss,
                    int* status, cudaStream_t st) {
  DistillArgs p;
  p.labels = labels; p.idx = idx; p.t = t; p.ld = ld; p.ldo = ldo; p.V = V; p.k = k; p.temp = temperature; p.inv_t = 1.0f / temperature; p.wc = wc; p.wk = wk; p.rows = rows;
  const bool count = labels != nullptr && normalizer <= 0;
  p.n_valid = count ? n_valid : nullptr;
  p.n_fixed = normalizer > 0 ? normalizer : M;
  const bool two = wc != 0.f && wk != 0.f && temperature != 1.0f;
  // EXP_ONE: the temperature of the term that has a weight
  p.cT = two || wk != 0.f ? LOG2E / temperature : LOG2E;
  p.c1 = two ? LOG2E : p.cT;
  p.count_here = 0;
  cudaError_t e = cudaSuccess;
  const size_t es = dtype_size(dt);
  p.same = ((reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(grad)) & 15u) == 0 && ((ld - ldo) * (int64_t)es) % 16 == 0;
  const bool in_warp = V * (int64_t)es / 16 <= WARP_MOST, in_ring = ring_supported(V, k, es);
  p.count_here = in_ring && count && M <= COUNT_HERE;
  if (count && !p.count_here) {
    e = launch_overlapped(distill_count_kernel, dim3(1), dim3(TALLY), 0, st, labels, M, V, n_valid);
    if (e != cudaSuccess) return e;
  }
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int N = Vec16<T>::N;
    const T* z = (const T*)logits;
    T* g = (T*)grad;
    if (in_ring) {
      auto held = [&](auto mode) -> cudaError_t {
        return in_warp ? warp_rows<T, mode>(z, g, p, M, st) : ring<T, mode>(z, g, p, M, status, st);
      };
      if (!two) return held(std::integral_constant<int, EXP_ONE>());
      if (temperature == 2.0f) return held(std::integral_constant<int, 2>());
      if (temperature == 3.0f) return held(std::integral_constant<int, 3>());
      if (temperature == 4.0f) return held(std::integral_constant<int, 4>());
      return held(std::integral_constant<int, EXP_TWO>());
    }
    const bool vec = ld % N == 0 && ldo % N == 0 && ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(grad)) & 15u) == 0;
    auto go = [&](auto kernel) -> cudaError_t { return launch_overlapped(kernel, dim3((unsigned)M), dim3(256), 0, st, z, g, p); };
    if (vec) return two ? go(distill_kernel<T, N, EXP_TWO>) : go(distill_kernel<T, N, EXP_ONE>);
    return two ? go(distill_kernel<T, 1, EXP_TWO>) : go(distill_kernel<T, 1, EXP_ONE>);
  };
  e = dt == DT_BF16 ? run(bf16()) : run(float());
  if (e != cudaSuccess) return e;
  return launch_overlapped(distill_loss_kernel, dim3(1), dim3(TALLY), 0, st, (const float*)rows, M, (const int*)p.n_valid, p.n_fixed, loss);
}

}  // namespace sl
