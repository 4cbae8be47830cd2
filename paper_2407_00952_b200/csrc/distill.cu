// Loss over the vocabulary against a teacher's top logits and the labels, with its gradient.  Per row m with logits z (V of
// them), temperature T, the teacher's k entries (idx_j, t_j) and the label y:
//   q = softmax_j(t_j / T) over the row's entries,  p1 = softmax(z),  pT = softmax(z / T)
//   row  = wc (-log p1[y])  +  wk T^2 sum_j q_j (log q_j - log pT[idx_j])
//   dz_v = ( wc (p1_v - [v = y])  +  wk T (pT_v - sum_{j: idx_j = v} q_j) ) / n
// Both softmaxes share the row's maximum.  One block per row: a pass for the maximum and the sums of exponentials (running, so
// the logits are read once for it), a pass that writes the gradient from the logits' second read (L1 or L2), then the at most
// k + 1 entries that carry a target are written again from their saved logits, with all of a repeated index's weights summed by
// the first of its entries in order: one rounding per output, no atomics.  Exponents are formed as (z - max) * log2(e) / T: for
// the entries that matter z - max is small, so the fp32 rounding of the product stays near 2^-24 of the probability.
#include "common.cuh"
#include "host_common.h"
#include "kernels.h"
#include "launch.cuh"

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
  float* rows; const int* n_valid; int n_fixed;
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

template <typename T, int W, int MODE>
__global__ void __launch_bounds__(512)
distill_kernel(const T* __restrict__ logits, T* __restrict__ grad, DistillArgs p) {   // grad may be logits
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
  const bool some = tmax != -INFINITY;     // no entry, or none with any weight: the teacher says nothing about this row
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
  const float wk = some && p.wk != 0.f ? p.wk : 0.f;
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

__global__ void distill_count_kernel(const int32_t* __restrict__ labels, int M, int V, int* __restrict__ n_valid) {
  overlap_sync();
  __shared__ int sh[32];
  int c = 0;
  for (int i = threadIdx.x; i < M; i += blockDim.x) c += (labels[i] >= 0 && labels[i] < V) ? 1 : 0;
  c = __reduce_add_sync(0xffffffffu, c);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = c;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < (int)(blockDim.x >> 5); ++w) c += sh[w];
    *n_valid = c;
  }
}

__global__ void distill_loss_kernel(const float* __restrict__ rows, int M, const int* __restrict__ n_valid, int n_fixed, float* __restrict__ loss) {
  overlap_sync();
  __shared__ double sh[32];
  double s = 0.0;
  for (int i = threadIdx.x; i < M; i += blockDim.x) s += (double)rows[i];
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < (int)(blockDim.x >> 5); ++w) s += sh[w];
    const int n = n_valid ? *n_valid : n_fixed;
    *loss = n > 0 ? (float)(s / n) : 0.f;
  }
}

}  // namespace

cudaError_t distill(int dt, const void* logits, int64_t ld, const int32_t* labels, const int32_t* idx, const float* t, int M, int V, int k,
                    float temperature, float wc, float wk, int normalizer, void* grad, int64_t ldo, float* rows, int* n_valid, float* loss,
                    cudaStream_t st) {
  DistillArgs p;
  p.labels = labels; p.idx = idx; p.t = t; p.ld = ld; p.ldo = ldo; p.V = V; p.k = k; p.temp = temperature; p.wc = wc; p.wk = wk; p.rows = rows;
  const bool count = labels != nullptr && normalizer <= 0;
  p.n_valid = count ? n_valid : nullptr;
  p.n_fixed = normalizer > 0 ? normalizer : M;
  const bool two = wc != 0.f && wk != 0.f && temperature != 1.0f;
  // EXP_ONE: the temperature of the term that has a weight
  p.cT = LOG2E / temperature;
  p.c1 = two || wk == 0.f ? LOG2E : p.cT;
  cudaError_t e = cudaSuccess;
  if (count) {
    e = launch_overlapped(distill_count_kernel, dim3(1), dim3(1024), 0, st, labels, M, V, n_valid);
    if (e != cudaSuccess) return e;
  }
  auto run = [&](auto type) -> cudaError_t {
    using T = decltype(type);
    constexpr int N = Vec16<T>::N;
    const bool vec = ld % N == 0 && ldo % N == 0 && ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(grad)) & 15u) == 0;
    auto go = [&](auto kernel) -> cudaError_t {
      return launch_overlapped(kernel, dim3((unsigned)M), dim3(256), 0, st, (const T*)logits, (T*)grad, p);
    };
    if (vec) return two ? go(distill_kernel<T, N, EXP_TWO>) : go(distill_kernel<T, N, EXP_ONE>);
    return two ? go(distill_kernel<T, 1, EXP_TWO>) : go(distill_kernel<T, 1, EXP_ONE>);
  };
  e = dt == DT_BF16 ? run(bf16()) : run(float());
  if (e != cudaSuccess) return e;
  return launch_overlapped(distill_loss_kernel, dim3(1), dim3(1024), 0, st, (const float*)rows, M, (const int*)p.n_valid, p.n_fixed, loss);
}

}  // namespace sl
