// Products of int8 codes for layers whose frozen weight is held in 8 bits:
//   y[m, n] = round( (sum_k xq[m, k] wq[n, k]) * (sx[m] sw[n]) + bias[n] + r[m, n] )
// The sum is exact: int8 products into 32-bit integers (K <= 65536 leaves a factor of two), so no kernel, split or order changes
// it; the scaling, bias and residual are fp32, rounded once to the output's type.
//   gemm_i8_pair_kernel   CTA pairs (cluster of 2, tcgen05 cta_group::2, kind::i8): tiles of 256 x 256 or 256 x 128, persistent,
//                         accumulator double buffered in tensor memory.  A 128-deep block of codes is 128 bytes per row, the
//                         128-byte swizzle row, and four products of depth 32; copies, ring and barriers are those of the bf16
//                         linear layers (gemm_tc.cu), at twice the operations per byte.
//   gemm_i8_split_kernel  few tiles: one 128 x 64 tile per cluster of 1-8 CTAs that share the contraction and add their integer
//                         sums through distributed shared memory.
//   gemm_i8_rows_kernel   up to 4 tokens: a pass over the weight in plain vector loads and dp4a, a warp per few channels.
//   gemm_i8_simt_kernel   codes whose rows do not start on 16-byte boundaries (copies cannot take them).
// Bounded by the tensor cores from some hundred tokens on (8192 x 4096 -> 11008 bf16 221 us, 3.34 POP/s: the chip's measured bf16 rate
// times two is 3.25), by the weight's one read below (1 x 4096 -> 11008 9.8 us; the read takes 6.9), by launch and ramp for small ones.
// Every wait on an mbarrier is bounded; when it expires the kernel records a code in `status` and returns.
#include "host_common.h"
#include "launch.cuh"
#include "tc_common.cuh"

namespace sl {
namespace {

using namespace tc;

constexpr int NUM_THREADS = 320;
constexpr int KB = 128;                    // codes per block of the contraction: one swizzle row
constexpr int TILE_BYTES = BM * KB;        // 128 rows

struct I8Params {
  int M, N, num_kb;
  int tiles_m, tiles_n;
  int x_rows;                              // rows of x that a copy brings: 128, or as many (of 8) as there are
  const float* sx; const float* sw;        // sw, bias, R may be null
  const void* bias; const void* R; void* Y;
  int* status;
};

// kind::i8 instruction descriptor: 32-bit integer accumulator, signed x signed, both operands K-major, no saturation
__host__ __device__ constexpr uint32_t make_idesc_i8(int m, int n) {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <int CG> __device__ __forceinline__ void mma_i8(uint32_t d_tmem, uint32_t alo, uint32_t blo, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CG == 1)
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(alo), "r"(blo), "r"(DESC_HI), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(alo), "r"(blo), "r"(DESC_HI), "r"(idesc), "r"(accumulate) : "memory");
}
// the four products of one block; advancing 32 codes along K inside the swizzled row is +2 in descriptor units
template <int CG> __device__ __forceinline__ void mma_block(uint32_t d_tmem, uint32_t alo, uint32_t blo, uint32_t idesc, bool first) {
  mma_i8<CG>(d_tmem, alo, blo, idesc, first ? 0u : 1u);
  mma_i8<CG>(d_tmem, alo + 2, blo + 2, idesc, 1u);
  mma_i8<CG>(d_tmem, alo + 4, blo + 4, idesc, 1u);
  mma_i8<CG>(d_tmem, alo + 6, blo + 6, idesc, 1u);
}

__device__ __forceinline__ void lds4(float* v, uint32_t addr) {
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void sts1(uint32_t addr, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
__device__ __forceinline__ float lds1(uint32_t addr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// Channel scale and bias of column n + lane (1 and 0 where there is none, 0 past the last column).
template <typename TO> __device__ __forceinline__ void load_channel(const I8Params& p, int n, int lane, float& sw, float& b) {
  const int c = n + lane;
  sw = c < p.N ? (p.sw ? __ldg(p.sw + c) : 1.0f) : 0.f;
  b = c < p.N && p.bias ? to_f<TO>(reinterpret_cast<const TO*>(p.bias)[c]) : 0.f;
}

// The residual's part of a chunk, requested before the accumulators are awaited.  VEC: this thread's row, 16 bytes at a time; else
// this thread's column.
template <typename TO, bool VEC> struct Residual {
  uint4 v[VEC ? 4 : 1];
  TO s[VEC ? 1 : 32];
  __device__ __forceinline__ void load(const I8Params& p, int m_warp0, int n, int lane) {
    if (!p.R) return;
    const TO* r = reinterpret_cast<const TO*>(p.R);
    if constexpr (VEC) {
      const bool in = m_warp0 + lane < p.M;
      const uint4* row = reinterpret_cast<const uint4*>(r + (size_t)(m_warp0 + lane) * p.N + n);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = in && n + 8 * j < p.N ? __ldcs(row + j) : make_uint4(0u, 0u, 0u, 0u);
    } else {
      const TO* col = r + (size_t)m_warp0 * p.N + n + lane;
#pragma unroll
      for (int q = 0; q < 32; ++q) s[q] = n + lane < p.N && m_warp0 + q < p.M ? col[(size_t)q * p.N] : from_f<TO>(0.f);
    }
  }
  // VEC: from a chunk that a copy has left in shared memory in the layout of stage_and_store
  __device__ __forceinline__ void take(uint32_t rbuf, int lane) {
    const uint32_t row = rbuf + (uint32_t)lane * 64u, sw = ((uint32_t)lane >> 1) & 3u;
#pragma unroll
    for (uint32_t j = 0; j < sizeof(v) / 16; ++j)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[j].x), "=r"(v[j].y), "=r"(v[j].z), "=r"(v[j].w) : "r"(row + ((j ^ sw) << 4)) : "memory");
  }
};

// One 32-row x 32-column chunk of accumulators (acc: this thread's row, columns [n, n + 32)) to the output.  `stage`: 4 KB of this
// warp.  Channel scales and biases arrive one per lane, requested a chunk ahead, and go round through shared memory (read from
// global memory by every lane, where a chunk needs them, they made the epilogue the longer half of the kernel: 32768 x 1024 ->
// 4096 128 us).  VEC: output and residual rows on 16-byte boundaries, bf16: staged like the bf16 layers' chunks and stored by TMA.
template <typename TO>
__device__ __forceinline__ void chunk_vec(const I8Params& p, const uint32_t* acc, float sx, float sw_lane, float b_lane, const Residual<TO, true>& res,
                                          int m_warp0, int n, int lane, uint32_t stage, int& buf, const CUtensorMap* mapY) {
  const uint32_t sbuf = stage + (uint32_t)buf * 2048u;
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");       // the store that last read this buffer
  __syncwarp();
  sts1(sbuf + 4u * lane, sw_lane);
  sts1(sbuf + 128u + 4u * lane, b_lane);
  __syncwarp();
  uint32_t packed[16];
  const uint64_t sx2 = pack2(sx, sx);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float w[4], b[4];
    lds4(w, sbuf + 16u * j);
    lds4(b, sbuf + 128u + 16u * j);
    const uint32_t rw[2] = {j & 1 ? res.v[j / 2].z : res.v[j / 2].x, j & 1 ? res.v[j / 2].w : res.v[j / 2].y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint64_t a2 = pack2(__int2float_rn((int)acc[4 * j + 2 * i]), __int2float_rn((int)acc[4 * j + 2 * i + 1]));
      uint64_t v = fma2(a2, mul2(sx2, pack2(w[2 * i], w[2 * i + 1])), pack2(b[2 * i], b[2 * i + 1]));
      if (p.R) v = add2(v, bf16x2_to_f32x2(rw[i]));
      float y0, y1;
      unpack2(v, y0, y1);
      const __nv_bfloat162 y2 = __floats2bfloat162_rn(y0, y1);
      packed[2 * j + i] = *reinterpret_cast<const uint32_t*>(&y2);
    }
  }
  __syncwarp();
  stage_and_store(sbuf, mapY, packed, lane, n, m_warp0);         // clipped at row M and column N
  buf ^= 1;
}

// Any N, alignment and type: channel scales and biases arrive one per lane and go round through shared memory, and each row of the
// chunk leaves as one coalesced store of the warp.
template <typename TO>
__device__ __forceinline__ void chunk_any(const I8Params& p, const uint32_t* acc, float sx, float sw_lane, float b_lane, const Residual<TO, false>& res,
                                          int m_warp0, int n, int lane, uint32_t sbuf) {
  sts1(sbuf + 4u * lane, sw_lane);
  sts1(sbuf + 128u + 4u * lane, b_lane);
  __syncwarp();
  float v[32];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float w[4], b[4];
    lds4(w, sbuf + 16u * j);
    lds4(b, sbuf + 128u + 16u * j);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[4 * j + i] = fmaf(__int2float_rn((int)acc[4 * j + i]), sx * w[i], b[i]);
  }
  __syncwarp();
  // word (row, column) at column ^ row of its row: no two lanes of a store or a load share a bank
#pragma unroll
  for (int i = 0; i < 32; ++i) sts1(sbuf + (uint32_t)lane * 128u + (uint32_t)((i ^ lane) << 2), v[i]);
  __syncwarp();
  if (n + lane < p.N) {
    TO* y = reinterpret_cast<TO*>(p.Y) + (size_t)m_warp0 * p.N + n + lane;
#pragma unroll
    for (int q = 0; q < 32; ++q) {
      float t = lds1(sbuf + (uint32_t)q * 128u + (uint32_t)((lane ^ q) << 2));
      if (p.R) t += to_f<TO>(res.s[q]);
      if (m_warp0 + q < p.M) y[(size_t)q * p.N] = from_f<TO>(t);
    }
  }
  __syncwarp();
}

// ------------------------------------------------------------------------------------------
// CTA pairs
// ------------------------------------------------------------------------------------------
// RES: a residual in VEC form.  Every epilogue warp has its 32 x 32 chunks brought into shared memory two ahead of their use: read row
// by row from memory 32768 x 1024 -> 4096 took 191 us instead of 164; the product alone takes 108.
template <int BN_, bool RES> struct PairCfg {
  static constexpr int BN = BN_;
  static constexpr int A_BYTES = TILE_BYTES;             // this CTA's 128 rows of x
  static constexpr int B_BYTES = (BN / 2) * KB;          // this CTA's half of the weight tile
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int STAGES = (BN == 256 ? 6 : 8) - (RES ? BN == 256 ? 1 : 2 : 0);
  static constexpr int R_BYTES = RES ? 8 * 2 * 2048 : 0;
  static constexpr int TMEM_COLS = 2 * BN;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + EPI_STAGE_BYTES + R_BYTES + 1024 + 512;
  static_assert(SMEM_BYTES <= 232448, "");
  static constexpr uint32_t IDESC = make_idesc_i8(2 * BM, BN);
};

template <typename TO, bool VEC, bool RES, int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(NUM_THREADS, 1)
gemm_i8_pair_kernel(const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapW, const __grid_constant__ CUtensorMap mapY,
                    const __grid_constant__ CUtensorMap mapR, I8Params p) {
  static_assert(VEC || !RES, "");
  using C = PairCfg<BN, RES>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - raw);
  const uint32_t epi_base = base + C::STAGES * C::STAGE_BYTES;
  const uint32_t r_base = epi_base + EPI_STAGE_BYTES;
  const uint32_t bar_base = r_base + C::R_BYTES;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };                         // used in the leader
  auto empty_bar = [&](int s) { return bar_base + 8u * (C::STAGES + s); };          // one per CTA
  auto tfull_bar = [&](int a) { return bar_base + 8u * (2 * C::STAGES + a); };      // one per CTA
  auto tempty_bar = [&](int a) { return bar_base + 8u * (2 * C::STAGES + 2 + a); }; // used in the leader
  auto r_bar = [&](int w, int b) { return bar_base + 8u * (2 * C::STAGES + 4 + 2 * w + b); };     // RES: of epilogue warp w
  uint8_t* tail = base_ptr + C::STAGES * C::STAGE_BYTES + EPI_STAGE_BYTES + C::R_BYTES + 8 * (2 * C::STAGES + 4 + 16);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(tail);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 8);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();           // 0 = leader of the pair
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 16); }
    if (RES) for (int i = 0; i < 16; ++i) mbar_init(r_bar(i >> 1, i & 1), 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_slot)), "r"((uint32_t)C::TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                // the partner's barriers are initialised too
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  overlap_sync();

  const int num_tiles = p.tiles_m * p.tiles_n;       // tiles of 256 x BN

  if (warp == 0) {
    // ---------------- TMA producer (both CTAs) ----------------
    const bool leader = elect_one();
    int stage = 0; uint32_t phase = 0;
    bool ok = true;
    for (int tile = pair; tile < num_tiles && ok; tile += npairs) {
      int tm, tn; tile_coords(tile, p.tiles_m, p.tiles_n, tm, tn);
      const int m0 = tm * 2 * BM + (int)rank * BM, n0 = tn * BN + (int)rank * (BN / 2);
      for (int kb = 0; kb < p.num_kb; ++kb) {
        if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, abort_flag, p.status, 61)) { ok = false; break; }
        const uint32_t leader_full = map_to_cta(full_bar(stage), 0);
        const uint32_t sa = base + stage * C::STAGE_BYTES, sb = sa + C::A_BYTES;
        if (leader) {
          // the first CTA's barrier collects the bytes of both CTAs' copies
          if (rank == 0) mbar_expect_tx(full_bar(stage), 2 * C::STAGE_BYTES);
          tma_load_2d_pair(sa, &mapX, leader_full, kb * KB, m0);
          tma_load_2d_pair(sb, &mapW, leader_full, kb * KB, n0);
        }
        __syncwarp();
        if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer (first CTA of the pair only) ----------------
    if (rank == 0) {
      const bool leader = elect_one();
      int stage = 0; uint32_t phase = 0;
      int as = 0; uint32_t aphase = 0;
      bool ok = true;
      const uint32_t a_lo0 = desc_lo(base);
      for (int tile = pair; tile < num_tiles && ok; tile += npairs) {
        if (!mbar_wait_warp(tempty_bar(as), aphase ^ 1u, abort_flag, p.status, 62)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + (uint32_t)(as * BN);
        for (int kb = 0; kb < p.num_kb; ++kb) {
          if (!mbar_wait_warp(full_bar(stage), phase, abort_flag, p.status, 63)) { ok = false; break; }
          const uint32_t alo = a_lo0 + (uint32_t)stage * (uint32_t)(C::STAGE_BYTES >> 4);
          const uint32_t blo = alo + (uint32_t)(C::A_BYTES >> 4);
          if (leader) {
            mma_block<2>(d_tmem, alo, blo, C::IDESC, kb == 0);
            tc_commit_pair(empty_bar(stage), 3);     // frees the stage in both CTAs
          }
          __syncwarp();
          if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        if (leader) tc_commit_pair(tfull_bar(as), 3);
        __syncwarp();
        if (++as == 2) { as = 0; aphase ^= 1u; }
      }
    }
  } else {
    // ---------------- epilogue (both CTAs, own 128 rows) ----------------
    const int q = warp & 3;
    const int half = (warp - 2) >> 2;
    const int c_begin = half * (BN / 2), c_end = c_begin + BN / 2;
    const int ew = warp - 2;
    int as = 0; uint32_t aphase = 0;
    const uint32_t stage = epi_base + (uint32_t)ew * 4096u, rbuf = r_base + (uint32_t)ew * 4096u;
    int buf = 0;
    bool ok = true;
    auto rows_of = [&](int tile, int& n0) {
      int tm, tn; tile_coords(tile, p.tiles_m, p.tiles_n, tm, tn);
      n0 = tn * BN;
      return tm * 2 * BM + (int)rank * BM + q * 32;
    };
    // RES: the chunks of this warp in the order of their use; `asked` counts those under way or done, `used` those done
    int r_tile = pair, r_c = c_begin, asked = 0, used = 0;
    auto ask = [&]() {
      while (r_tile < num_tiles) {
        int n0;
        const int m = rows_of(r_tile, n0), n = n0 + r_c;
        if (m >= p.M || n >= p.N) { r_tile += npairs; r_c = c_begin; continue; }      // what is left of this tile is outside
        if (lane == 0) {
          mbar_expect_tx(r_bar(ew, asked & 1), 2048);
          tma_load_2d(rbuf + (uint32_t)(asked & 1) * 2048u, &mapR, r_bar(ew, asked & 1), n, m);
        }
        ++asked;
        r_c += 32;
        if (r_c >= c_end) { r_tile += npairs; r_c = c_begin; }
        return;
      }
    };
    if (RES) { ask(); ask(); }
    for (int tile = pair; tile < num_tiles && ok; tile += npairs) {
      int n0;
      const int m_warp0 = rows_of(tile, n0);
      // in flight while the accumulator is awaited
      const float sx = m_warp0 + lane < p.M ? __ldg(p.sx + m_warp0 + lane) : 0.f;
      float sw = 0.f, b = 0.f;
      load_channel<TO>(p, n0 + c_begin, lane, sw, b);
      if (!mbar_wait(tfull_bar(as), aphase, abort_flag, p.status, 64)) { ok = false; break; }
      tc_fence_after();
      const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(as * BN);
      if (m_warp0 < p.M) {
        if constexpr (VEC) {
          // accumulators one chunk ahead of their use
          uint32_t acc[2][32];
          tc_ld32(t_row + (uint32_t)c_begin, reinterpret_cast<float*>(acc[0]));
#pragma unroll
          for (int k = 0; k < BN / 64; ++k) {
            const int c = c_begin + 32 * k, n = n0 + c;
            if (n >= p.N || !ok) break;
            tc_wait_ld();
            float sw_next = 0.f, b_next = 0.f;
            if (k + 1 < BN / 64) {
              tc_ld32(t_row + (uint32_t)(c + 32), reinterpret_cast<float*>(acc[(k + 1) & 1]));
              load_channel<TO>(p, n + 32, lane, sw_next, b_next);
            }
            Residual<TO, true> res;
            if (RES) {
              if (!mbar_wait(r_bar(ew, used & 1), (uint32_t)(used >> 1) & 1u, abort_flag, p.status, 65)) { ok = false; break; }
              res.take(rbuf + (uint32_t)(used & 1) * 2048u, lane);
              ++used;
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // read before a copy writes the buffer again
              __syncwarp();
              ask();
            }
            chunk_vec<TO>(p, acc[k & 1], sx, sw, b, res, m_warp0, n, lane, stage, buf, &mapY);
            sw = sw_next; b = b_next;
          }
          tc_wait_ld();                                // also where the last columns were past N
        } else {
#pragma unroll 1
          for (int c = c_begin; c < c_end; c += 32) {
            const int n = n0 + c;
            if (n >= p.N) break;
            Residual<TO, false> res;
            res.load(p, m_warp0, n, lane);
            float sw_next = 0.f, b_next = 0.f;
            if (c + 32 < c_end) load_channel<TO>(p, n + 32, lane, sw_next, b_next);
            uint32_t acc[32];
            tc_ld32(t_row + (uint32_t)c, reinterpret_cast<float*>(acc));
            tc_wait_ld();
            chunk_any<TO>(p, acc, sx, sw, b, res, m_warp0, n, lane, stage);
            sw = sw_next; b = b_next;
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_to_cta(tempty_bar(as), 0));   // 16 arrivals free the stage
      if (++as == 2) { as = 0; aphase ^= 1u; }
    }
    epilogue_drain(lane);
  }

  // ---------------- teardown ----------------
  __syncwarp();
  if (*abort_flag) {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                // neither CTA leaves while its partner may still touch it
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::TMEM_COLS) : "memory");
  }
}

// ------------------------------------------------------------------------------------------
// few tiles: one 128 x 64 tile per cluster, the contraction split over its S CTAs
// ------------------------------------------------------------------------------------------
// Every CTA contracts its range of blocks into its own tensor memory; piece (warp) u of the tile, 32 x 32 accumulators, is added
// up by CTA u % S from what the others sent it through distributed shared memory.
template <int S> struct SplitCfg {
  static constexpr int BN = 64;
  static constexpr int A_BYTES = TILE_BYTES;
  static constexpr int B_BYTES = BN * KB;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int STAGES = 7;
  static constexpr int RECV_BYTES = (8 / S) * (S - 1) * 4096;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + RECV_BYTES + 1024 + 256;
  static constexpr uint32_t IDESC = make_idesc_i8(BM, BN);
  static_assert(STAGES * STAGE_BYTES >= EPI_STAGE_BYTES && 8 % S == 0 && SMEM_BYTES <= 232448, "");
};

template <typename TO, bool VEC, int S>
__global__ void __launch_bounds__(NUM_THREADS, 1)
gemm_i8_split_kernel(const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapW, const __grid_constant__ CUtensorMap mapY,
                     I8Params p) {
  using C = SplitCfg<S>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - raw);
  const uint32_t recv_base = base + C::STAGES * C::STAGE_BYTES;
  const uint32_t bar_base = recv_base + C::RECV_BYTES;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (C::STAGES + s); };
  const uint32_t tfull_bar = bar_base + 8u * (2 * C::STAGES);
  uint8_t* tail = base_ptr + C::STAGES * C::STAGE_BYTES + C::RECV_BYTES + 8 * (2 * C::STAGES + 1);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(tail);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 8);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = S > 1 ? (int)cluster_ctarank() : 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    mbar_init(tfull_bar, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_slot)), "r"((uint32_t)C::BN) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (S > 1) cluster_arrive();                       // awaited before the first store to another CTA
  const uint32_t tmem_base = *tmem_slot;
  overlap_sync();

  const int kb0 = (int)((long long)p.num_kb * rank / S), kb1 = (int)((long long)p.num_kb * (rank + 1) / S);   // never empty: num_kb >= S
  int tm, tn;
  tile_coords((int)blockIdx.x / S, p.tiles_m, p.tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * C::BN;

  if (warp == 0) {
    const bool leader = elect_one();
    int stage = 0; uint32_t phase = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, abort_flag, p.status, 71)) break;
      const uint32_t sa = base + stage * C::STAGE_BYTES, sb = sa + C::A_BYTES;
      if (leader) {
        // rows of the x tile past the last token stay as they are: their accumulators are not stored
        mbar_expect_tx(full_bar(stage), C::B_BYTES + p.x_rows * KB);
        tma_load_2d(sb, &mapW, full_bar(stage), kb * KB, n0);
        tma_load_2d(sa, &mapX, full_bar(stage), kb * KB, m0);
      }
      __syncwarp();
      if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
    }
  } else if (warp == 1) {
    const bool leader = elect_one();
    int stage = 0; uint32_t phase = 0;
    bool ok = true;
    const uint32_t a_lo0 = desc_lo(base);
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!mbar_wait_warp(full_bar(stage), phase, abort_flag, p.status, 73)) { ok = false; break; }
      const uint32_t alo = a_lo0 + (uint32_t)stage * (uint32_t)(C::STAGE_BYTES >> 4);
      if (leader) {
        mma_block<1>(tmem_base, alo, alo + (uint32_t)(C::A_BYTES >> 4), C::IDESC, kb == kb0);
        tc_commit(empty_bar(stage));
      }
      __syncwarp();
      if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
    }
    if (ok && leader) tc_commit(tfull_bar);
  }
  __syncwarp();

  // ---------------- epilogue ----------------
  const int ew = warp - 2;                           // epilogue warp 0..7
  const int q = warp & 3, half = ew >> 2;
  const int m_warp0 = m0 + q * 32, n = n0 + 32 * half;
  const int u = half * 4 + q, owner = u % S;         // this warp's piece and the CTA that adds it up
  const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(32 * half);
  const bool live = warp >= 2 && m_warp0 < p.M && n < p.N;
  uint32_t acc[32];
  float sx = 0.f, sw = 0.f, b = 0.f;
  Residual<TO, VEC> res;
  bool ok = false;
  if (warp >= 2) {
    if (live && owner == rank) {
      res.load(p, m_warp0, n, lane);
      sx = m_warp0 + lane < p.M ? __ldg(p.sx + m_warp0 + lane) : 0.f;
      load_channel<TO>(p, n, lane, sw, b);
    }
    ok = mbar_wait(tfull_bar, 0u, abort_flag, p.status, 74);
    tc_fence_after();
    if (live && ok) {
      tc_ld32(t_row, reinterpret_cast<float*>(acc));
      tc_wait_ld();
    }
  }
  if constexpr (S > 1) {
    __syncwarp();
    cluster_wait();                                  // every CTA of the cluster runs: its shared memory exists
    if (live && ok && owner != rank) {
      const int sender = rank < owner ? rank : rank - 1;
      const uint32_t dst = map_to_cta(recv_base + (uint32_t)(((u / S) * (S - 1) + sender) * 4096 + lane * 16), (uint32_t)owner);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (uint32_t)(i * 512)), "r"(acc[4 * i]), "r"(acc[4 * i + 1]),
                     "r"(acc[4 * i + 2]), "r"(acc[4 * i + 3]) : "memory");
    }
    __syncwarp();
    cluster_sync_all();
  }
  if (live && ok && owner == rank) {
    if constexpr (S > 1) {
#pragma unroll
      for (int s = 0; s < S - 1; ++s) {
        const uint32_t src = recv_base + (uint32_t)(((u / S) * (S - 1) + s) * 4096 + lane * 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t x0, x1, x2, x3;
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x0), "=r"(x1), "=r"(x2), "=r"(x3) : "r"(src + (uint32_t)(i * 512)) : "memory");
          acc[4 * i] += x0; acc[4 * i + 1] += x1; acc[4 * i + 2] += x2; acc[4 * i + 3] += x3;
        }
      }
    }
    // the output staging takes the operand ring, which is idle: every product has completed
    const uint32_t stage = base + (uint32_t)ew * 4096u;
    int buf = 0;
    if constexpr (VEC) chunk_vec<TO>(p, acc, sx, sw, b, res, m_warp0, n, lane, stage, buf, &mapY);
    else chunk_any<TO>(p, acc, sx, sw, b, res, m_warp0, n, lane, stage);
  }
  if (warp >= 2) epilogue_drain(lane);

  __syncwarp();
  if (*abort_flag) {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::BN) : "memory");
  }
}

// ------------------------------------------------------------------------------------------
// few tokens
// ------------------------------------------------------------------------------------------
// The time of a weight read once: a warp takes C channels (rows of W) and all MR tokens, 512 bytes of a row per step, four codes
// per dp4a; x comes from L1, C times less often than W from memory.
template <typename TO, int MR, int C>
__global__ void __launch_bounds__(256)
gemm_i8_rows_kernel(const int8_t* __restrict__ x, int64_t ldx, const int8_t* __restrict__ w, int64_t ldw, int K, I8Params p) {
  overlap_sync();
  const int lane = threadIdx.x & 31, n0 = ((int)blockIdx.x * 8 + (threadIdx.x >> 5)) * C;
  if (n0 >= p.N) return;
  int acc[MR][C];
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int c = 0; c < C; ++c) acc[m][c] = 0;
  auto row = [&](int c) { return w + (int64_t)min(n0 + c, p.N - 1) * ldw; };
  auto token = [&](int m) { return x + (int64_t)min(m, p.M - 1) * ldx; };
  auto add = [&](const uint4 (&b)[C], const uint4& a, int m) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      acc[m][c] = __dp4a((int)a.x, (int)b[c].x, acc[m][c]);
      acc[m][c] = __dp4a((int)a.y, (int)b[c].y, acc[m][c]);
      acc[m][c] = __dp4a((int)a.z, (int)b[c].z, acc[m][c]);
      acc[m][c] = __dp4a((int)a.w, (int)b[c].w, acc[m][c]);
    }
  };
  const int whole = K & ~15;
  constexpr int U = 8 / C;                 // steps whose weights are under way together
  for (int k0 = lane * 16; k0 < whole; k0 += 512 * U) {
    uint4 b[U][C];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + 512 * u < whole) {
#pragma unroll
        for (int c = 0; c < C; ++c) b[u][c] = __ldcs(reinterpret_cast<const uint4*>(row(c) + k0 + 512 * u));
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + 512 * u < whole) {
#pragma unroll
        for (int m = 0; m < MR; ++m) add(b[u], *reinterpret_cast<const uint4*>(token(m) + k0 + 512 * u), m);
      }
  }
  if (lane < K - whole) {                  // the last codes one by one: what lies behind a row does not count
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
      for (int c = 0; c < C; ++c) acc[m][c] += (int)token(m)[whole + lane] * (int)row(c)[whole + lane];
  }
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int sum = __reduce_add_sync(0xffffffffu, acc[m][c]), n = n0 + c;
      if (lane != (m * C + c) % 32 || m >= p.M || n >= p.N) continue;
      const size_t at = (size_t)m * p.N + n;
      float v = fmaf(__int2float_rn(sum), p.sx[m] * (p.sw ? p.sw[n] : 1.0f), p.bias ? to_f<TO>(reinterpret_cast<const TO*>(p.bias)[n]) : 0.f);
      if (p.R) v += to_f<TO>(reinterpret_cast<const TO*>(p.R)[at]);
      reinterpret_cast<TO*>(p.Y)[at] = from_f<TO>(v);
    }
}

// ------------------------------------------------------------------------------------------
// any alignment: 64 x 64 tiles, four codes per instruction (dp4a) from shared memory
// ------------------------------------------------------------------------------------------
template <typename TO>
__global__ void __launch_bounds__(256)
gemm_i8_simt_kernel(const int8_t* __restrict__ x, int64_t ldx, const int8_t* __restrict__ w, int64_t ldw, int K, I8Params p) {   // tiles_m x tiles_n blocks
  overlap_sync();
  constexpr int T = 64, D = 64;
  __shared__ __align__(16) int8_t xs[T][D + 4], ws[T][D + 4];
  const int m0 = (int)(blockIdx.x / p.tiles_n) * T, n0 = (int)(blockIdx.x % p.tiles_n) * T;
  const int tm = threadIdx.x >> 4, tn = threadIdx.x & 15;      // rows tm + 16 i, columns tn + 16 j
  int acc[4][4] = {};
  for (int k0 = 0; k0 < K; k0 += D) {
    for (int e = threadIdx.x; e < T * D; e += 256) {
      const int r = e / D, c = e % D;
      xs[r][c] = m0 + r < p.M && k0 + c < K ? x[(int64_t)(m0 + r) * ldx + k0 + c] : (int8_t)0;
      ws[r][c] = n0 + r < p.N && k0 + c < K ? w[(int64_t)(n0 + r) * ldw + k0 + c] : (int8_t)0;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < D; c += 4) {
      int a[4], b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = *reinterpret_cast<const int*>(&xs[tm + 16 * i][c]);
        b[i] = *reinterpret_cast<const int*>(&ws[tn + 16 * i][c]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(a[i], b[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + tm + 16 * i;
    if (m >= p.M) continue;
    const float sx = p.sx[m];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + tn + 16 * j;
      if (n >= p.N) continue;
      const size_t at = (size_t)m * p.N + n;
      float v = fmaf(__int2float_rn(acc[i][j]), sx * (p.sw ? p.sw[n] : 1.0f), p.bias ? to_f<TO>(reinterpret_cast<const TO*>(p.bias)[n]) : 0.f);
      if (p.R) v += to_f<TO>(reinterpret_cast<const TO*>(p.R)[at]);
      reinterpret_cast<TO*>(p.Y)[at] = from_f<TO>(v);
    }
  }
}

// ---- host side -----------------------------------------------------------------------------
int g_pairs[MAX_DEVICES] = {};                   // CTA pairs that can be resident at once
int g_clusters[MAX_DEVICES][3] = {};             // clusters of 2, 4 and 8 CTAs
PerDeviceOnce g_once;

bool map_codes(CUtensorMap* m, const void* ptr, int64_t rows, int64_t cols, int64_t ld, uint32_t box_rows) {
  return cached_map_2d_u8(m, ptr, rows, cols, ld, KB, box_rows, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

// output and residual: chunks of 32 x 32 in the epilogue's staging layout
bool map_tile(CUtensorMap* m, const void* ptr, int64_t rows, int64_t cols, CUtensorMapL2promotion promo = CU_TENSOR_MAP_L2_PROMOTION_NONE) {
  return cached_map_2d(m, ptr, rows, cols, cols, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B, promo);
}

template <typename K> int clusters_resident(K kernel, int size, int smem) {
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(size); cfg.blockDim = dim3(NUM_THREADS); cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = size; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
  cfg.attrs = &at; cfg.numAttrs = 1;
  int n = 0;
  return cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess ? n : 0;
}

template <typename K> cudaError_t allow_smem(K kernel, PerDeviceOnce& once, int smem) {
  const int dev = current_device();
  if (!once.needed(dev)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess) once.done(dev);
  return e;
}

template <typename TO, bool VEC, bool RES, int BN> cudaError_t launch_pair_t(const I8Args& a, I8Params p, CUtensorMap mX, CUtensorMap mY, cudaStream_t st) {
  using C = PairCfg<BN, RES>;
  static PerDeviceOnce once;
  const cudaError_t e = allow_smem(gemm_i8_pair_kernel<TO, VEC, RES, BN>, once, C::SMEM_BYTES);
  if (e != cudaSuccess) return e;
  CUtensorMap mW, mR = mY;
  if (!map_codes(&mW, a.W, a.N, a.K, a.ldw, BN / 2)) return cudaErrorInvalidValue;
  // (a chunk's rows are 64 bytes: the next chunk's come into L2 with them)
  if (RES && !map_tile(&mR, a.R, a.M, a.N, CU_TENSOR_MAP_L2_PROMOTION_L2_256B)) return cudaErrorInvalidValue;
  p.tiles_m = (a.M + 2 * BM - 1) / (2 * BM); p.tiles_n = (a.N + BN - 1) / BN;
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  const int most = g_pairs[current_device()], pairs = tiles < most ? (int)tiles : most;
  return launch_overlapped(gemm_i8_pair_kernel<TO, VEC, RES, BN>, dim3(2 * pairs), dim3(NUM_THREADS), C::SMEM_BYTES, st, mX, mW, mY, mR, p);
}
template <typename TO, bool VEC, int BN> cudaError_t launch_pair(const I8Args& a, I8Params p, CUtensorMap mX, CUtensorMap mY, cudaStream_t st) {
  if constexpr (VEC)
    if (a.R) return launch_pair_t<TO, VEC, true, BN>(a, p, mX, mY, st);
  return launch_pair_t<TO, VEC, false, BN>(a, p, mX, mY, st);
}

template <typename TO, bool VEC, int S> cudaError_t launch_split(const I8Args& a, I8Params p, CUtensorMap mX, CUtensorMap mY, cudaStream_t st) {
  using C = SplitCfg<S>;
  static PerDeviceOnce once;
  const cudaError_t e = allow_smem(gemm_i8_split_kernel<TO, VEC, S>, once, C::SMEM_BYTES);
  if (e != cudaSuccess) return e;
  CUtensorMap mW;
  if (!map_codes(&mW, a.W, a.N, a.K, a.ldw, C::BN)) return cudaErrorInvalidValue;
  p.tiles_m = (a.M + BM - 1) / BM; p.tiles_n = (a.N + C::BN - 1) / C::BN;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.tiles_m * p.tiles_n * S)); cfg.blockDim = dim3(NUM_THREADS);
  cfg.dynamicSmemBytes = C::SMEM_BYTES; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = S; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = chain_attribute(at, 1);
  return cudaLaunchKernelEx(&cfg, gemm_i8_split_kernel<TO, VEC, S>, mX, mW, mY, p);
}

// The kernel with the least estimated time (ns): a fixed part, the time of a 128-deep block, rounds over the chip.  Each kernel was timed
// on 19 shapes (8 to 8192 tokens, 768 to 65536 deep), without and with a residual and with fp32 output: the one picked took at most 9 % more
// than the fastest.  Examples, us (pairs 256 and 128 wide, clusters of 1, 2, 4, 8): 16 x 4096 -> 4096 -, -, 9.4, 7.2, 11.1, 20.4;
// 256 x 4096 -> 4096 15.0, 10.0, 9.9, 14.4, 23.6, 46.0; 300 x 65536 -> 256 144, 79, 95, 49, 27, 16.7; 4096 x 4096 -> 11008 116, 133, 364 ...
// The epilogue is not in the estimate: with a residual 4096 x 1024 -> 1024 takes 10.5 in the 256-wide tiles it gets, 9.8 in the others.
enum Pick { PICK_PAIR256, PICK_PAIR128, PICK_SPLIT1, PICK_SPLIT2, PICK_SPLIT4, PICK_SPLIT8 };
Pick pick(const I8Args& a) {
  const int dev = current_device();
  const int64_t sms = num_sms(), kb = (a.K + KB - 1) / KB;
  auto cdiv = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
  Pick best = PICK_SPLIT1;
  int64_t best_ns = INT64_MAX;
  auto offer = [&](Pick k, int64_t ns) { if (ns < best_ns) { best_ns = ns; best = k; } };
  auto split = [&](Pick k, int s, int64_t slots, int64_t fixed) {
    if (slots < 1 || kb < 2 * s) { if (s > 1) return; }
    const int64_t rounds = cdiv(cdiv(a.M, BM) * cdiv(a.N, 64), slots < 1 ? sms : slots);
    offer(k, fixed + rounds * cdiv(kb, s) * 190 + (rounds - 1) * 3000);
  };
  split(PICK_SPLIT1, 1, sms, 3600);
  split(PICK_SPLIT2, 2, g_clusters[dev][0], 4700);
  split(PICK_SPLIT4, 4, g_clusters[dev][1], 5000);
  split(PICK_SPLIT8, 8, g_clusters[dev][2], 5500);
  if (g_pairs[dev] > 0 && a.M > BM) {
    offer(PICK_PAIR256, 5500 + cdiv(cdiv(a.M, 2 * BM) * cdiv(a.N, 256), g_pairs[dev]) * kb * 275);
    offer(PICK_PAIR128, 4500 + cdiv(cdiv(a.M, 2 * BM) * cdiv(a.N, 128), g_pairs[dev]) * kb * 200);
  }
  return best;
}

template <typename TO, bool VEC> cudaError_t launch_tc(const I8Args& a, I8Params p, cudaStream_t st) {
  CUtensorMap mX, mY;
  const Pick k = pick(a);
  const bool split = k != PICK_PAIR256 && k != PICK_PAIR128;
  p.x_rows = split && a.M < BM ? (a.M + 7) / 8 * 8 : BM;
  if (!map_codes(&mX, a.X, a.M, a.K, a.ldx, (uint32_t)p.x_rows)) return cudaErrorInvalidValue;
  mY = mX;
  if (VEC && !map_tile(&mY, a.Y, a.M, a.N)) return cudaErrorInvalidValue;
  switch (k) {
    case PICK_PAIR256: return launch_pair<TO, VEC, 256>(a, p, mX, mY, st);
    case PICK_PAIR128: return launch_pair<TO, VEC, 128>(a, p, mX, mY, st);
    case PICK_SPLIT2: return launch_split<TO, VEC, 2>(a, p, mX, mY, st);
    case PICK_SPLIT4: return launch_split<TO, VEC, 4>(a, p, mX, mY, st);
    case PICK_SPLIT8: return launch_split<TO, VEC, 8>(a, p, mX, mY, st);
    default: return launch_split<TO, VEC, 1>(a, p, mX, mY, st);
  }
}

// Tokens up to which a pass over the weight beats the tensor cores' tiles: 4 of 4096 -> 4096 8.6 us against 8.3, of 768 -> 2304 3.6
// against 4.5; 8 of 4096 -> 4096 14.2 against 8.4.  Channels per warp: 4096 -> 11008, two and four: 1 token 9.8 and 9.7 us, 2 tokens
// 14.7 and 10.6, 4 tokens 21.2 and 14.7; 4096 -> 4096 5.7 and 6.5, 6.7 and 7.5, 9.5 and 9.9 (few warps).  One: 6.2, 8.7.
constexpr int ROWS_MOST = 4, WIDE_ROWS = 8192;
template <typename TO> cudaError_t launch_rows(const I8Args& a, const I8Params& p, cudaStream_t st) {
  auto go = [&](auto kernel, int channels) {
    return launch_overlapped(kernel, dim3((unsigned)((a.N + 8 * channels - 1) / (8 * channels))), dim3(256), 0, st, a.X, a.ldx, a.W, a.ldw, a.K, p);
  };
  if (a.M == 1) return go(gemm_i8_rows_kernel<TO, 1, 2>, 2);
  if (a.N >= WIDE_ROWS) return a.M == 2 ? go(gemm_i8_rows_kernel<TO, 2, 4>, 4) : go(gemm_i8_rows_kernel<TO, 4, 4>, 4);
  return a.M == 2 ? go(gemm_i8_rows_kernel<TO, 2, 2>, 2) : go(gemm_i8_rows_kernel<TO, 4, 2>, 2);
}

bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

int gemm_i8_init() {
  if (!tensor_map_encoder()) return -1;
  const int dev = current_device(), sms = num_sms();
  if (dev < 0 || sms < 1) return -1;
  if (!g_once.needed(dev)) return 0;
  const int pairs = clusters_resident(gemm_i8_pair_kernel<bf16, true, true, 256>, 2, PairCfg<256, true>::SMEM_BYTES);
  g_pairs[dev] = pairs < sms / 2 ? pairs : sms / 2;
  g_clusters[dev][0] = clusters_resident(gemm_i8_split_kernel<bf16, true, 2>, 2, SplitCfg<2>::SMEM_BYTES);
  g_clusters[dev][1] = clusters_resident(gemm_i8_split_kernel<bf16, true, 4>, 4, SplitCfg<4>::SMEM_BYTES);
  g_clusters[dev][2] = clusters_resident(gemm_i8_split_kernel<bf16, true, 8>, 8, SplitCfg<8>::SMEM_BYTES);
  cudaGetLastError();
  g_once.done(dev);
  return 0;
}

cudaError_t gemm_i8(const I8Args& a, int* status, cudaStream_t st) {
  I8Params p = {};
  p.M = a.M; p.N = a.N; p.num_kb = (a.K + KB - 1) / KB;
  p.sx = a.x_scales; p.sw = a.w_scales; p.bias = a.bias; p.R = a.R; p.Y = a.Y; p.status = status;
  if (a.ldx % 16 != 0 || a.ldw % 16 != 0 || !al16(a.X) || !al16(a.W)) {
    p.tiles_m = (a.M + 63) / 64; p.tiles_n = (a.N + 63) / 64;
    const dim3 grid((unsigned)p.tiles_m * (unsigned)p.tiles_n);
    if (a.dtype == DT_BF16) return launch_overlapped(gemm_i8_simt_kernel<bf16>, grid, dim3(256), 0, st, a.X, a.ldx, a.W, a.ldw, a.K, p);
    return launch_overlapped(gemm_i8_simt_kernel<float>, grid, dim3(256), 0, st, a.X, a.ldx, a.W, a.ldw, a.K, p);
  }
  if (a.M <= ROWS_MOST) return a.dtype == DT_BF16 ? launch_rows<bf16>(a, p, st) : launch_rows<float>(a, p, st);
  if (a.dtype != DT_BF16) return launch_tc<float, false>(a, p, st);
  if (a.N % 8 == 0 && al16(a.Y) && al16(a.R)) return launch_tc<bf16, true>(a, p, st);
  return launch_tc<bf16, false>(a, p, st);
}

}  // namespace sl
