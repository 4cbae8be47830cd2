// Stand-alone operator entry points for adapters over frozen weights held in 8 bits: the row codec, the norm with an int8
// output, products of codes, and the loss against a teacher's top logits.  Host code only.
#include <cuda_runtime.h>

#include <cmath>

#include "../../include/splitlora.h"
#include "host_common.h"
#include "kernels.h"
#include "launch.cuh"

using namespace sl;

namespace {
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool dtype_ok(int dt) { return dt == DT_F32 || dt == DT_BF16; }
bool aligned_elem(int dt, const void* p) { return aligned(p, dt == DT_BF16 ? 2 : 4); }
// Where a side of a matrix is indexed in 32 bits: tiles and strides past its end stay inside them.
constexpr int64_t SIDE_MOST = 1 << 30;
bool rows_ok(int64_t M) { return M >= 1 && M <= 2147483647LL; }
int done(cudaError_t e) { return e == cudaSuccess ? SPLITLORA_OK : SPLITLORA_ERR_CUDA; }
}  // namespace

extern "C" {

int splitlora_quantize_rows(int dtype, const void* x, const float* col_scale, int64_t M, int d, int8_t* codes, int64_t ld_codes, float* scales,
                            void* stream) {
  LaunchChain chain;
  if (!dtype_ok(dtype) || !x || !codes || !scales || !rows_ok(M) || d < 1 || d > QUANT_MAX_WIDTH || ld_codes < d) return SPLITLORA_ERR_ARG;
  if (!aligned_elem(dtype, x) || !aligned(col_scale, 4) || !aligned(scales, 4)) return SPLITLORA_ERR_ALIGN;
  return done(quantize_rows(dtype, x, col_scale, M, d, codes, ld_codes, scales, (cudaStream_t)stream));
}

int splitlora_dequantize_rows(int dtype, const int8_t* codes, int64_t ld_codes, const float* scales, int64_t M, int d, void* y, void* stream) {
  LaunchChain chain;
  if (!dtype_ok(dtype) || !y || !codes || !scales || !rows_ok(M) || d < 1 || d > QUANT_MAX_WIDTH || ld_codes < d) return SPLITLORA_ERR_ARG;
  if (!aligned_elem(dtype, y) || !aligned(scales, 4)) return SPLITLORA_ERR_ALIGN;
  return done(dequantize_rows(dtype, codes, ld_codes, scales, M, d, y, (cudaStream_t)stream));
}

int splitlora_rmsnorm_quantize(int dtype, const void* x, const void* residual, const void* g, float eps, int64_t M, int d, void* h, void* y,
                               int8_t* codes, int64_t ld_codes, float* scales, void* stream) {
  LaunchChain chain;
  if (!dtype_ok(dtype) || !x || !g || !codes || !scales || !rows_ok(M) || d < 1 || d > ROWS_MAX_WIDTH || ld_codes < d || !(eps >= 0.f) || std::isinf(eps))
    return SPLITLORA_ERR_ARG;
  for (const void* p : {x, residual, g, (const void*)h, (const void*)y})
    if (!aligned_elem(dtype, p)) return SPLITLORA_ERR_ALIGN;
  if (!aligned(scales, 4)) return SPLITLORA_ERR_ALIGN;
  return done(rmsnorm_quantize(dtype, x, residual, g, M, d, eps, h, y, codes, ld_codes, scales, (cudaStream_t)stream));
}

int splitlora_rmsnorm_bwd_workspace_bytes(int64_t M, int d, size_t* bytes) {
  if (!bytes || !rows_ok(M) || d < 1 || d > ROWS_MAX_WIDTH) return SPLITLORA_ERR_ARG;
  *bytes = rmsnorm_dg_scratch_floats(M, d) * 4;
  return SPLITLORA_OK;
}

int splitlora_rmsnorm_bwd(int dtype, const void* dy, const void* h, const void* g, const void* residual, float eps, int64_t M, int d, void* dx,
                          float* dg, void* workspace, size_t workspace_bytes, void* stream) {
  LaunchChain chain;
  if (!dtype_ok(dtype) || !dy || !h || !g || !dx || !rows_ok(M) || d < 1 || d > ROWS_MAX_WIDTH || !(eps >= 0.f) || std::isinf(eps)) return SPLITLORA_ERR_ARG;
  for (const void* p : {dy, h, g, residual, (const void*)dx})
    if (!aligned_elem(dtype, p)) return SPLITLORA_ERR_ALIGN;
  if (dg) {
    if (!workspace || workspace_bytes < rmsnorm_dg_scratch_floats(M, d) * 4) return SPLITLORA_ERR_WORKSPACE;
    if (!aligned(dg, 4) || !aligned(workspace, 16)) return SPLITLORA_ERR_ALIGN;
  }
  return done(rmsnorm_gain_bwd(dtype, dy, h, g, residual, M, d, eps, dx, dg, (float*)workspace, (cudaStream_t)stream));
}

int splitlora_linear_i8(int dtype, const int8_t* x, int64_t ld_x, const float* x_scales, const int8_t* W, int64_t ld_w, const float* w_scales,
                        const void* bias, const void* residual, int M, int n_in, int n_out, void* y, void* stream) {
  LaunchChain chain;
  if (!dtype_ok(dtype) || !x || !x_scales || !W || !y || M < 1 || M > SIDE_MOST || n_in < 1 || n_in > QUANT_MAX_WIDTH || n_out < 1 ||
      n_out > SIDE_MOST || ld_x < n_in || ld_w < n_in)
    return SPLITLORA_ERR_ARG;
  if ((int64_t)((M + 63) / 64) * ((n_out + 63) / 64) > (1 << 28)) return SPLITLORA_ERR_ARG;
  if (!aligned(x_scales, 4) || !aligned(w_scales, 4)) return SPLITLORA_ERR_ALIGN;
  for (const void* p : {bias, residual, (const void*)y})
    if (!aligned_elem(dtype, p)) return SPLITLORA_ERR_ALIGN;
  int* status = library_status_word();
  if (gemm_i8_init() != 0 || !status) return SPLITLORA_ERR_CUDA;
  I8Args a;
  a.dtype = dtype; a.M = M; a.N = n_out; a.K = n_in; a.X = x; a.ldx = ld_x; a.W = W; a.ldw = ld_w; a.x_scales = x_scales; a.w_scales = w_scales;
  a.bias = bias; a.R = residual; a.Y = y;
  return done(gemm_i8(a, status, (cudaStream_t)stream));
}

int splitlora_distill_loss(int dtype, const void* logits, int64_t ld, const int32_t* labels, const int32_t* top_idx, const float* top_logits, int M,
                           int vocab, int k, float temperature, float ce_weight, float kd_weight, int64_t normalizer, void* dlogits, int64_t ld_grad,
                           float* row_loss, float* loss, int32_t* n_valid, void* stream) {
  LaunchChain chain;
  if (!dtype_ok(dtype) || !logits || !top_idx || !top_logits || !dlogits || !row_loss || !loss || !n_valid || M < 1 || M > SIDE_MOST || vocab < 1 ||
      k < 1 || k > DISTILL_MAX_K || ld < vocab || ld > SIDE_MOST || ld_grad < vocab || ld_grad > SIDE_MOST || normalizer < 0 || normalizer > 2147483647LL)
    return SPLITLORA_ERR_ARG;
  if (!(temperature >= 1e-3f) || !(temperature <= 1e3f) || !std::isfinite(ce_weight) || !std::isfinite(kd_weight)) return SPLITLORA_ERR_ARG;
  if (!labels && ce_weight != 0.f) return SPLITLORA_ERR_ARG;
  if (dlogits == logits && ld != ld_grad) return SPLITLORA_ERR_ARG;
  if (!aligned_elem(dtype, logits) || !aligned_elem(dtype, dlogits)) return SPLITLORA_ERR_ALIGN;
  for (const void* p : {(const void*)labels, (const void*)top_idx, (const void*)top_logits, (const void*)row_loss, (const void*)loss, (const void*)n_valid})
    if (!aligned(p, 4)) return SPLITLORA_ERR_ALIGN;
  int* status = library_status_word();
  if (!status) return SPLITLORA_ERR_CUDA;
  return done(distill(dtype, logits, ld, labels, top_idx, top_logits, M, vocab, k, temperature, ce_weight, kd_weight, (int)normalizer, dlogits, ld_grad,
                      row_loss, n_valid, loss, status, (cudaStream_t)stream));
}

}  // extern "C"
