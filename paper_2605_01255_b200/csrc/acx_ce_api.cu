// C ABI of the vocabulary cross entropy: argument checks and dispatch.
#include <cmath>

#include "acx_checks.h"
#include "acx_internal.h"

namespace acx {
namespace {

acx_status validate_ce(const acx_ce_desc* d, CeProblem* out) {
  if (!d || d->struct_size != sizeof(acx_ce_desc)) return ACX_ERR_INVALID_ARG;
  if (d->io_dtype != ACX_BF16) return ACX_ERR_INVALID_ARG;
  if (!std::isfinite(d->logit_scale) || d->reserved != 0) return ACX_ERR_INVALID_ARG;
  if (d->tokens < 0 || d->tokens > (int64_t(1) << 24)) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d->d < 8 || d->d % 8 || d->d > (int64_t(1) << 16)) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d->vocab < 1 || d->vocab > (int64_t(1) << 22)) return ACX_ERR_UNSUPPORTED_SHAPE;
  out->m = d->tokens;
  out->d = d->d;
  out->vocab = d->vocab;
  out->logit_scale = d->logit_scale;
  return ACX_OK;
}

}  // namespace
}  // namespace acx

using namespace acx;

extern "C" {

size_t acx_ce_workspace_bytes(const acx_ce_desc* desc, int op) {
  CeProblem p;
  if (validate_ce(desc, &p) != ACX_OK) return 0;
  if (op == ACX_OP_CE_FWD) return ce_fwd_workspace_bytes(p);
  if (op == ACX_OP_CE_BWD) return ce_bwd_workspace_bytes(p);
  return 0;
}

acx_status acx_linear_ce_fwd(const acx_ce_desc* desc, const void* X, const void* W, const int64_t* targets, const float* weight, float* loss,
                             float* lse, float* total, void* ws, size_t ws_bytes, void* cuda_stream) {
  CeProblem p;
  const acx_status s = validate_ce(desc, &p);
  if (s != ACX_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (p.m == 0) return total ? from_cuda(cudaMemsetAsync(total, 0, 2 * sizeof(float), st)) : ACX_OK;
  if (any_null(X, W, targets, loss, lse)) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(X, W, targets, weight, loss, lse, ws) || (reinterpret_cast<uintptr_t>(total) & 3u)) return ACX_ERR_ALIGNMENT;
  if (!ws || ws_bytes < ce_fwd_workspace_bytes(p)) return ACX_ERR_WORKSPACE;
  int* status = device_status_ptr();
  if (!status) return ACX_ERR_CUDA;
  return from_cuda(ce_fwd(p, X, W, targets, weight, loss, lse, total, ws, status, st));
}

acx_status acx_linear_ce_bwd(const acx_ce_desc* desc, const void* X, const void* W, const int64_t* targets, const float* weight,
                             const float* lse, const float* denom, float scale, void* dX, void* dW, void* ws, size_t ws_bytes,
                             void* cuda_stream) {
  return acx_linear_ce_bwd_loss(desc, X, W, targets, weight, lse, nullptr, denom, scale, dX, dW, ws, ws_bytes, cuda_stream);
}

acx_status acx_linear_ce_bwd_loss(const acx_ce_desc* desc, const void* X, const void* W, const int64_t* targets, const float* weight,
                                  const float* lse, const float* loss, const float* denom, float scale, void* dX, void* dW, void* ws,
                                  size_t ws_bytes, void* cuda_stream) {
  CeProblem p;
  const acx_status s = validate_ce(desc, &p);
  if (s != ACX_OK) return s;
  if (!std::isfinite(scale)) return ACX_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (p.m == 0) {
    if (misaligned(dW)) return ACX_ERR_ALIGNMENT;
    return dW ? from_cuda(cudaMemsetAsync(dW, 0, size_t(p.vocab) * size_t(p.d) * 2, st)) : ACX_OK;
  }
  if (any_null(X, W, targets, lse) || (!dX && !dW)) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(X, W, targets, weight, lse, loss, dX, dW, ws) || (reinterpret_cast<uintptr_t>(denom) & 3u)) return ACX_ERR_ALIGNMENT;
  if (!ws || ws_bytes < ce_bwd_workspace_bytes(p)) return ACX_ERR_WORKSPACE;
  int* status = device_status_ptr();
  if (!status) return ACX_ERR_CUDA;
  return from_cuda(ce_bwd(p, X, W, targets, weight, lse, loss, denom, scale, dX, dW, ws, status, st));
}

}  // extern "C"
