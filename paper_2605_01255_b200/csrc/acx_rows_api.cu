// C ABI of the row operators (8-bit checkpoints, gated activation, residual join): argument checks and dispatch.
#include <cmath>

#include "acx_checks.h"
#include "acx_internal.h"

namespace acx {
namespace {

acx_status validate_rows(const acx_rows_desc* d, Rows* out) {
  if (!d || d->struct_size != sizeof(acx_rows_desc)) return ACX_ERR_INVALID_ARG;
  if (d->io_dtype != ACX_F32 && d->io_dtype != ACX_BF16) return ACX_ERR_INVALID_ARG;
  if (d->rows < 0 || d->rows > (int64_t(1) << 31) - 1) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d->cols < 8 || d->cols % 8 || d->cols > (int64_t(1) << 24)) return ACX_ERR_UNSUPPORTED_SHAPE;
  // the kernels number runs of at least 16 groups along one grid dimension
  if (d->rows * ((d->cols + ACX_Q8_GROUP - 1) / ACX_Q8_GROUP) / 16 >= 0x7FFFFFFFll) return ACX_ERR_UNSUPPORTED_SHAPE;
  out->rows = d->rows;
  out->cols = d->cols;
  out->bf16 = d->io_dtype == ACX_BF16;
  return ACX_OK;
}
bool bad_stride(const Rows& d, int64_t ld) { return ld < d.cols || ld % 8 || ld > (int64_t(1) << 40); }

acx_status validate_norm(const acx_rows_desc* d, Rows* out) {
  const acx_status s = validate_rows(d, out);
  return s == ACX_OK && out->cols > kMaxNormCols ? ACX_ERR_UNSUPPORTED_SHAPE : s;
}

}  // namespace
}  // namespace acx

using namespace acx;

extern "C" {

size_t acx_rows_workspace_bytes(const acx_rows_desc* desc, int op) {
  Rows d;
  if (op != ACX_OP_NORM_BWD || validate_norm(desc, &d) != ACX_OK || d.rows == 0) return 0;
  return norm_join_bwd_workspace_bytes(d);
}

acx_status acx_q8_store(const acx_rows_desc* desc, const void* X, int64_t ldx, int8_t* codes, float* scales, void* cuda_stream) {
  Rows d;
  const acx_status s = validate_rows(desc, &d);
  if (s != ACX_OK) return s;
  if (bad_stride(d, ldx)) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d.rows == 0) return ACX_OK;
  if (any_null(X, codes, scales)) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(X, codes, scales)) return ACX_ERR_ALIGNMENT;
  return from_cuda(q8_store(d, X, ldx, codes, scales, static_cast<cudaStream_t>(cuda_stream)));
}

acx_status acx_q8_load(const acx_rows_desc* desc, const int8_t* codes, const float* scales, void* X, int64_t ldx, void* cuda_stream) {
  Rows d;
  const acx_status s = validate_rows(desc, &d);
  if (s != ACX_OK) return s;
  if (bad_stride(d, ldx)) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d.rows == 0) return ACX_OK;
  if (any_null(X, codes, scales)) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(X, codes, scales)) return ACX_ERR_ALIGNMENT;
  return from_cuda(q8_load(d, codes, scales, X, ldx, static_cast<cudaStream_t>(cuda_stream)));
}

acx_status acx_swiglu_fwd(const acx_rows_desc* desc, const void* G, int64_t ldg, const void* U, int64_t ldu, void* H, int8_t* Gq, float* Gs,
                          int8_t* Uq, float* Us, void* cuda_stream) {
  Rows d;
  const acx_status s = validate_rows(desc, &d);
  if (s != ACX_OK) return s;
  if (bad_stride(d, ldg) || bad_stride(d, ldu)) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d.rows == 0) return ACX_OK;
  if (any_null(G, U, H)) return ACX_ERR_INVALID_ARG;
  const bool keep = Gq || Gs || Uq || Us;
  if (keep && any_null(Gq, Gs, Uq, Us)) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(G, U, H, Gq, Gs, Uq, Us)) return ACX_ERR_ALIGNMENT;
  return from_cuda(swiglu_fwd(d, G, ldg, U, ldu, H, Gq, Gs, Uq, Us, static_cast<cudaStream_t>(cuda_stream)));
}

acx_status acx_swiglu_bwd(const acx_rows_desc* desc, const void* dH, const int8_t* Gq, const float* Gs, const int8_t* Uq, const float* Us,
                          void* dG, int64_t lddg, void* dU, int64_t lddu, void* cuda_stream) {
  Rows d;
  const acx_status s = validate_rows(desc, &d);
  if (s != ACX_OK) return s;
  if (bad_stride(d, lddg) || bad_stride(d, lddu)) return ACX_ERR_UNSUPPORTED_SHAPE;
  if (d.rows == 0) return ACX_OK;
  if (any_null(dH, Gq, Gs, Uq, Us, dG, dU)) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(dH, Gq, Gs, Uq, Us, dG, dU)) return ACX_ERR_ALIGNMENT;
  return from_cuda(swiglu_bwd(d, dH, Gq, Gs, Uq, Us, dG, lddg, dU, lddu, static_cast<cudaStream_t>(cuda_stream)));
}

acx_status acx_norm_join_fwd(const acx_rows_desc* desc, const void* h, const void* b, const void* w_post, const void* gate,
                             const void* w_pre, void* h_out, void* y, int8_t* Hq, float* Hs, int8_t* Bq, float* Bs, float* rstd_post,
                             float* rstd_pre, float eps, float alpha, void* cuda_stream) {
  Rows d;
  const acx_status s = validate_norm(desc, &d);
  if (s != ACX_OK) return s;
  if (!(eps >= 0.f) || std::isinf(eps) || !(alpha == alpha)) return ACX_ERR_INVALID_ARG;
  if (d.rows == 0) return ACX_OK;
  if (any_null(h, w_pre, y)) return ACX_ERR_INVALID_ARG;
  if (b ? !h_out : (w_post || gate || h_out || Bq || Bs || rstd_post)) return ACX_ERR_INVALID_ARG;
  if (!w_post && rstd_post) return ACX_ERR_INVALID_ARG;
  const bool keep = Hq || Hs || Bq || Bs || rstd_post || rstd_pre;
  if (keep && (any_null(Hq, Hs, rstd_pre) || (b && any_null(Bq, Bs)) || (w_post && !rstd_post))) return ACX_ERR_INVALID_ARG;
  if (any_misaligned(h, b, w_post, gate, w_pre, h_out, y) || any_misaligned(Hq, Hs, Bq, Bs, rstd_post, rstd_pre)) return ACX_ERR_ALIGNMENT;
  return from_cuda(norm_join_fwd(d, h, b, w_post, gate, w_pre, h_out, y, Hq, Hs, Bq, Bs, rstd_post, rstd_pre, eps, alpha,
                                 static_cast<cudaStream_t>(cuda_stream)));
}

acx_status acx_norm_join_bwd(const acx_rows_desc* desc, const void* dy, const void* dh_next, const void* w_post, const void* gate,
                             const void* w_pre, const int8_t* Hq, const float* Hs, const int8_t* Bq, const float* Bs,
                             const float* rstd_post, const float* rstd_pre, void* dh, void* db, float* dw_post, float* dgate,
                             float* dw_pre, float alpha, void* ws, size_t ws_bytes, void* cuda_stream) {
  Rows d;
  const acx_status s = validate_norm(desc, &d);
  if (s != ACX_OK) return s;
  if (!(alpha == alpha)) return ACX_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (any_misaligned(dy, dh_next, w_post, gate, w_pre, Hq, Hs, Bq, Bs) || any_misaligned(rstd_post, rstd_pre, dh, db, dw_post, dgate, dw_pre, ws))
    return ACX_ERR_ALIGNMENT;
  if (d.rows == 0) {
    float* const v[3] = {dw_post, dgate, dw_pre};
    for (float* p : v)
      if (p && cudaMemsetAsync(p, 0, size_t(d.cols) * sizeof(float), st) != cudaSuccess) return ACX_ERR_CUDA;
    return ACX_OK;
  }
  if (any_null(dy, w_pre, Hq, Hs, rstd_pre, dh)) return ACX_ERR_INVALID_ARG;
  // what belongs to a part that is absent must be absent too
  if ((w_post == nullptr) != (rstd_post == nullptr) || (!w_post && dw_post) || (!gate && dgate)) return ACX_ERR_INVALID_ARG;
  const bool join = Bq != nullptr;
  if ((Bs != nullptr) != join || (db != nullptr) != join || (!join && (w_post || gate))) return ACX_ERR_INVALID_ARG;
  if (!ws || ws_bytes < norm_join_bwd_workspace_bytes(d)) return ACX_ERR_WORKSPACE;
  return from_cuda(norm_join_bwd(d, dy, dh_next, w_post, gate, w_pre, Hq, Hs, Bq, Bs, rstd_post, rstd_pre, dh, db, dw_post, dgate, dw_pre,
                                 alpha, ws, st));
}

}  // extern "C"
