// The C ABI's row-wise operators (include/isp.h): argument checks and dispatch.  No handle: the arrays are the current device's.
#include "elem.h"
#include "rowwise.h"

namespace {

isp_status check_types(int dtype, int param) {
  if (dtype != ISP_F32 && dtype != ISP_BF16 && dtype != ISP_F16) return isp_fail(ISP_EUNSUPPORTED, "unknown element type %d", dtype);
  if (param != ISP_F32 && param != dtype) return isp_fail(ISP_EUNSUPPORTED, "the parameters are fp32 or of the matrix's type");
  return ISP_OK;
}
isp_status check_rows(int64_t n, int32_t d) {
  if (n < 0) return isp_fail(ISP_EINVAL, "negative size");
  if (d <= 0) return isp_fail(ISP_EINVAL, "the rows are empty");
  if (d > 2147483647 - 65536) return isp_fail(ISP_EUNSUPPORTED, "rows of %d elements", d);  // (column numbers stay below 2^31)
  return ISP_OK;
}

}  // namespace

extern "C" {

isp_status isp_layer_norm(const void* X, int64_t ldx, int64_t n, int32_t d, int dtype, const void* weight, const void* bias, int param_dtype,
                          float eps, void* Y, int64_t ldy, float* mean, float* rstd, void* stream) {
  ISP_TRY(check_types(dtype, param_dtype));
  ISP_TRY(check_rows(n, d));
  ISP_TRY(isp_check_dense(X, ldx, d, n, "X"));
  ISP_TRY(isp_check_dense(Y, ldy, d, n, "Y"));
  if (!(eps >= 0.f)) return isp_fail(ISP_EINVAL, "eps is negative");
  return isp_layer_norm_launch(X, ldx, n, d, dtype, weight, bias, param_dtype, eps, Y, ldy, mean, rstd, (hipStream_t)stream);
}

isp_status isp_layer_norm_backward_workspace(int64_t n, int32_t d, size_t* bytes) {
  if (!bytes) return isp_fail(ISP_EINVAL, "bytes is NULL");
  ISP_TRY(check_rows(n, d));
  *bytes = isp_layer_norm_sums_bytes(n, d);
  return ISP_OK;
}

isp_status isp_layer_norm_backward(const void* X, int64_t ldx, const void* dY, int64_t lddy, int64_t n, int32_t d, int dtype, const void* weight,
                                   int param_dtype, const float* mean, const float* rstd, void* dX, int64_t lddx, void* dweight, void* dbias,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  ISP_TRY(check_types(dtype, param_dtype));
  ISP_TRY(check_rows(n, d));
  ISP_TRY(isp_check_dense(X, ldx, d, n, "X"));
  ISP_TRY(isp_check_dense(dY, lddy, d, n, "dY"));
  if (dX) ISP_TRY(isp_check_dense(dX, lddx, d, n, "dX"));
  if (n > 0 && (!mean || !rstd)) return isp_fail(ISP_EINVAL, "mean or rstd is NULL");
  if (dweight || dbias) ISP_TRY(isp_check_workspace(workspace, workspace_bytes, isp_layer_norm_sums_bytes(n, d)));
  return isp_layer_norm_bwd_launch(X, ldx, dY, lddy, n, d, dtype, weight, param_dtype, mean, rstd, dX, lddx, dweight, dbias, workspace,
                                   (hipStream_t)stream);
}

static isp_status check_top(int32_t n_classes, int32_t top) {
  if (top < 0 || top > n_classes) return isp_fail(ISP_EINVAL, "top is not in [0, n_classes]");
  if (top > ISP_MAX_TOP) return isp_fail(ISP_EUNSUPPORTED, "at most %d alternatives", ISP_MAX_TOP);
  return ISP_OK;
}

isp_status isp_label_logprob_workspace(int64_t n, int32_t n_classes, int32_t top, size_t* bytes) {
  if (!bytes) return isp_fail(ISP_EINVAL, "bytes is NULL");
  ISP_TRY(check_rows(n, n_classes));
  ISP_TRY(check_top(n_classes, top));
  *bytes = isp_label_logprob_parts_bytes(n, n_classes, top);
  return ISP_OK;
}

isp_status isp_label_logprob(const void* Z, int64_t ldz, int64_t n, int32_t n_classes, int dtype, const int64_t* labels, float* logprob,
                             float* entropy, float* stats, int32_t top, float* top_logprob, int32_t* top_index, void* workspace,
                             size_t workspace_bytes, void* stream) {
  ISP_TRY(check_types(dtype, dtype));
  ISP_TRY(check_rows(n, n_classes));
  ISP_TRY(check_top(n_classes, top));
  ISP_TRY(isp_check_dense(Z, ldz, n_classes, n, "Z"));
  if (n > 0 && logprob && !labels) return isp_fail(ISP_EINVAL, "labels is NULL");
  ISP_TRY(isp_check_workspace(workspace, workspace_bytes, isp_label_logprob_parts_bytes(n, n_classes, top)));
  return isp_label_logprob_launch(Z, ldz, n, n_classes, dtype, labels, logprob, entropy, stats, top, top_logprob, top_index, workspace,
                                  (hipStream_t)stream);
}

isp_status isp_label_logprob_backward(const void* Z, int64_t ldz, int64_t n, int32_t n_classes, int dtype, const int64_t* labels, const float* stats,
                                      const float* entropy, const float* d_logprob, const float* d_entropy, void* dZ, int64_t lddz, void* stream) {
  ISP_TRY(check_types(dtype, dtype));
  ISP_TRY(check_rows(n, n_classes));
  ISP_TRY(isp_check_dense(Z, ldz, n_classes, n, "Z"));
  ISP_TRY(isp_check_dense(dZ, lddz, n_classes, n, "dZ"));
  if (n > 0 && !stats) return isp_fail(ISP_EINVAL, "stats is NULL");
  if (n > 0 && d_logprob && !labels) return isp_fail(ISP_EINVAL, "labels is NULL");
  if (n > 0 && d_entropy && !entropy) return isp_fail(ISP_EINVAL, "entropy is NULL");
  return isp_label_logprob_bwd_launch(Z, ldz, n, n_classes, dtype, labels, stats, entropy, d_logprob, d_entropy, dZ, lddz, (hipStream_t)stream);
}

}  // extern "C"
