// The row-wise operators' launches (layer_norm.hip, label_logprob.hip): arguments as in include/isp.h, checked by the callers.
#pragma once
#include "isp_internal.h"

constexpr int ISP_MAX_TOP = ISP_WAVE;  // alternatives: a lane each

static inline int64_t isp_ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Lanes that hold a row of d elements, `vec` to a load: the fewest whose vectors span it, four at least, a wavefront at most.
static inline int isp_row_lanes(int64_t d, int vec) {
  int l = 4;
  while (l < ISP_WAVE && (int64_t)l * vec < d) l *= 2;
  return l;
}

size_t isp_layer_norm_sums_bytes(int64_t n, int32_t d);
isp_status isp_layer_norm_launch(const void* X, int64_t ldx, int64_t n, int32_t d, int dtype, const void* weight, const void* bias, int param,
                                 float eps, void* Y, int64_t ldy, float* mean, float* rstd, hipStream_t s);
isp_status isp_layer_norm_bwd_launch(const void* X, int64_t ldx, const void* dY, int64_t lddy, int64_t n, int32_t d, int dtype, const void* weight,
                                     int param, const float* mean, const float* rstd, void* dX, int64_t lddx, void* dweight, void* dbias, void* ws,
                                     hipStream_t s);

size_t isp_label_logprob_parts_bytes(int64_t n, int32_t n_classes, int32_t top);
isp_status isp_label_logprob_launch(const void* Z, int64_t ldz, int64_t n, int32_t n_classes, int dtype, const int64_t* labels, float* logprob,
                                    float* entropy, float* stats, int32_t top, float* top_logprob, int32_t* top_index, void* ws, hipStream_t s);
isp_status isp_label_logprob_bwd_launch(const void* Z, int64_t ldz, int64_t n, int32_t n_classes, int dtype, const int64_t* labels,
                                        const float* stats, const float* entropy, const float* d_logprob, const float* d_entropy, void* dZ,
                                        int64_t lddz, hipStream_t s);
