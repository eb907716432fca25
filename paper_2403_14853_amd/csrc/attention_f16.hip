// Attention over the stored entries of a CSR matrix, fp16 operands (one unit per type: they compile side by side).
#include "attention.h"

isp_status isp_att_forward_f16(const isp_csr* A, const att_args& a, hipStream_t s) { return att_forward<f16_t>(A, a, s); }
isp_status isp_att_backward_f16(const isp_csr* A, const att_args& a, const att_grads& o, hipStream_t s) { return att_backward<f16_t>(A, a, o, s); }
