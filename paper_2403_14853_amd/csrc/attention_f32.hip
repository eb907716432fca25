// Attention over the stored entries of a CSR matrix, fp32 operands (one unit per type: they compile side by side).
#include "attention.h"

isp_status isp_att_forward_f32(const isp_csr* A, const att_args& a, hipStream_t s) { return att_forward<float>(A, a, s); }
isp_status isp_att_backward_f32(const isp_csr* A, const att_args& a, const att_grads& o, hipStream_t s) { return att_backward<float>(A, a, o, s); }
