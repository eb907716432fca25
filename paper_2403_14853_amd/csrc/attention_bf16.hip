// Attention over the stored entries of a CSR matrix, bf16 operands (one unit per type: they compile side by side).
#include "attention.h"

isp_status isp_att_forward_bf16(const isp_csr* A, const att_args& a, hipStream_t s) { return att_forward<bf16_t>(A, a, s); }
isp_status isp_att_backward_bf16(const isp_csr* A, const att_args& a, const att_grads& o, hipStream_t s) { return att_backward<bf16_t>(A, a, o, s); }
