// The attention's entry points (include/isp.h): argument checks, workspaces, dispatch by element type.  The kernels: attention.h.
#include "attention_args.h"
#include "elem.h"
#include "group_stream.h"

namespace {

isp_status check_heads(const isp_csr* A, int32_t heads, int32_t kv_heads, int32_t dh) {
  using namespace isp_dev;
  if (!A) return isp_fail(ISP_EINVAL, "handle is NULL");
  if (heads <= 0 || kv_heads <= 0 || dh <= 0) return isp_fail(ISP_EINVAL, "heads, kv_heads and head_dim must be positive");
  if (heads % kv_heads) return isp_fail(ISP_EINVAL, "heads (%d) is not a multiple of kv_heads (%d)", heads, kv_heads);
  if (dh > ATT_MAX_DIM) return isp_fail(ISP_EUNSUPPORTED, "heads of more than %d columns", ATT_MAX_DIM);
  if (heads > ATT_MAX_HEADS) return isp_fail(ISP_EUNSUPPORTED, "more than %d heads", ATT_MAX_HEADS);
  if (A->info.block_cost > GS_MAX_ROWS || A->info.block_cost + A->v.hub_t > GS_MAX_ENT || A->v.seg_len > GS_MAX_ENT)
    return isp_fail(ISP_EUNSUPPORTED, "the work partition does not fit the kernels' tables");
  return ISP_OK;
}
isp_status check_operand(const void* p, int64_t ld, int32_t width, int64_t rows, int dtype, const char* name) {
  ISP_TRY(isp_check_dense(p, ld, width, rows, name));
  if (rows > 0 && ld > 0xffffffffll / isp_dtype_size(dtype))
    return isp_fail(ISP_EUNSUPPORTED, "the rows of %s are 4 GB or more apart", name);
  return ISP_OK;
}
isp_status check_type(int dtype, unsigned flags, const isp_csr* A) {
  if (dtype != ISP_F32 && dtype != ISP_BF16 && dtype != ISP_F16) return isp_fail(ISP_EUNSUPPORTED, "unknown element type %d", dtype);
  if (flags & ~ISP_BIAS_BY_A) return isp_fail(ISP_EUNSUPPORTED, "unknown flag bits 0x%x", flags & ~ISP_BIAS_BY_A);
  if ((flags & ISP_BIAS_BY_A) && !A->v.values) return isp_fail(ISP_EINVAL, "ISP_BIAS_BY_A needs a matrix with values");
  return ISP_OK;
}

size_t forward_bytes(const isp_csr* A, int32_t heads, int32_t dh) { return isp_align((size_t)A->v.n_seg * heads * (dh + 2) * sizeof(float)); }
// and for the copy of K and V, where the rule takes one
size_t packed_bytes(const isp_csr* A, int32_t kv_heads, int32_t dh, int dtype, bool whole) {
  const int64_t row = (int64_t)kv_heads * dh * isp_dtype_size(dtype);
  return isp_dev::att_packs(row, whole, A->v.nnz, A->v.n_cols) ? (size_t)A->v.n_cols * isp_dev::att_packed_pitch(row) : 0;
}

struct backward_space {  // (offsets)
  size_t part, carry, carry2, total;
};
backward_space backward_bytes(const isp_csr* A, int32_t heads, int32_t kv_heads, int32_t dh) {
  backward_space b;
  const int group = heads / kv_heads;
  b.part = isp_align((size_t)A->v.n_rows * heads * sizeof(att_num));
  const size_t row = (size_t)A->v.n_seg * heads * (2 * dh + 1), col = A->At ? (size_t)A->At->v.n_seg * 2 * kv_heads * dh : 0;
  b.carry = b.part + isp_align((row > col ? row : col) * sizeof(float));
  const size_t carry = group > isp_dev::att_share(group, 4) ? isp_align((size_t)A->v.n_cols * kv_heads * dh * sizeof(float)) : 0;
  b.carry2 = b.carry + carry;
  b.total = b.carry2 + carry;
  return b;
}

att_args make_args(int32_t heads, int32_t kv_heads, int32_t dh, float scale, unsigned flags) {
  att_args a{};
  a.heads = heads;
  a.kv_heads = kv_heads;
  a.group = heads / kv_heads;
  a.dh = dh;
  a.scale = scale;
  a.bias = (flags & ISP_BIAS_BY_A) != 0;
  a.passes = 1;
  return a;
}

}  // namespace

extern "C" {

isp_status isp_attention_workspace(const isp_csr_t* A, int32_t heads, int32_t kv_heads, int32_t head_dim, int dtype, size_t* bytes) {
  if (!bytes) return isp_fail(ISP_EINVAL, "bytes is NULL");
  ISP_TRY(check_heads(A, heads, kv_heads, head_dim));
  ISP_TRY(check_type(dtype, 0, A));
  const int64_t row = (int64_t)kv_heads * head_dim * isp_dtype_size(dtype);  // (dense rows)
  *bytes = forward_bytes(A, heads, head_dim) + packed_bytes(A, kv_heads, head_dim, dtype, row % isp_dev::ATT_LINE == 0);
  return ISP_OK;
}

isp_status isp_attention(const isp_csr_t* A, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv, int32_t heads,
                         int32_t kv_heads, int32_t head_dim, float scale, unsigned flags, int dtype, void* Y, int64_t ldy, float* stats,
                         void* workspace, size_t workspace_bytes, void* stream) {
  ISP_TRY(check_heads(A, heads, kv_heads, head_dim));
  ISP_TRY(isp_check_device(A));
  ISP_TRY(check_type(dtype, flags, A));
  const int64_t live = A->v.nnz > 0 ? 1 : 0;
  ISP_TRY(check_operand(Q, ldq, heads * head_dim, live * A->v.n_rows, dtype, "Q"));
  ISP_TRY(check_operand(K, ldk, kv_heads * head_dim, live * A->v.n_cols, dtype, "K"));
  ISP_TRY(check_operand(V, ldv, kv_heads * head_dim, live * A->v.n_cols, dtype, "V"));
  ISP_TRY(isp_check_dense(Y, ldy, heads * head_dim, A->v.n_rows, "Y"));
  const uint32_t size = isp_dtype_size(dtype);
  const auto lines = [&](const void* p, int64_t ld) { return (uintptr_t)p % isp_dev::ATT_LINE == 0 && ld * size % isp_dev::ATT_LINE == 0; };
  const size_t parts = forward_bytes(A, heads, head_dim), copy = packed_bytes(A, kv_heads, head_dim, dtype, lines(K, ldk) && ldv == ldk && (uintptr_t)V % 4 == 0);
  const bool pack = copy && workspace_bytes >= parts + copy;
  ISP_TRY(isp_check_workspace(workspace, workspace_bytes, parts + (pack ? copy : 0)));
  att_args a = make_args(heads, kv_heads, head_dim, scale, flags);
  a.q = Q, a.k = K, a.v = V;
  a.pq = (uint32_t)ldq * size, a.pk = (uint32_t)ldk * size, a.pv = (uint32_t)ldv * size;
  a.y = Y, a.ldy = ldy;
  a.stats = stats;
  a.part = static_cast<float*>(workspace);
  if (pack) {
    a.packed = static_cast<char*>(workspace) + parts;
    a.n_cols = A->v.n_cols;
  }
  if (dtype == ISP_F32) return isp_att_forward_f32(A, a, (hipStream_t)stream);
  if (dtype == ISP_BF16) return isp_att_forward_bf16(A, a, (hipStream_t)stream);
  return isp_att_forward_f16(A, a, (hipStream_t)stream);
}

isp_status isp_attention_backward_workspace(const isp_csr_t* A, int32_t heads, int32_t kv_heads, int32_t head_dim, size_t* bytes) {
  if (!bytes) return isp_fail(ISP_EINVAL, "bytes is NULL");
  ISP_TRY(check_heads(A, heads, kv_heads, head_dim));
  *bytes = backward_bytes(A, heads, kv_heads, head_dim).total;
  return ISP_OK;
}

isp_status isp_attention_backward(const isp_csr_t* A, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                                  int32_t heads, int32_t kv_heads, int32_t head_dim, float scale, unsigned flags, int dtype, const float* stats,
                                  const void* dY, int64_t lddy, void* dQ, int64_t lddq, void* dK, int64_t lddk,
                                  void* dV, int64_t lddv, void* workspace, size_t workspace_bytes, void* stream) {
  ISP_TRY(check_heads(A, heads, kv_heads, head_dim));
  ISP_TRY(isp_check_device(A));
  if (A->is_transpose) return isp_fail(ISP_EINVAL, "pass the source handle, not its transpose");
  if ((dK == nullptr) != (dV == nullptr) && A->v.n_cols > 0) return isp_fail(ISP_EINVAL, "dK and dV are wanted together or not at all");
  if (dK && !A->At) return isp_fail(ISP_EINVAL, "call isp_csr_transpose_cached on the handle first");
  ISP_TRY(check_type(dtype, flags, A));
  const int32_t width = heads * head_dim, kv_width = kv_heads * head_dim;
  const int64_t live = A->v.nnz > 0 ? 1 : 0, n = A->v.n_rows, m = A->v.n_cols;
  ISP_TRY(check_operand(Q, ldq, width, live * n, dtype, "Q"));
  ISP_TRY(check_operand(K, ldk, kv_width, live * m, dtype, "K"));
  ISP_TRY(check_operand(V, ldv, kv_width, live * m, dtype, "V"));
  ISP_TRY(check_operand(dY, lddy, width, live * n, dtype, "dY"));
  if (n > 0 && !stats) return isp_fail(ISP_EINVAL, "stats is NULL");
  if (dQ) ISP_TRY(isp_check_dense(dQ, lddq, width, n, "dQ"));
  if (dK) ISP_TRY(isp_check_dense(dK, lddk, kv_width, m, "dK"));
  if (dV) ISP_TRY(isp_check_dense(dV, lddv, kv_width, m, "dV"));
  const backward_space b = backward_bytes(A, heads, kv_heads, head_dim);
  ISP_TRY(isp_check_workspace(workspace, workspace_bytes, b.total));
  const uint32_t size = isp_dtype_size(dtype);
  char* ws = static_cast<char*>(workspace);
  att_args a = make_args(heads, kv_heads, head_dim, scale, flags);
  a.q = Q, a.k = K, a.v = V, a.dy = dY;
  a.pq = (uint32_t)ldq * size, a.pk = (uint32_t)ldk * size, a.pv = (uint32_t)ldv * size, a.pdy = (uint32_t)lddy * size;
  a.stats = const_cast<float*>(stats);
  a.stat = reinterpret_cast<att_num*>(ws);
  a.part = reinterpret_cast<float*>(ws + b.part);
  a.carry = reinterpret_cast<float*>(ws + b.carry);
  a.carry2 = reinterpret_cast<float*>(ws + b.carry2);
  const att_grads o{dQ, dK, dV, lddq, lddk, lddv};
  if (dtype == ISP_F32) return isp_att_backward_f32(A, a, o, (hipStream_t)stream);
  if (dtype == ISP_BF16) return isp_att_backward_bf16(A, a, o, (hipStream_t)stream);
  return isp_att_backward_f16(A, a, o, (hipStream_t)stream);
}

}  // extern "C"
