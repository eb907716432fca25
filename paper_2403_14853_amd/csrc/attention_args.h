// What the passes of the attention over a CSR matrix take (attention.h), and how its entry points (attention.hip) reach them.
#pragma once
#include "isp_internal.h"

constexpr int ATT_MAX_DIM = 256;     // columns of a head: 64 lanes of four
constexpr int ATT_MAX_HEADS = 4096;

struct att_args {
  const void *q, *k, *v, *dy;
  uint32_t pq, pk, pv, pdy;  // distances between rows in bytes
  int heads, kv_heads, group, dh;  // group = heads / kv_heads
  int lph;                   // lanes per head: a power of two
  float scale;
  int bias;                  // the matrix's values are added to the scores
  void *y, *y2;              // output rows (forward y, backward dq or dk; y2: dv)
  int64_t ldy, ldy2;         // in elements
  float* stats;              // (m, l) per row and head: written by the forward (may be NULL), read by the backward
  float4* stat;              // backward: (m, 1 / l, D, -) per row and head, in the workspace
  float* part;               // partial rows of the split rows' segments, in the workspace
  float *carry, *carry2;     // dk and dv between the passes over a key head's query heads, fp32, rows of kv_heads * dh, in the workspace
  int pass, passes;
};
struct att_grads {
  void *dq, *dk, *dv;
  int64_t lddq, lddk, lddv;
};

// Query heads of a key head that a lane takes at once: as many of four as divide them.
inline int att_share(int group) { return group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1; }

isp_status isp_att_forward_f32(const isp_csr* A, const att_args& a, hipStream_t s);
isp_status isp_att_forward_bf16(const isp_csr* A, const att_args& a, hipStream_t s);
isp_status isp_att_forward_f16(const isp_csr* A, const att_args& a, hipStream_t s);
isp_status isp_att_backward_f32(const isp_csr* A, const att_args& a, const att_grads& o, hipStream_t s);
isp_status isp_att_backward_bf16(const isp_csr* A, const att_args& a, const att_grads& o, hipStream_t s);
isp_status isp_att_backward_f16(const isp_csr* A, const att_args& a, const att_grads& o, hipStream_t s);
