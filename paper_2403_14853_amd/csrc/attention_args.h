// What the passes of the attention over a CSR matrix take (attention.h), and how its entry points (attention.hip) reach them.
#pragma once
#include "attention_rule.h"
#include "isp_internal.h"

constexpr int ATT_MAX_DIM = 256;     // columns of a head: 64 lanes of four
constexpr int ATT_MAX_HEADS = 4096;

// What the columns' pass of the backward reads of a row and head: the reference of its scores, 1 / (the sum of exp(s - m)), D.  16 bytes: eight heads'
// are one line (12: 169 k rows, 2.4 M entries, 8 heads of 16, fp32 288 / 299 us).
struct __attribute__((aligned(16))) att_num {
  float m, inv, d, spare;
};

struct att_args {
  const void *q, *k, *v, *dy;
  uint32_t pq, pk, pv, pdy;  // distances between rows in bytes
  int heads, kv_heads, group, dh;  // group = heads / kv_heads
  int lph;                   // lanes per head: a power of two
  float scale;
  int bias;                  // the matrix's values are added to the scores
  void *y, *y2;              // output rows (forward y, backward dq or dk; y2: dv)
  int64_t ldy, ldy2;         // in elements
  void* packed;              // forward: room for K's and V's rows next to each other (NULL: they are read as they lie)
  int64_t n_cols;
  float* stats;              // (m, l) per row and head: written by the forward (may be NULL), read by the backward
  att_num* stat;             // backward, per row and head, in the workspace
  float* part;               // partial rows of the split rows' segments, in the workspace
  float *carry, *carry2;     // dk and dv between the passes over a key head's query heads, fp32, rows of kv_heads * dh, in the workspace
  int pass, passes;
};
struct att_grads {
  void *dq, *dk, *dv;
  int64_t lddq, lddk, lddv;
};

isp_status isp_att_forward_f32(const isp_csr* A, const att_args& a, hipStream_t s);
isp_status isp_att_forward_bf16(const isp_csr* A, const att_args& a, hipStream_t s);
isp_status isp_att_forward_f16(const isp_csr* A, const att_args& a, hipStream_t s);
isp_status isp_att_backward_f32(const isp_csr* A, const att_args& a, const att_grads& o, hipStream_t s);
isp_status isp_att_backward_bf16(const isp_csr* A, const att_args& a, const att_grads& o, hipStream_t s);
isp_status isp_att_backward_f16(const isp_csr* A, const att_args& a, const att_grads& o, hipStream_t s);
