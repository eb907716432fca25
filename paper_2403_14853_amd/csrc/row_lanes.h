// Whole rows in registers (gfx950, wave64): what layer norm and the label log probabilities share.  LPR consecutive lanes hold a row
// of up to LPR * VEC * NV elements, vector v of lane q the columns [v * LPR * VEC + q * VEC, ...); a wavefront works on 64 / LPR rows.
#pragma once
#include "elem.h"
#include "group_stream.h"

namespace isp_dev {

// A lane's columns.  Where the width is no multiple of VEC the row's last vector moves back to end with the last column: dup of its
// leading elements belong to the vector before it.  They are left out of sums; what is computed for them is what
// the other vector computes, so both store the same bits.  Vectors past the row read its first columns and store nothing.
// Needs d >= VEC.
template <int VEC, int LPR, int NV>
struct row_cols {
  int off[NV], dup[NV];  // dup = VEC: no element counts
  bool on[NV];
  __device__ __forceinline__ row_cols(int q, int d) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * LPR + q) * VEC;
      on[v] = col < d;
      off[v] = !on[v] ? 0 : col + VEC > d ? d - VEC : col;
      dup[v] = on[v] ? col - off[v] : VEC;
    }
  }
  __device__ __forceinline__ bool counts(int v, int c) const { return c >= dup[v]; }
};

template <int LPR>
__device__ __forceinline__ float lanes_sum(float v) { return group_allreduce<LPR>(v); }

// The maximum over LPR consecutive lanes (4 and more), in all of them.  NaN counts as nothing.
template <int LPR>
__device__ __forceinline__ float lanes_max(float v) {
  v = fmaxf(v, dpp_of<DPP_XOR1>(v));
  v = fmaxf(v, dpp_of<DPP_XOR2>(v));
  if constexpr (LPR >= 8) v = fmaxf(v, dpp_of<DPP_HALF_MIRROR>(v));
  if constexpr (LPR >= 16) v = fmaxf(v, dpp_of<DPP_ROR8>(v));
  if constexpr (LPR >= 32) v = fmaxf(v, __shfl_xor(v, 16));
  if constexpr (LPR >= 64) v = fmaxf(v, __shfl_xor(v, 32));
  return v;
}

// Sums of K values over a workgroup of BT threads, in every thread.  buf: 2 * K * BT / 64 floats of LDS, used in halves by turns (turn: 0, 1, 0,
// ... from call to call), so that one barrier a call is enough.
template <int K, int BT>
__device__ __forceinline__ void block_sums(float (&v)[K], float* buf, int turn) {
  constexpr int WAVES = BT / ISP_WAVE;
  const int lane = threadIdx.x & (ISP_WAVE - 1), w = threadIdx.x >> 6;
  float* b = buf + turn * K * WAVES;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] = group_allreduce<ISP_WAVE>(v[k]);
    if (lane == 0) b[k * WAVES + w] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float t = b[k * WAVES];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) t += b[k * WAVES + i];
    v[k] = t;
  }
}

}  // namespace isp_dev
