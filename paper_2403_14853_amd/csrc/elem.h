// Element types of the operators that take half precision too (isp_dtype): vectors of them in memory, floats in registers.
#pragma once
#include "isp_internal.h"

namespace isp_dev {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// W consecutive elements at any address that is aligned for one (the hardware takes such vector accesses in global memory).
template <class T, int W>
struct raw_vec {
  typedef T type __attribute__((ext_vector_type(W), aligned(sizeof(T))));
};
template <class T>
struct raw_vec<T, 1> {
  typedef T type;
};
template <class T, int W>
using raw_t = typename raw_vec<T, W>::type;

template <class T, int W>
__device__ __forceinline__ raw_t<T, W> load_raw(const T* p) {
  return *reinterpret_cast<const raw_t<T, W>*>(p);
}
template <class T, int W>
__device__ __forceinline__ void to_float(const raw_t<T, W>& v, float (&o)[W]) {
  if constexpr (W == 1) o[0] = (float)v;
  else
#pragma unroll
    for (int c = 0; c < W; ++c) o[c] = (float)v[c];
}
// (one rounding, to nearest even)
template <class T, int W>
__device__ __forceinline__ raw_t<T, W> from_float(const float (&o)[W]) {
  raw_t<T, W> v;
  if constexpr (W == 1) v = (T)o[0];
  else
#pragma unroll
    for (int c = 0; c < W; ++c) v[c] = (T)o[c];
  return v;
}
template <class T, int W>
__device__ __forceinline__ void store_raw(T* p, const float (&o)[W]) {
  *reinterpret_cast<raw_t<T, W>*>(p) = from_float<T, W>(o);
}

// A parameter array whose type is known at run time only (read or written once per launch and column).
__device__ __forceinline__ float load_param(const void* p, int dtype, int64_t i) {
  if (dtype == ISP_F32) return static_cast<const float*>(p)[i];
  if (dtype == ISP_BF16) return (float)static_cast<const bf16_t*>(p)[i];
  return (float)static_cast<const f16_t*>(p)[i];
}
__device__ __forceinline__ void store_param(void* p, int dtype, int64_t i, float v) {
  if (dtype == ISP_F32) static_cast<float*>(p)[i] = v;
  else if (dtype == ISP_BF16) static_cast<bf16_t*>(p)[i] = (bf16_t)v;
  else static_cast<f16_t*>(p)[i] = (f16_t)v;
}

constexpr float LOG2E = 1.44269504088896340736f;
// e^x by the hardware's 2^x (about 1 ulp of it; the product's rounding adds |x| 2^-24).  Results below 2^-126 are zero.
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }
constexpr float NEG_INF = -__builtin_inff();

}  // namespace isp_dev

static inline int isp_dtype_size(int dtype) { return dtype == ISP_F32 ? 4 : 2; }
