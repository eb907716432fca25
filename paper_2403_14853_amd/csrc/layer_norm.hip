// Layer norm over the rows of a dense matrix and its gradients (gfx950).
//   y = h w + bias,  h = (x - mean) rstd,  rstd = (mean (x - mean)^2 + eps)^-1/2
//   dx = rstd (g - mean g - h mean(g h)),  g = dy w;   dw = sum over the rows of dy h,  dbias = sum of dy
// Everything is held in 32 bits; outputs are rounded once, to the type of the matrix or the parameters.
//
// Memory-bound: a row is read once, kept in registers while its mean and then its centred squares are summed (no difference of large
// sums), and written once.  Up to 1024 columns lane groups hold whole rows (row_lanes.h), so that narrow rows leave no
// lane idle and need no barrier; up to 16384 a workgroup holds a row (the backward beyond 8192 columns spills 4 registers in fp32 and 38 in fp16:
// 4,096 x 16,384 170 us = 4.7 TB/s and 109 us = 3.7); beyond, it passes over the row again.
// The sums over the rows have one accumulator per lane and column while a workgroup passes over its rows; the workgroups' sums are
// rows of the workspace that a second launch adds, in a fixed order and in 64 bits.  No atomics: results repeat bit for bit.
#include "row_lanes.h"
#include "rowwise.h"

namespace {
using namespace isp_dev;

constexpr int LN_REG = 16;       // elements of a row per lane
constexpr int LN_GROUP = 1024;   // widest row that a lane group holds
constexpr int LN_BLOCK = 16384;  // widest row that a workgroup holds

struct ln_args {
  const void* x;
  int64_t ldx;
  const void* dy;
  int64_t lddy;
  int64_t n;
  int d;
  const void *w, *b;
  int param;
  float eps;
  void* y;  // (backward: dx)
  int64_t ldy;
  float *mean, *rstd;
  float* sums;  // backward: a row of dw and a row of dbias per workgroup, or NULL
};

template <class T, int VEC, int NV>
__device__ __forceinline__ void load_cols(const T* p, const int (&off)[NV], float (&o)[NV][VEC]) {
#pragma unroll
  for (int v = 0; v < NV; ++v) to_float<T, VEC>(load_raw<T, VEC>(p + off[v]), o[v]);
}
template <int VEC, int NV>
__device__ __forceinline__ void load_params(const void* p, int param, float none, const int (&off)[NV], float (&o)[NV][VEC]) {
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int c = 0; c < VEC; ++c) o[v][c] = p ? load_param(p, param, off[v] + c) : none;
}

// ---- rows in lane groups -----------------------------------------------------------------------------------------------
template <class T, int VEC, int LPR, int NV>
__global__ void __launch_bounds__(ISP_WG) k_ln_fwd(ln_args a) {
  constexpr int ROWS = ISP_WG / LPR;
  const int q = threadIdx.x % LPR;
  const row_cols<VEC, LPR, NV> rc(q, a.d);
  float w[NV][VEC], b[NV][VEC];
  load_params<VEC, NV>(a.w, a.param, 1.f, rc.off, w);
  load_params<VEC, NV>(a.b, a.param, 0.f, rc.off, b);
  const float inv = 1.f / (float)a.d;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR; row < a.n; row += step) {
    float x[NV][VEC];
    load_cols<T, VEC, NV>(static_cast<const T*>(a.x) + row * a.ldx, rc.off, x);
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int c = 0; c < VEC; ++c) s += rc.counts(v, c) ? x[v][c] : 0.f;
    const float mean = lanes_sum<LPR>(s) * inv;
    s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        x[v][c] -= mean;
        s += rc.counts(v, c) ? x[v][c] * x[v][c] : 0.f;
      }
    const float rstd = 1.f / sqrtf(lanes_sum<LPR>(s) * inv + a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int c = 0; c < VEC; ++c) x[v][c] = fmaf(x[v][c] * rstd, w[v][c], b[v][c]);
      if (rc.on[v]) store_raw<T, VEC>(static_cast<T*>(a.y) + row * a.ldy + rc.off[v], x[v]);
    }
    if (q == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

template <class T, int VEC, int LPR, int NV>
__global__ void __launch_bounds__(ISP_WG) k_ln_bwd(ln_args a) {
  constexpr int ROWS = ISP_WG / LPR;
  __shared__ float part[ISP_WAVES_PER_WG][2][LPR * NV * VEC];
  const int q = threadIdx.x % LPR;
  const row_cols<VEC, LPR, NV> rc(q, a.d);
  float w[NV][VEC], dw[NV][VEC], db[NV][VEC];
  load_params<VEC, NV>(a.w, a.param, 1.f, rc.off, w);
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int c = 0; c < VEC; ++c) dw[v][c] = db[v][c] = 0.f;
  const float inv = 1.f / (float)a.d;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR; row < a.n; row += step) {
    float x[NV][VEC], g[NV][VEC];
    load_cols<T, VEC, NV>(static_cast<const T*>(a.x) + row * a.ldx, rc.off, x);
    load_cols<T, VEC, NV>(static_cast<const T*>(a.dy) + row * a.lddy, rc.off, g);
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        x[v][c] = (x[v][c] - mean) * rstd;
        dw[v][c] = fmaf(g[v][c], x[v][c], dw[v][c]);
        db[v][c] += g[v][c];
        g[v][c] *= w[v][c];
        s1 += rc.counts(v, c) ? g[v][c] : 0.f;
        s2 += rc.counts(v, c) ? g[v][c] * x[v][c] : 0.f;
      }
    if (a.y) {
      s1 = lanes_sum<LPR>(s1) * inv;
      s2 = lanes_sum<LPR>(s2) * inv;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int c = 0; c < VEC; ++c) g[v][c] = (g[v][c] - s1 - x[v][c] * s2) * rstd;
        if (rc.on[v]) store_raw<T, VEC>(static_cast<T*>(a.y) + row * a.ldy + rc.off[v], g[v]);
      }
    }
  }
  if (!a.sums) return;
  // the wavefront's groups, then the workgroup's wavefronts
  const int lane = threadIdx.x & (ISP_WAVE - 1), wave = threadIdx.x >> 6;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
#pragma unroll
      for (int o = LPR; o < ISP_WAVE; o <<= 1) {
        dw[v][c] += __shfl_xor(dw[v][c], o);
        db[v][c] += __shfl_xor(db[v][c], o);
      }
      if (lane < LPR) {
        part[wave][0][(v * LPR + q) * VEC + c] = dw[v][c];
        part[wave][1][(v * LPR + q) * VEC + c] = db[v][c];
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.d; i += ISP_WG) {
    const int which = i >= a.d, col = which ? i - a.d : i;
    const int full = col / VEC * VEC;  // (a moved-back vector's elements sit dup places further on)
    const int at = full + VEC > a.d ? col + (full + VEC - a.d) : col;
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < ISP_WAVES_PER_WG; ++k) t += part[k][which][at];
    a.sums[(int64_t)blockIdx.x * 2 * a.d + i] = t;
  }
}

// ---- a row per workgroup -------------------------------------------------------------------------------------------------
template <class T, int VEC, int BT, int NV>
__global__ void __launch_bounds__(BT) k_ln_fwd_wide(ln_args a) {
  __shared__ float buf[2][2 * BT / ISP_WAVE];
  const row_cols<VEC, BT, NV> rc(threadIdx.x, a.d);
  float w[NV][VEC], b[NV][VEC];
  load_params<VEC, NV>(a.w, a.param, 1.f, rc.off, w);
  load_params<VEC, NV>(a.b, a.param, 0.f, rc.off, b);
  const float inv = 1.f / (float)a.d;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x, turn ^= 1) {
    float x[NV][VEC];
    load_cols<T, VEC, NV>(static_cast<const T*>(a.x) + row * a.ldx, rc.off, x);
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int c = 0; c < VEC; ++c) s[0] += rc.counts(v, c) ? x[v][c] : 0.f;
    block_sums<1, BT>(s, buf[0], turn);
    const float mean = s[0] * inv;
    s[0] = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        x[v][c] -= mean;
        s[0] += rc.counts(v, c) ? x[v][c] * x[v][c] : 0.f;
      }
    block_sums<1, BT>(s, buf[1], turn);
    const float rstd = 1.f / sqrtf(s[0] * inv + a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int c = 0; c < VEC; ++c) x[v][c] = fmaf(x[v][c] * rstd, w[v][c], b[v][c]);
      if (rc.on[v]) store_raw<T, VEC>(static_cast<T*>(a.y) + row * a.ldy + rc.off[v], x[v]);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

template <class T, int VEC, int BT, int NV>
__global__ void __launch_bounds__(BT) k_ln_bwd_wide(ln_args a) {
  __shared__ float buf[2 * 2 * BT / ISP_WAVE];
  const row_cols<VEC, BT, NV> rc(threadIdx.x, a.d);
  float w[NV][VEC], dw[NV][VEC], db[NV][VEC];
  load_params<VEC, NV>(a.w, a.param, 1.f, rc.off, w);
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int c = 0; c < VEC; ++c) dw[v][c] = db[v][c] = 0.f;
  const float inv = 1.f / (float)a.d;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x, turn ^= 1) {
    float x[NV][VEC], g[NV][VEC];
    load_cols<T, VEC, NV>(static_cast<const T*>(a.x) + row * a.ldx, rc.off, x);
    load_cols<T, VEC, NV>(static_cast<const T*>(a.dy) + row * a.lddy, rc.off, g);
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        x[v][c] = (x[v][c] - mean) * rstd;
        dw[v][c] = fmaf(g[v][c], x[v][c], dw[v][c]);
        db[v][c] += g[v][c];
        g[v][c] *= w[v][c];
        s[0] += rc.counts(v, c) ? g[v][c] : 0.f;
        s[1] += rc.counts(v, c) ? g[v][c] * x[v][c] : 0.f;
      }
    if (a.y) {
      block_sums<2, BT>(s, buf, turn);
      s[0] *= inv;
      s[1] *= inv;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int c = 0; c < VEC; ++c) g[v][c] = (g[v][c] - s[0] - x[v][c] * s[1]) * rstd;
        if (rc.on[v]) store_raw<T, VEC>(static_cast<T*>(a.y) + row * a.ldy + rc.off[v], g[v]);
      }
    }
  }
  if (!a.sums) return;
  float* o = a.sums + (int64_t)blockIdx.x * 2 * a.d;
#pragma unroll
  for (int v = 0; v < NV; ++v)
    if (rc.on[v]) {
      store_raw<float, VEC>(o + rc.off[v], dw[v]);
      store_raw<float, VEC>(o + a.d + rc.off[v], db[v]);
    }
}

// ---- rows wider than a workgroup holds: passes over the row -----------------------------------------------------------------
template <class T, int BT>
__global__ void __launch_bounds__(BT) k_ln_fwd_any(ln_args a) {
  __shared__ float buf[2][2 * BT / ISP_WAVE];
  const float inv = 1.f / (float)a.d;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x, turn ^= 1) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    float s[1] = {0.f};
#pragma unroll 8
    for (int c = threadIdx.x; c < a.d; c += BT) s[0] += (float)x[c];
    block_sums<1, BT>(s, buf[0], turn);
    const float mean = s[0] * inv;
    s[0] = 0.f;
#pragma unroll 8
    for (int c = threadIdx.x; c < a.d; c += BT) {
      const float t = (float)x[c] - mean;
      s[0] += t * t;
    }
    block_sums<1, BT>(s, buf[1], turn);
    const float rstd = 1.f / sqrtf(s[0] * inv + a.eps);
#pragma unroll 4
    for (int c = threadIdx.x; c < a.d; c += BT) {
      const float w = a.w ? load_param(a.w, a.param, c) : 1.f, b = a.b ? load_param(a.b, a.param, c) : 0.f;
      y[c] = (T)fmaf(((float)x[c] - mean) * rstd, w, b);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

template <class T, int BT>
__global__ void __launch_bounds__(BT) k_ln_bwd_any(ln_args a) {
  __shared__ float buf[2 * 2 * BT / ISP_WAVE];
  const float inv = 1.f / (float)a.d;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x, turn ^= 1) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    T* dx = static_cast<T*>(a.y) + row * a.ldy;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s[2] = {0.f, 0.f};
#pragma unroll 4
    for (int c = threadIdx.x; c < a.d; c += BT) {
      const float h = ((float)x[c] - mean) * rstd, g = (float)dy[c] * (a.w ? load_param(a.w, a.param, c) : 1.f);
      s[0] += g;
      s[1] = fmaf(g, h, s[1]);
    }
    block_sums<2, BT>(s, buf, turn);
    s[0] *= inv;
    s[1] *= inv;
#pragma unroll 4
    for (int c = threadIdx.x; c < a.d; c += BT) {
      const float h = ((float)x[c] - mean) * rstd, g = (float)dy[c] * (a.w ? load_param(a.w, a.param, c) : 1.f);
      dx[c] = (T)((g - s[0] - h * s[1]) * rstd);
    }
  }
}
// workgroup (i, r): columns [i * BT, (i + 1) * BT) of the rows r, r + gridDim.y, ...
template <class T, int BT>
__global__ void __launch_bounds__(BT) k_ln_sums_any(ln_args a) {
  const int c = blockIdx.x * BT + threadIdx.x;
  if (c >= a.d) return;
  float dw = 0.f, db = 0.f;
#pragma unroll 4
  for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
    const float h = ((float)static_cast<const T*>(a.x)[row * a.ldx + c] - a.mean[row]) * a.rstd[row];
    const float g = (float)static_cast<const T*>(a.dy)[row * a.lddy + c];
    dw = fmaf(g, h, dw);
    db += g;
  }
  a.sums[(int64_t)blockIdx.y * 2 * a.d + c] = dw;
  a.sums[((int64_t)blockIdx.y * 2 + 1) * a.d + c] = db;
}

// The workgroups' rows of sums, added up: 16 columns per workgroup (from column col0 of dw's and dbias's on), 64 threads to a column, each a run of
// consecutive rows.
constexpr int LN_COLS = 16, LN_RUNS = 64;
__global__ void __launch_bounds__(LN_COLS* LN_RUNS) k_ln_sums(const float* __restrict__ sums, int rows, int d, void* dw, void* db, int param, int64_t col0) {
  __shared__ double part[LN_RUNS][LN_COLS];
  const int c = threadIdx.x % LN_COLS, r = threadIdx.x / LN_COLS;
  const int64_t col = col0 + (int64_t)blockIdx.x * LN_COLS + c, cols = 2 * (int64_t)d;
  const int per = (rows + LN_RUNS - 1) / LN_RUNS;
  const int lo = r * per, hi = lo + per < rows ? lo + per : rows;
  double s = 0.;
  if (col < cols)
#pragma unroll 8
    for (int i = lo; i < hi; ++i) s += (double)sums[i * cols + col];
  part[r][c] = s;
  __syncthreads();
  if (r == 0 && col < cols) {
    double t = 0.;
#pragma unroll
    for (int i = 0; i < LN_RUNS; ++i) t += part[i][c];
    if (col < d) {
      if (dw) store_param(dw, param, col, (float)t);
    } else if (db) {
      store_param(db, param, col - d, (float)t);
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------
// Workgroups of the backward pass (its rows of sums): as many as there are rows for, up to four per compute unit in lane groups, two or one where a
// workgroup holds a row, whose sums take as much memory as eight rows of an fp32 matrix per workgroup.
int64_t ln_bwd_groups(int64_t n, int d) {
  if (d <= LN_GROUP) {
    const int64_t rows = ISP_WG / isp_row_lanes(d, 8);  // (of the type with the widest vectors; a bound for both)
    const int64_t g = isp_ceil_div(n, rows);
    return g < 1024 ? g : 1024;
  }
  const int64_t most = d <= 4096 ? 512 : d <= LN_BLOCK ? 256 : 64;
  return n < most ? n : most;
}

template <class T, int VEC, int LPR, int NV>
void ln_group(const ln_args& a, bool bwd, hipStream_t s) {
  const int64_t rows = ISP_WG / LPR;
  if (!bwd) {
    const int64_t g = isp_ceil_div(a.n, rows);
    k_ln_fwd<T, VEC, LPR, NV><<<(unsigned)(g < 4096 ? g : 4096), ISP_WG, 0, s>>>(a);
  } else {
    k_ln_bwd<T, VEC, LPR, NV><<<(unsigned)ln_bwd_groups(a.n, a.d), ISP_WG, 0, s>>>(a);
  }
}
template <class T, int VEC, int BT, int NV>
void ln_wide(const ln_args& a, bool bwd, hipStream_t s) {
  if (!bwd) k_ln_fwd_wide<T, VEC, BT, NV><<<(unsigned)(a.n < 2048 ? a.n : 2048), BT, 0, s>>>(a);
  else k_ln_bwd_wide<T, VEC, BT, NV><<<(unsigned)ln_bwd_groups(a.n, a.d), BT, 0, s>>>(a);
}
template <class T>
void ln_run(const ln_args& a, bool bwd, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(T), MAX = LN_REG / VEC;
  if (a.d < VEC) return ln_group<T, 1, 8, 1>(a, bwd, s);
  if (a.d <= LN_GROUP) {
    switch (isp_row_lanes(a.d, VEC)) {
      case 4: return ln_group<T, VEC, 4, 1>(a, bwd, s);
      case 8: return ln_group<T, VEC, 8, 1>(a, bwd, s);
      case 16: return ln_group<T, VEC, 16, 1>(a, bwd, s);
      case 32: return ln_group<T, VEC, 32, 1>(a, bwd, s);
    }
    if (a.d <= ISP_WAVE * VEC) return ln_group<T, VEC, 64, 1>(a, bwd, s);
    if (MAX == 2 || a.d <= ISP_WAVE * VEC * 2) return ln_group<T, VEC, 64, 2>(a, bwd, s);
    return ln_group<T, VEC, 64, MAX>(a, bwd, s);
  }
  if (a.d <= 256 * VEC * (MAX / 2)) return ln_wide<T, VEC, 256, MAX / 2>(a, bwd, s);
  if (a.d <= 256 * VEC * MAX) return ln_wide<T, VEC, 256, MAX>(a, bwd, s);
  if (a.d <= 1024 * VEC * (MAX / 2)) return ln_wide<T, VEC, 1024, MAX / 2>(a, bwd, s);
  if (a.d <= LN_BLOCK) return ln_wide<T, VEC, 1024, MAX>(a, bwd, s);
  const unsigned g = (unsigned)(a.n < 2048 ? a.n : 2048);
  if (!bwd) {
    k_ln_fwd_any<T, 1024><<<g, 1024, 0, s>>>(a);
    return;
  }
  if (a.y) k_ln_bwd_any<T, 1024><<<g, 1024, 0, s>>>(a);
  if (a.sums) k_ln_sums_any<T, 256><<<dim3((unsigned)isp_ceil_div(a.d, 256), (unsigned)ln_bwd_groups(a.n, a.d)), 256, 0, s>>>(a);
}
void ln_dispatch(const ln_args& a, int dtype, bool bwd, hipStream_t s) {
  if (dtype == ISP_F32) ln_run<float>(a, bwd, s);
  else if (dtype == ISP_BF16) ln_run<bf16_t>(a, bwd, s);
  else ln_run<f16_t>(a, bwd, s);
}

}  // namespace

size_t isp_layer_norm_sums_bytes(int64_t n, int32_t d) { return isp_align((size_t)ln_bwd_groups(n, d) * 2 * (size_t)d * sizeof(float)); }

isp_status isp_layer_norm_launch(const void* X, int64_t ldx, int64_t n, int32_t d, int dtype, const void* weight, const void* bias, int param,
                                 float eps, void* Y, int64_t ldy, float* mean, float* rstd, hipStream_t s) {
  if (n == 0) return ISP_OK;
  ln_args a{X, ldx, nullptr, 0, n, d, weight, bias, param, eps, Y, ldy, mean, rstd, nullptr};
  ln_dispatch(a, dtype, false, s);
  ISP_LAUNCH_CHECK();
  return ISP_OK;
}

isp_status isp_layer_norm_bwd_launch(const void* X, int64_t ldx, const void* dY, int64_t lddy, int64_t n, int32_t d, int dtype, const void* weight,
                                     int param, const float* mean, const float* rstd, void* dX, int64_t lddx, void* dweight, void* dbias, void* ws,
                                     hipStream_t s) {
  const bool sums = dweight || dbias;
  if (n > 0 && (dX || sums)) {
    ln_args a{X, ldx, dY, lddy, n, d, weight, nullptr, param, 0.f, dX, lddx, const_cast<float*>(mean), const_cast<float*>(rstd),
              sums ? static_cast<float*>(ws) : nullptr};
    ln_dispatch(a, dtype, true, s);
    ISP_LAUNCH_CHECK();
  }
  if (sums) {  // (of no rows: zeros)
    const int rows = n > 0 ? (int)ln_bwd_groups(n, d) : 0;
    constexpr int64_t MOST = (1ll << 31) / LN_RUNS;  // columns of a launch, which has to stay below 2^32 threads
    for (int64_t c0 = 0, cols = 2 * (int64_t)d; c0 < cols; c0 += MOST) {
      const int64_t some = cols - c0 < MOST ? cols - c0 : MOST;
      k_ln_sums<<<(unsigned)isp_ceil_div(some, LN_COLS), LN_COLS * LN_RUNS, 0, s>>>(static_cast<const float*>(ws), rows, d, dweight, dbias, param, c0);
    }
    ISP_LAUNCH_CHECK();
  }
  return ISP_OK;
}
