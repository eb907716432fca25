// Log probabilities of given labels over the rows of a score matrix, with entropy and the top alternatives, and their gradient (gfx950).
//   m = max z, T = sum exp(z - m), U = sum exp(z - m) (z - m)
//   log p_j = (z_j - m) - log T;   S = -sum p log p = log T - U / T  (both terms are positive: nothing cancels)
//   dz_j = a (1[j = label] - p_j) - e p_j (log p_j + S),  a, e the upstream gradients of log p_label and S
// One pass over the scores, in 32 bits: rows of up to 1024 scores lie in the registers of a lane group (row_lanes.h); longer ones are streamed
// with a running maximum per lane, to which T and U are rescaled once per 16 scores, by a wavefront, by the eight of a
// workgroup, or, where there are few rows, by several workgroups whose parts a second launch joins.  Ten vector
// instructions per score, an exponential among them, keep pace with the loads of long rows (2,053 x 65,521, bf16: 80 us = 3.4 TB/s, vector ALU 41 % busy).
// On rows of tens of scores the sums over lanes and the row's end come to as much again (21 per score), and the vector ALU bounds the forward (2.45 M x 47,
// bf16: 102 us, 63 % busy at 2.9 TB/s of misses); the backward is bound by memory (129 us, 4.2 TB/s).
// What a row holds decides: -inf is a class left out (p = 0); a row with nothing left has log probabilities of -inf, entropy 0 and no gradient;
// NaN and +inf make the row's results NaN.
//
// The top alternatives are ordered by score, then by index: a score's bits, made to order like unsigned numbers (-0 as 0, NaN above all), and
// the index's complement make one key of 64 bits.  A wavefront keeps the best `top` keys it has met in order, one per lane; of a
// tile of scores only those above the last of them are looked at, which is few after the first tiles.
#include "row_lanes.h"
#include "rowwise.h"

namespace {
using namespace isp_dev;

typedef unsigned long long u64;

constexpr int LP_GROUP = 1024;              // longest row that a lane group holds
constexpr int LP_WAVES = 8;                 // wavefronts per workgroup of the streaming kernel
constexpr int LP_TILE = 1024;               // scores that a wavefront takes at a time
constexpr int LP_CHUNK = LP_WAVES * LP_TILE;

struct lp_args {
  const void* z;
  int64_t ldz, n;
  int classes;
  const int64_t* labels;
  float *logprob, *entropy, *stats;  // stats: (m, log T) of each row
  int top;
  float* top_logprob;
  int32_t* top_index;
  int splits;   // workgroups per row
  float* part;  // of each: m, T, U, and its keys behind all of those
};

__device__ __forceinline__ unsigned order_bits(float x) {
  const unsigned b = __float_as_uint(x + 0.f);  // (-0 becomes 0)
  return x != x ? 0xffffffffu : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_order_bits(unsigned k) {
  return __uint_as_float(k == 0xffffffffu ? 0x7fc00000u : k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ u64 key_of(unsigned bits, int index) { return (u64)bits << 32 | (unsigned)~index; }
__device__ __forceinline__ unsigned max_u(unsigned a, unsigned b) { return a > b ? a : b; }
template <int CTRL>
__device__ __forceinline__ unsigned dpp_u(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }
// The maximum over LPR consecutive lanes (4 and more), in all of them.
template <int LPR>
__device__ __forceinline__ unsigned lanes_max_u(unsigned v) {
  v = max_u(v, dpp_u<DPP_XOR1>(v));
  v = max_u(v, dpp_u<DPP_XOR2>(v));
  if constexpr (LPR >= 8) v = max_u(v, dpp_u<DPP_HALF_MIRROR>(v));
  if constexpr (LPR >= 16) v = max_u(v, dpp_u<DPP_ROR8>(v));
  if constexpr (LPR >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max_u(r[0], r[1]);
  }
  if constexpr (LPR >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max_u(r[0], r[1]);
  }
  return v;
}
// of keys: the greatest score first, then, among the lanes that have it, the lowest index
template <int LPR>
__device__ __forceinline__ u64 lanes_max_key(u64 k) {
  const unsigned hi = lanes_max_u<LPR>((unsigned)(k >> 32));
  const unsigned lo = lanes_max_u<LPR>((unsigned)(k >> 32) == hi ? (unsigned)k : 0u);
  return (u64)hi << 32 | lo;
}

// The running sums of some scores: m their maximum (-inf: none counts yet).
struct lp_sums {
  float m, t, u;
};
// rescaled to the maximum `to`, which is m or above
__device__ __forceinline__ lp_sums lp_rescale(const lp_sums& s, float to) {
  const float gap = s.m == NEG_INF || s.m == to ? 0.f : s.m - to;  // (nothing counts: t = u = 0)
  const float f = fast_exp(gap);
  return {to, s.t * f, f > 0.f ? f * fmaf(s.t, gap, s.u) : 0.f};  // (a gap as wide as the type's range times t is -inf)
}
__device__ __forceinline__ lp_sums lp_join(const lp_sums& a, const lp_sums& b) {
  const float m = fmaxf(a.m, b.m);
  const lp_sums x = lp_rescale(a, m), y = lp_rescale(b, m);
  return {m, x.t + y.t, x.u + y.u};
}
// scores of at most s.m
template <int N>
__device__ __forceinline__ void lp_add_to(lp_sums& s, const float (&z)[N]) {
  const float base = s.m == NEG_INF ? 0.f : s.m;
  float t[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};  // (short sums first: a long row's errors stay small)
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const float g = z[c] - base, e = fast_exp(g);
    t[c % 4] += e;
    u[c % 4] = fmaf(e, fmaxf(g, -3e38f), u[c % 4]);  // (e = 0 where g = -inf; a NaN is in e already)
  }
  s.t += (t[0] + t[1]) + (t[2] + t[3]);
  s.u += (u[0] + u[1]) + (u[2] + u[3]);
}
template <int N>
__device__ __forceinline__ void lp_add(lp_sums& s, const float (&z)[N]) {
  float m = s.m;
#pragma unroll
  for (int c = 0; c < N; ++c) m = fmaxf(m, z[c]);
  s = lp_rescale(s, m);
  lp_add_to(s, z);
}

constexpr float LN2 = 0.693147180559945309f;
// (the hardware's base-2 logarithm and reciprocal, about 1 ulp each: t is 1 or more)
struct lp_row {
  float m, log_t;
  bool empty;
  __device__ __forceinline__ lp_row(const lp_sums& s) : m(s.m), log_t(__builtin_amdgcn_logf(s.t) * LN2), empty(s.t == 0.f) {}
  __device__ __forceinline__ float logprob(float z) const { return empty ? NEG_INF : (z - m) - log_t; }
};
// one lane per row
template <class T>
__device__ __forceinline__ void lp_store(const lp_args& a, int64_t row, const lp_sums& s, const lp_row& r) {
  if (a.logprob) {
    const int64_t y = a.labels[row];
    a.logprob[row] = y >= 0 && y < a.classes ? r.logprob((float)static_cast<const T*>(a.z)[row * a.ldz + y]) : 0.f;
  }
  if (a.entropy) a.entropy[row] = r.empty ? 0.f : r.log_t - s.u * __builtin_amdgcn_rcpf(s.t);
  if (a.stats) {
    a.stats[2 * row] = r.m;
    a.stats[2 * row + 1] = r.log_t;
  }
}
__device__ __forceinline__ void lp_store_top(const lp_args& a, int64_t row, int place, u64 key, const lp_row& r) {
  const float z = from_order_bits((unsigned)(key >> 32));
  if (a.top_logprob) a.top_logprob[row * a.top + place] = r.logprob(z);
  if (a.top_index) a.top_index[row * a.top + place] = (int32_t)~(unsigned)key;
}

// ---- rows in lane groups ---------------------------------------------------------------------------------------------
template <class T, int VEC, int LPR, int NV, bool TOP>
__global__ void __launch_bounds__(ISP_WG) k_lp_group(lp_args a) {
  constexpr int ROWS = ISP_WG / LPR;
  const int q = threadIdx.x % LPR;
  const row_cols<VEC, LPR, NV> rc(q, a.classes);
  const int64_t step = (int64_t)gridDim.x * ROWS;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR; row < a.n; row += step) {
    float z[NV * VEC];
    const T* p = static_cast<const T*>(a.z) + row * a.ldz;
    float m = NEG_INF;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float t[VEC];
      to_float<T, VEC>(load_raw<T, VEC>(p + rc.off[v]), t);
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        z[v * VEC + c] = rc.counts(v, c) ? t[c] : NEG_INF;
        m = fmaxf(m, z[v * VEC + c]);
      }
    }
    lp_sums s{lanes_max<LPR>(m), 0.f, 0.f};
    lp_add_to(s, z);
    s.t = lanes_sum<LPR>(s.t);
    s.u = lanes_sum<LPR>(s.u);
    const lp_row r(s);
    if (q == 0) lp_store<T>(a, row, s, r);
    if constexpr (TOP) {
      unsigned bits[NV * VEC];
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int c = 0; c < VEC; ++c) bits[v * VEC + c] = rc.counts(v, c) ? order_bits(z[v * VEC + c]) : 0u;
      for (int k = 0; k < a.top; ++k) {
        u64 mine = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int c = 0; c < VEC; ++c) {
            const u64 key = bits[v * VEC + c] ? key_of(bits[v * VEC + c], rc.off[v] + c) : 0;
            mine = key > mine ? key : mine;
          }
        const u64 best = lanes_max_key<LPR>(mine);
        if (mine == best && best) {
          lp_store_top(a, row, k, best, r);
          const int at = (int)~(unsigned)best;
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int c = 0; c < VEC; ++c)
              if (rc.off[v] + c == at && rc.counts(v, c)) bits[v * VEC + c] = 0;
        }
      }
    }
  }
}

// ---- rows streamed by wavefronts -----------------------------------------------------------------------------------------
// The best keys that a wavefront has met, in order: lane i holds the i-th (0: none yet).
struct lp_list {
  u64 key = 0;
  __device__ __forceinline__ u64 last(int top) const {  // (top is wave-uniform)
    const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)(key >> 32), top - 1), lo = (unsigned)__builtin_amdgcn_readlane((int)key, top - 1);
    return (u64)hi << 32 | lo;
  }
  __device__ __forceinline__ void insert(u64 x, int lane) {
    const u64 before = __shfl_up(key, 1);
    key = key > x ? key : lane == 0 || before > x ? x : before;
  }
  // N keys per lane
  template <int N>
  __device__ __forceinline__ void merge(u64 (&mine)[N], int top, int lane) {
    for (;;) {
      u64 m = mine[0];
#pragma unroll
      for (int i = 1; i < N; ++i) m = mine[i] > m ? mine[i] : m;
      const u64 best = lanes_max_key<ISP_WAVE>(m);
      if (best <= last(top)) break;
      insert(best, lane);
#pragma unroll
      for (int i = 0; i < N; ++i) mine[i] = mine[i] == best ? 0 : mine[i];
    }
  }
};

// A tile as it lies in memory: scores behind the row's end as -inf.
template <class T>
struct lp_tile {
  static constexpr int VEC = 16 / sizeof(T), NV = 16 / VEC;
  raw_t<T, VEC> raw[NV];
  __device__ __forceinline__ void load(const T* p, int at, int end, int lane) {
    if (at + LP_TILE <= end) {
#pragma unroll
      for (int v = 0; v < NV; ++v) raw[v] = load_raw<T, VEC>(p + at + (v * ISP_WAVE + lane) * VEC);
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
          const int i = at + (v * ISP_WAVE + lane) * VEC + c;
          raw[v][c] = i < end ? p[i] : (T)NEG_INF;
        }
    }
  }
  __device__ __forceinline__ void get(float (&z)[16]) const {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float t[VEC];
      to_float<T, VEC>(raw[v], t);
#pragma unroll
      for (int c = 0; c < VEC; ++c) z[v * VEC + c] = t[c];
    }
  }
};

// WPR wavefronts to a row: 1, or all of the workgroup's.
template <class T, int WPR, bool TOP>
__global__ void __launch_bounds__(LP_WAVES* ISP_WAVE) k_lp_stream(lp_args a) {
  constexpr int VEC = 16 / sizeof(T);
  __shared__ float sums[LP_WAVES][3];
  __shared__ u64 keys[LP_WAVES][ISP_WAVE];
  __shared__ unsigned floor_bits;
  const int lane = threadIdx.x & (ISP_WAVE - 1), w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t row = WPR == 1 ? (int64_t)blockIdx.x * LP_WAVES + w : (int64_t)(blockIdx.x / (unsigned)a.splits);
  if (row >= a.n) return;  // (the whole workgroup, or a wavefront that meets no barrier)
  const T* p = static_cast<const T*>(a.z) + row * a.ldz;
  const int first = WPR == 1 ? 0 : (int)(blockIdx.x % (unsigned)a.splits) * LP_WAVES + w, stride = WPR == 1 ? 1 : a.splits * LP_WAVES;
  const int tiles = (a.classes + LP_TILE - 1) / LP_TILE;
  if constexpr (TOP && WPR > 1) {
    if (threadIdx.x == 0) floor_bits = 0u;
    __syncthreads();
  }
  lp_sums s{NEG_INF, 0.f, 0.f};
  lp_list list;
  unsigned last = 0;  // the score bits of the list's last key
  lp_tile<T> next;
  if (first < tiles) next.load(p, first * LP_TILE, a.classes, lane);
  for (int tile = first; tile < tiles; tile += stride) {
    float z[16];
    next.get(z);
    if (tile + stride < tiles) next.load(p, (tile + stride) * LP_TILE, a.classes, lane);  // (on its way while this one is worked on)
    lp_add(s, z);
    if constexpr (TOP) {
      float m = NEG_INF;
#pragma unroll
      for (int c = 0; c < 16; ++c) m = fmaxf(m, z[c]);
      const unsigned low = WPR > 1 ? __hip_atomic_load(&floor_bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) : 0u;  // (what a wavefront of the row has `top` keys from is enough for all of them)
      const unsigned mb = order_bits(m);
      // (s.t: once a NaN has come by every tile is looked at)
      if (__any((mb > last && mb >= low) || s.t != s.t)) {
        unsigned bits[16];
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          const int i = tile * LP_TILE + (c / VEC * ISP_WAVE + lane) * VEC + c % VEC;
          bits[c] = i < a.classes ? order_bits(z[c]) : 0u;
        }
        for (;;) {
          unsigned mine = bits[0];
#pragma unroll
          for (int c = 1; c < 16; ++c) mine = max_u(mine, bits[c]);
          const unsigned hi = lanes_max_u<ISP_WAVE>(mine);
          if (hi == 0 || hi <= last || hi < low) break;  // (later scores that equal the list's last come after it)
          int at = 0;
#pragma unroll
          for (int c = 15; c >= 0; --c) at = bits[c] == hi ? c : at;
          const int index = tile * LP_TILE + (at / VEC * ISP_WAVE + lane) * VEC + at % VEC;
          const unsigned lo = lanes_max_u<ISP_WAVE>(mine == hi ? (unsigned)~index : 0u);
          list.insert((u64)hi << 32 | lo, lane);
          last = (unsigned)(list.last(a.top) >> 32);
          if (mine == hi && (unsigned)~index == lo) {
#pragma unroll
            for (int c = 0; c < 16; ++c) bits[c] = c == at ? 0u : bits[c];
          }
        }
        if (WPR > 1 && lane == 0 && last > low) atomicMax(&floor_bits, last);
      }
    }
  }
  // the lanes, then the wavefronts
  {
    const float m = lanes_max<ISP_WAVE>(s.m);
    s = lp_rescale(s, m);
    s.t = lanes_sum<ISP_WAVE>(s.t);
    s.u = lanes_sum<ISP_WAVE>(s.u);
  }
  if constexpr (WPR > 1) {
    if (lane == 0) {
      sums[w][0] = s.m;
      sums[w][1] = s.t;
      sums[w][2] = s.u;
    }
    if constexpr (TOP) keys[w][lane] = lane < a.top ? list.key : 0;
    __syncthreads();
    if (w > 0) return;
    // (eight lanes have a wavefront's sums each, the others nothing)
    s = lane < LP_WAVES ? lp_sums{sums[lane][0], sums[lane][1], sums[lane][2]} : lp_sums{NEG_INF, 0.f, 0.f};
    const float m = lanes_max<ISP_WAVE>(s.m);
    s = lp_rescale(s, m);
    s.t = lanes_sum<ISP_WAVE>(s.t);
    s.u = lanes_sum<ISP_WAVE>(s.u);
    if constexpr (TOP) {
      u64 mine[LP_WAVES];
#pragma unroll
      for (int i = 0; i < LP_WAVES; ++i) mine[i] = keys[i][lane];
      list = lp_list();
      list.merge(mine, a.top, lane);
    }
    if (a.splits > 1) {
      float* o = a.part + 3 * (int64_t)blockIdx.x;
      if (lane == 0) {
        o[0] = s.m;
        o[1] = s.t;
        o[2] = s.u;
      }
      if (TOP && lane < a.top) {
        u64* k = reinterpret_cast<u64*>(a.part + (3 * a.n * a.splits + 1) / 2 * 2);
        k[(int64_t)blockIdx.x * a.top + lane] = list.key;
      }
      return;
    }
  }
  const lp_row r(s);
  if (lane == 0) lp_store<T>(a, row, s, r);
  if (TOP && lane < a.top) lp_store_top(a, row, lane, list.key, r);
}

// The workgroups' parts of a row, joined by a wavefront.
template <class T, bool TOP>
__global__ void __launch_bounds__(ISP_WAVE) k_lp_join(lp_args a) {
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  const float* o = a.part + 3 * row * a.splits;
  lp_sums s{NEG_INF, 0.f, 0.f};
  for (int i = lane; i < a.splits; i += ISP_WAVE) s = lp_join(s, {o[3 * i], o[3 * i + 1], o[3 * i + 2]});
  const float m = lanes_max<ISP_WAVE>(s.m);
  s = lp_rescale(s, m);
  s.t = lanes_sum<ISP_WAVE>(s.t);
  s.u = lanes_sum<ISP_WAVE>(s.u);
  const lp_row r(s);
  if (lane == 0) lp_store<T>(a, row, s, r);
  if constexpr (TOP) {
    const u64* k = reinterpret_cast<const u64*>(a.part + (3 * a.n * a.splits + 1) / 2 * 2) + row * a.splits * a.top;
    lp_list list;
    const int n = a.splits * a.top;
    for (int i = 0; i < n; i += 4 * ISP_WAVE) {
      u64 mine[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) mine[j] = i + j * ISP_WAVE + lane < n ? k[i + j * ISP_WAVE + lane] : 0;
      list.merge(mine, a.top, lane);
    }
    if (lane < a.top) lp_store_top(a, row, lane, list.key, r);
  }
}

// ---- gradient ------------------------------------------------------------------------------------------------------------
struct lp_bwd_args {
  const void* z;
  int64_t ldz, n;
  int classes;
  const int64_t* labels;
  const float *stats, *entropy, *da, *de;
  void* dz;
  int64_t lddz;
  int chunks;  // of a long row
};
struct lp_grad {
  float m, log_t, a, e, s;
  int label;  // -1: none
  bool none;  // the row has no gradient
  __device__ __forceinline__ lp_grad(const lp_bwd_args& g, int64_t row) {
    const int64_t y = g.da ? g.labels[row] : -1;
    label = y >= 0 && y < g.classes ? (int)y : -1;
    a = label >= 0 ? g.da[row] : 0.f;
    e = g.de ? g.de[row] : 0.f;
    m = g.stats[2 * row];
    log_t = g.stats[2 * row + 1];
    s = g.de ? g.entropy[row] : 0.f;
    none = (a == 0.f && e == 0.f) || log_t == NEG_INF;
  }
  __device__ __forceinline__ float of(float z, int j) const {
    const float lp = (z - m) - log_t, p = fast_exp(lp);
    return a * ((j == label ? 1.f : 0.f) - p) - e * p * (fmaxf(lp, -3e38f) + s);  // (p = 0 where lp = -inf)
  }
};

template <class T, int VEC, int LPR, int NV>
__global__ void __launch_bounds__(ISP_WG) k_lp_group_bwd(lp_bwd_args g) {
  constexpr int ROWS = ISP_WG / LPR;
  const row_cols<VEC, LPR, NV> rc(threadIdx.x % LPR, g.classes);
  const int64_t step = (int64_t)gridDim.x * ROWS;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR; row < g.n; row += step) {
    const lp_grad r(g, row);
    const T* p = static_cast<const T*>(g.z) + row * g.ldz;
    T* o = static_cast<T*>(g.dz) + row * g.lddz;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float t[VEC];
#pragma unroll
      for (int c = 0; c < VEC; ++c) t[c] = 0.f;
      if (!r.none) {
        to_float<T, VEC>(load_raw<T, VEC>(p + rc.off[v]), t);
#pragma unroll
        for (int c = 0; c < VEC; ++c) t[c] = r.of(t[c], rc.off[v] + c);
      }
      if (rc.on[v]) store_raw<T, VEC>(o + rc.off[v], t);
    }
  }
}

// A workgroup per chunk of 16 scores a thread.
template <class T>
__global__ void __launch_bounds__(ISP_WG) k_lp_chunk_bwd(lp_bwd_args g) {
  constexpr int VEC = 16 / sizeof(T), NV = 16 / VEC;
  const int64_t total = g.n * g.chunks;
  for (int64_t b = blockIdx.x; b < total; b += gridDim.x) {
    const int64_t row = b / g.chunks;
    const int c0 = (int)(b - row * g.chunks) * ISP_WG * 16;
    const lp_grad r(g, row);
    const T* p = static_cast<const T*>(g.z) + row * g.ldz;
    T* o = static_cast<T*>(g.dz) + row * g.lddz;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      int at = c0 + (v * ISP_WG + (int)threadIdx.x) * VEC;
      if (at >= g.classes) continue;
      if (at + VEC > g.classes) at = g.classes - VEC;  // (the row's last vector ends with its last score)
      float t[VEC];
#pragma unroll
      for (int c = 0; c < VEC; ++c) t[c] = 0.f;
      if (!r.none) {
        to_float<T, VEC>(load_raw<T, VEC>(p + at), t);
#pragma unroll
        for (int c = 0; c < VEC; ++c) t[c] = r.of(t[c], at + c);
      }
      store_raw<T, VEC>(o + at, t);
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------
constexpr int64_t LP_THREADS = 1ll << 31;  // of a launch, which has to stay below 2^32 of them

// A wavefront per row where there are rows for all of the chip's wavefronts, or a workgroup would have less than a tile for each of its own.
bool lp_wave_rows(int64_t n, int classes) { return n >= 4096 || classes <= 2 * LP_TILE; }
// Workgroups per row: one, or, with too few rows for two per compute unit, as many as that takes and the row has chunks for.
int lp_splits(int64_t n, int classes) {
  if (n == 0 || classes <= LP_GROUP || lp_wave_rows(n, classes)) return 1;
  const int64_t want = isp_ceil_div(512, n), have = isp_ceil_div(classes, LP_CHUNK);
  return (int)(want < have ? want : have);
}
template <class T, int VEC, int LPR, int NV>
void lp_group(const lp_args& a, hipStream_t s) {
  const int64_t g = isp_ceil_div(a.n, ISP_WG / LPR);
  const unsigned grid = (unsigned)(g < 8192 ? g : 8192);
  if (a.top > 0) k_lp_group<T, VEC, LPR, NV, true><<<grid, ISP_WG, 0, s>>>(a);
  else k_lp_group<T, VEC, LPR, NV, false><<<grid, ISP_WG, 0, s>>>(a);
}
template <class T, int VEC, int LPR, int NV>
void lp_group(const lp_bwd_args& a, hipStream_t s) {
  const int64_t g = isp_ceil_div(a.n, ISP_WG / LPR);
  k_lp_group_bwd<T, VEC, LPR, NV><<<(unsigned)(g < 8192 ? g : 8192), ISP_WG, 0, s>>>(a);
}
template <class T, class A>
void lp_short_rows(const A& a, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(T), MAX = 16 / VEC;
  if (a.classes < VEC) return lp_group<T, 1, 8, 1>(a, s);
  switch (isp_row_lanes(a.classes, VEC)) {
    case 4: return lp_group<T, VEC, 4, 1>(a, s);
    case 8: return lp_group<T, VEC, 8, 1>(a, s);
    case 16: return lp_group<T, VEC, 16, 1>(a, s);
    case 32: return lp_group<T, VEC, 32, 1>(a, s);
  }
  if (a.classes <= ISP_WAVE * VEC) return lp_group<T, VEC, 64, 1>(a, s);
  if (MAX == 2 || a.classes <= ISP_WAVE * VEC * 2) return lp_group<T, VEC, 64, 2>(a, s);
  return lp_group<T, VEC, 64, MAX>(a, s);
}

template <class T>
void lp_run(const lp_args& a, hipStream_t s) {
  if (a.classes <= LP_GROUP) return lp_short_rows<T>(a, s);
  const int bt = LP_WAVES * ISP_WAVE;
  if (lp_wave_rows(a.n, a.classes)) {
    constexpr int64_t MOST = LP_THREADS / ISP_WAVE;
    for (int64_t r0 = 0; r0 < a.n; r0 += MOST) {
      lp_args b = a;
      b.z = static_cast<const T*>(a.z) + r0 * a.ldz;
      b.n = a.n - r0 < MOST ? a.n - r0 : MOST;
      if (a.labels) b.labels += r0;
      if (a.logprob) b.logprob += r0;
      if (a.entropy) b.entropy += r0;
      if (a.stats) b.stats += 2 * r0;
      if (a.top_logprob) b.top_logprob += r0 * a.top;
      if (a.top_index) b.top_index += r0 * a.top;
      const unsigned grid = (unsigned)isp_ceil_div(b.n, LP_WAVES);
      if (a.top > 0) k_lp_stream<T, 1, true><<<grid, bt, 0, s>>>(b);
      else k_lp_stream<T, 1, false><<<grid, bt, 0, s>>>(b);
    }
    return;
  }
  const unsigned grid = (unsigned)(a.n * a.splits);
  if (a.top > 0) k_lp_stream<T, LP_WAVES, true><<<grid, bt, 0, s>>>(a);
  else k_lp_stream<T, LP_WAVES, false><<<grid, bt, 0, s>>>(a);
  if (a.splits > 1) {
    if (a.top > 0) k_lp_join<T, true><<<(unsigned)a.n, ISP_WAVE, 0, s>>>(a);
    else k_lp_join<T, false><<<(unsigned)a.n, ISP_WAVE, 0, s>>>(a);
  }
}
template <class T>
void lp_run(const lp_bwd_args& a, hipStream_t s) {
  if (a.classes <= LP_GROUP) return lp_short_rows<T>(a, s);
  const int64_t total = a.n * a.chunks;
  k_lp_chunk_bwd<T><<<(unsigned)(total < LP_THREADS / ISP_WG ? total : LP_THREADS / ISP_WG), ISP_WG, 0, s>>>(a);
}

}  // namespace

size_t isp_label_logprob_parts_bytes(int64_t n, int32_t n_classes, int32_t top) {
  const int64_t parts = n * lp_splits(n, n_classes);
  if (parts == n) return 0;
  return isp_align((size_t)(3 * parts + 1) / 2 * 8 + (size_t)parts * (size_t)top * 8);
}

isp_status isp_label_logprob_launch(const void* Z, int64_t ldz, int64_t n, int32_t n_classes, int dtype, const int64_t* labels, float* logprob,
                                    float* entropy, float* stats, int32_t top, float* top_logprob, int32_t* top_index, void* ws, hipStream_t s) {
  if (n == 0) return ISP_OK;
  const lp_args a{Z, ldz, n, n_classes, labels, logprob, entropy, stats, top, top_logprob, top_index, lp_splits(n, n_classes), static_cast<float*>(ws)};
  if (dtype == ISP_F32) lp_run<float>(a, s);
  else if (dtype == ISP_BF16) lp_run<bf16_t>(a, s);
  else lp_run<f16_t>(a, s);
  ISP_LAUNCH_CHECK();
  return ISP_OK;
}

isp_status isp_label_logprob_bwd_launch(const void* Z, int64_t ldz, int64_t n, int32_t n_classes, int dtype, const int64_t* labels,
                                        const float* stats, const float* entropy, const float* d_logprob, const float* d_entropy, void* dZ,
                                        int64_t lddz, hipStream_t s) {
  if (n == 0) return ISP_OK;
  const lp_bwd_args a{Z, ldz, n, n_classes, labels, stats, entropy, d_logprob, d_entropy, dZ, lddz, (int)isp_ceil_div(n_classes, ISP_WG * 16)};
  if (dtype == ISP_F32) lp_run<float>(a, s);
  else if (dtype == ISP_BF16) lp_run<bf16_t>(a, s);
  else lp_run<f16_t>(a, s);
  ISP_LAUNCH_CHECK();
  return ISP_OK;
}
