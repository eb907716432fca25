// Attention over the stored entries of a CSR matrix (gfx950, wave64): the three passes' kernels, instantiated per element type in attention_*.hip.
//   forward   s_p = scale <q_i, k_j> + bias_p,  P = softmax over row i's entries,  y_i = sum_p P_p v_j           (p = (i, j))
//   backward  t_p = <dy_i, v_j>,  D_i = sum_p P_p t_p,  dS_p = P_p (t_p - D_i)
//             rows of A:    dq_i = scale sum_p dS_p k_j = scale (sum_p P_p t_p k_j - D_i sum_p P_p k_j),  P_p = exp(s_p - m_i) / l_i
//             rows of A^T:  dk_j = scale sum_p dS_p q_i,   dv_j = sum_p P_p dy_i
// with `heads` query heads on `kv_heads` key heads: query head h reads key head h / R, R = heads / kv_heads.
//
// The work items and runs of run_stream.h.  A lane has W consecutive columns of one key head (and of RQ of the R query heads that read
// it); lph lanes span a head, a group of LPG lanes LPG / lph heads, and G = 64 / LPG groups stream their runs of entries side by side.  Scores are sums over
// lph lanes; each gathered row of K and V serves the group's heads at once, and RQ query heads share it in registers.  Heads that don't fit
// the group are other workgroups' (blockIdx.y), query heads beyond RQ too (blockIdx.z).  No score is ever written: the backward computes them again.
//
// Softmax in one pass: a row's (m, l, y) are a reference for its scores, the sum of exp(s - m) and of exp(s - m) v.  m is the
// first score, and moves only to a score that is above it by more than ATT_SLACK: almost no step has to rescale, and the sums' weights
// are at most e^8 (values of up to fp32's range over 3000 times the row's entries fit).  The backward's are divided by l: at most 1.  Parts
// of a row that a run boundary cuts, or a split row's segments, are joined by their references, in a fixed order.
// In the backward the rows' pass forms D beside dq's two sums, so that y, which has been rounded, is not needed, and leaves it to the
// columns' pass.
// Entries whose bias is -inf count for nothing, whatever their operands hold; a row without others has y = 0, l = 0.
// Everything is held in 32 bits (dot products of 16-bit operands: att_operand); outputs are rounded once.
#pragma once
#include "attention_args.h"
#include "elem.h"
#include "run_stream.h"

namespace {
using namespace isp_dev;

constexpr float ATT_SLACK = 8.f;
// The reference of a row that has met nothing: finite, so that differences to it are numbers; a score of -inf is below it, too.
constexpr float ATT_NONE = -3.402823466e38f;

// What a lane leaves in of its vector of a row operand: its own elements, as factors (fp32), or as bits that products of 16-bit pairs take (att_dot).
template <class T, int W>
struct att_mask {
  typedef uint32_t bits __attribute__((ext_vector_type(W / 2)));
  bits keep;
  __device__ __forceinline__ void set(int j, bool own, float) {
    const uint32_t half = 0xffffu << (16 * (j & 1));
    keep[j / 2] = (j & 1 ? keep[j / 2] : 0u) | (own ? half : 0u);
  }
};
template <int W>
struct att_mask<float, W> {
  float own[W], scaled[W];  // 1 or the scale for those, else 0
  __device__ __forceinline__ void set(int j, bool o, float scale) {
    own[j] = o ? 1.f : 0.f;
    scaled[j] = o ? scale : 0.f;
  }
};
// Whether the values are added to the scores, as an entry's work asks or knows.  The loops with eight columns to a lane, which serve long rows, are there
// with and without: a step without branches is one block to the compiler (233 k rows, 40 M entries, 3 heads of 20, fp16 935 / 864 us).  With four
// the kernels would double for nothing (forward, 1 M rows, 17 M entries 660 / 669, rows 1111 / 1156).
constexpr int ATT_PLAIN = 0, ATT_BIAS = 1, ATT_ASK = 2;

// Where a lane works.
template <class T, int W, bool TINY>
struct att_lane {
  int lph;    // lanes per head
  int hk;     // key head (of a lane without one: the last)
  int c;      // first column of its vector within the head: the last vector of a head moves back to end with it
  int lo, hi; // elements [lo, hi) of the vector are its own (a moved-back vector's leading ones belong to the vector before)
  att_mask<T, W> mask;
  bool live, first;  // first: has the head's first column
  __device__ __forceinline__ att_lane(const att_args& a, int q, int hb) {
    lph = a.lph;
    const int h = (int)blockIdx.y * hb + q / lph, c0 = (q % lph) * W;
    live = h < a.kv_heads && c0 < a.dh;
    hk = h < a.kv_heads ? h : a.kv_heads - 1;
    c = TINY ? 0 : c0 + W <= a.dh ? c0 : a.dh - W;
    lo = live ? c0 - c : W;
    hi = TINY ? a.dh : W;
    first = live && c0 == 0;
#pragma unroll
    for (int j = 0; j < W; ++j) mask.set(j, j >= lo && j < hi, a.scale);
  }
  __device__ __forceinline__ int col(int head, int dh) const { return head * dh + c; }
};

// A lane's vector as it lies in memory.
template <class T, int W, bool TINY>
__device__ __forceinline__ raw_t<T, W> att_load(const T* p, int dh) {
  if constexpr (TINY) {  // (heads of fewer than W columns: what lies behind may not be ours)
    raw_t<T, W> v;
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = p[j < dh ? j : dh - 1];
    return v;
  } else {
    return load_raw<T, W>(p);
  }
}
template <class T, int W, bool TINY>
__device__ __forceinline__ void att_store(T* p, int dh, const float (&o)[W]) {
  if constexpr (TINY) {
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < dh) p[j] = (T)o[j];
  } else {
    store_raw<T, W>(p, o);
  }
}

// N sums over lph lanes (lph: a power of two, at most LPG; wave-uniform).
template <int LPG, int N>
__device__ __forceinline__ void att_sums(float (&v)[N], int lph) {
#define ISP_STAGE(n, expr)                           \
  if (LPG >= n && lph >= n) {                        \
    _Pragma("unroll") for (int k = 0; k < N; ++k) v[k] += expr; \
  }
  ISP_STAGE(2, dpp_of<DPP_XOR1>(v[k]))
  ISP_STAGE(4, dpp_of<DPP_XOR2>(v[k]))
  ISP_STAGE(8, dpp_of<DPP_HALF_MIRROR>(v[k]))
  ISP_STAGE(16, dpp_of<DPP_ROR8>(v[k]))
  ISP_STAGE(32, __shfl_xor(v[k], 16))
  ISP_STAGE(64, __shfl_xor(v[k], 32))
#undef ISP_STAGE
}

// A row operand's vector as a lane multiplies it with gathered ones: elements that are not its own count for nothing in a dot product.  (They are of
// the same head, or the head is nobody's: an infinity or NaN among the gathered ones is in the dot product anyway.)
// fp32: floats, with the scale in those of the scores.  16 bits: pairs as they lie, for the instruction that multiplies two pairs and adds both
// products to a sum in 32 bits: half the instructions of fp32 from
// fp16, less than half from bf16, which would have to be converted, and half the registers; the scale is then the score's.
// That instruction's result is off by at most 3 2^-24 of the three terms (2.9 in 10^6 random triples of like and of unlike magnitudes; .1 to .4 on
// average, as much as two fused multiply-adds), in which a subnormal operand counts as the type's smallest normal number: products are lined up by
// the operands' exponents as they are stored.  Next to a subnormal operand that is less than 2^-10 of what its own rounding to 16 bits is worth.  (fp16
// with fused multiply-adds instead: 40 M entries, 3 heads of 20 917 / 961 us, 6 M, 2 of 128 with the backward 1222 / 1513.)
template <class T, int W>
struct att_operand {
  raw_t<T, W> v;
  static constexpr bool SCALED = false;
  __device__ __forceinline__ void set(const raw_t<T, W>& r, const att_mask<T, W>& m, bool) {
    typedef typename att_mask<T, W>::bits bits;
    v = __builtin_bit_cast(raw_t<T, W>, __builtin_bit_cast(bits, r) & m.keep);
  }
};
template <int W>
struct att_operand<float, W> {
  float v[W];
  static constexpr bool SCALED = true;
  __device__ __forceinline__ void set(const raw_t<float, W>& r, const att_mask<float, W>& m, bool scaled) {
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = r[j] * (scaled ? m.scaled[j] : m.own[j]);
  }
};
template <int W>
__device__ __forceinline__ float att_dot(const att_operand<float, W>& a, const raw_t<float, W>& b) {
  float s = a.v[0] * b[0];
#pragma unroll
  for (int j = 1; j < W; ++j) s = fmaf(a.v[j], b[j], s);
  return s;
}
template <class T, int W>
__device__ __forceinline__ float att_dot(const att_operand<T, W>& a, const raw_t<T, W>& b) {
  typedef T pair __attribute__((ext_vector_type(2)));
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < W; j += 2) {
    const pair x = {a.v[j], a.v[j + 1]}, y = {b[j], b[j + 1]};
    if constexpr (__is_same(T, f16_t)) s = __builtin_amdgcn_fdot2(x, y, s, false);
    else s = __builtin_amdgcn_fdot2_f32_bf16(x, y, s, false);
  }
  return s;
}
// Makes scores of N query heads' sums of products, but for the factor that is returned (the scale, where neither the operands have it nor a bias was added).
// mask(out): the entry counts for nothing where `out`.
template <class Operand, int BIAS, int N, int M, class Mask>
__device__ __forceinline__ float att_scores(const att_args& a, float (&z)[M], float bias, Mask&& mask) {
  const bool biased = BIAS == ATT_ASK ? a.bias : BIAS == ATT_BIAS;
  if (biased) {
    const bool out = bias == NEG_INF;
#pragma unroll
    for (int r = 0; r < N; ++r) z[r] = Operand::SCALED ? z[r] + bias : fmaf(z[r], a.scale, bias);
    if (__any(out)) {
#pragma unroll
      for (int r = 0; r < N; ++r) z[r] = out ? NEG_INF : z[r];
      mask(out);
    }
  }
  return Operand::SCALED || biased ? 1.f : a.scale;
}
// ... and its distance to m
template <class Operand>
__device__ __forceinline__ float att_gap(float z, float f, float m) { return Operand::SCALED ? z - m : fmaf(z, f, -m); }

// 1 / l by the hardware's reciprocal (about 1 ulp); 0 where the row has nothing.
__device__ __forceinline__ float att_inverse(float l) { return l == 0.f ? 0.f : __builtin_amdgcn_rcpf(l); }

template <class T>
__device__ __forceinline__ const T* att_row(const void* base, uint32_t row, uint32_t pitch) {  // (pitch in bytes)
  return reinterpret_cast<const T*>(static_cast<const char*>(base) + (uint64_t)row * pitch);
}

// ---- forward -------------------------------------------------------------------------------------------------------
template <class T_, int W_, int RQ_, bool TINY_>
struct att_fwd {
  using T = T_;
  static constexpr int W = W_, RQ = RQ_, RING = 4, PARTS = RQ, MOST = 4;
  static constexpr bool WIDE = sizeof(T) == 2;
  static constexpr bool TINY = TINY_;
  using lane_t = att_lane<T, W, TINY>;
  using operand = att_operand<T, W>;
  struct gathered { raw_t<T, W> k, v; };
  struct source { const T *k, *v; };  // the lane's columns of row 0
  struct requested { raw_t<T, W> q[RQ]; };
  struct row_t { operand q[RQ]; };
  struct part { float y[W], m, l; };  // of a query head

  static __device__ __forceinline__ int head(const att_args& a, const lane_t& ln, int r) { return ln.hk * a.group + (int)blockIdx.z * RQ + r; }
  static __device__ __forceinline__ void clear(part& s) {
    s.m = ATT_NONE;
    s.l = 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) s.y[j] = 0.f;
  }
  static __device__ __forceinline__ source sources(const att_args& a, const lane_t& ln) {
    const int at = ln.col(ln.hk, a.dh);
    return {static_cast<const T*>(a.k) + at, static_cast<const T*>(a.v) + at};
  }
  static __device__ __forceinline__ void gather(const att_args& a, const source& o, int col, gathered& x) {
    x.k = att_load<T, W, TINY>(att_row<T>(o.k, col, a.pk), a.dh);
    x.v = att_load<T, W, TINY>(att_row<T>(o.v, col, a.pv), a.dh);
  }
  static __device__ __forceinline__ void request(const att_args& a, const lane_t& ln, int row, requested& o) {
    const T* p = att_row<T>(a.q, row, a.pq) + ln.col(head(a, ln, 0), a.dh);
#pragma unroll
    for (int r = 0; r < RQ; ++r) o.q[r] = att_load<T, W, TINY>(p + r * a.dh, a.dh);
  }
  static __device__ __forceinline__ void row(const att_args& a, const lane_t& ln, const requested& o, row_t& w) {
#pragma unroll
    for (int r = 0; r < RQ; ++r) w.q[r].set(o.q[r], ln.mask, true);
  }
  template <int LPG, int BIAS>
  static __device__ __forceinline__ void edge(const att_args& a, const lane_t& ln, float bias, const gathered& g, const row_t& w, part (&s)[PARTS]) {
    float v[W], z[RQ];
    to_float<T, W>(g.v, v);
#pragma unroll
    for (int r = 0; r < RQ; ++r) z[r] = att_dot(w.q[r], g.k);
    att_sums<LPG, RQ>(z, ln.lph);
    const float f = att_scores<operand, BIAS, RQ>(a, z, bias, [&](bool out) {  // (whatever its operands hold)
#pragma unroll
      for (int j = 0; j < W; ++j) v[j] = out ? 0.f : v[j];
    });
    float gap[RQ];
    bool move = false;
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      gap[r] = att_gap<operand>(z[r], f, s[r].m);
      move |= gap[r] > ATT_SLACK;
    }
    if (__any(move)) {
#pragma unroll
      for (int r = 0; r < RQ; ++r) {
        const bool up = gap[r] > ATT_SLACK;
        const float less = up ? fast_exp(-gap[r]) : 1.f, to = operand::SCALED ? z[r] : z[r] * f;
        s[r].m = up ? to : s[r].m;
        gap[r] = up ? to - to : gap[r];  // (0; +inf: NaN)
        s[r].l *= less;
#pragma unroll
        for (int j = 0; j < W; ++j) s[r].y[j] *= less;
      }
    }
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      const float p = fast_exp(gap[r]);
      s[r].l += p;
#pragma unroll
      for (int j = 0; j < W; ++j) s[r].y[j] = fmaf(p, v[j], s[r].y[j]);
    }
  }
  static __device__ __forceinline__ void join(part& s, const part& o) {
    const float m = fmaxf(s.m, o.m);
    const float f = s.m == m ? 1.f : fast_exp(s.m - m), g = o.m == m ? 1.f : fast_exp(o.m - m);  // (both none: 1, of nothing)
    s.m = m;
    s.l = s.l * f + o.l * g;
#pragma unroll
    for (int j = 0; j < W; ++j) s.y[j] = s.y[j] * f + o.y[j] * g;
  }
  static __device__ __forceinline__ void store(const att_args& a, const lane_t& ln, int row, const part (&s)[PARTS]) {
    if (!ln.live) return;
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      const int h = head(a, ln, r);
      const float f = att_inverse(s[r].l);
      float o[W];
#pragma unroll
      for (int j = 0; j < W; ++j) o[j] = s[r].y[j] * f;
      att_store<T, W, TINY>(static_cast<T*>(a.y) + (int64_t)row * a.ldy + ln.col(h, a.dh), a.dh, o);
      if (ln.first && a.stats) {
        float* st = a.stats + ((int64_t)row * a.heads + h) * 2;
        st[0] = s[r].m;
        st[1] = s[r].l;
      }
    }
  }
  static __device__ __forceinline__ void store(const att_args& a, const lane_t& ln, int row, const part (&s)[PARTS], const row_t&) { store(a, ln, row, s); }
  static __device__ __forceinline__ void store_empty(const att_args& a, const lane_t& ln, int row, const part (&s)[PARTS]) { store(a, ln, row, s); }
  // a segment's partial row: heads * dh sums, then (m, l) of each head
  static __device__ __forceinline__ void store_part(const att_args& a, const lane_t& ln, int seg, const part (&s)[PARTS]) {
    if (!ln.live) return;
    float* p = a.part + (int64_t)seg * a.heads * (a.dh + 2);
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      const int h = head(a, ln, r);
      att_store<float, W, TINY>(p + ln.col(h, a.dh), a.dh, s[r].y);
      if (ln.first) {
        p[a.heads * a.dh + 2 * h] = s[r].m;
        p[a.heads * a.dh + 2 * h + 1] = s[r].l;
      }
    }
  }
};

// ---- backward ------------------------------------------------------------------------------------------------------
// over A's rows: dq, and D
template <class T_, int W_, int RQ_, bool TINY_>
struct att_bwd_row {
  using T = T_;
  static constexpr int W = W_, RQ = RQ_, RING = 4, PARTS = RQ, MOST = 2;
  static constexpr bool WIDE = sizeof(T) == 2;
  static constexpr bool TINY = TINY_;
  using lane_t = att_lane<T, W, TINY>;
  using operand = att_operand<T, W>;
  struct gathered { raw_t<T, W> k, v; };
  struct source { const T *k, *v; };
  struct requested { raw_t<T, W> q[RQ], dy[RQ]; float2 ml[RQ]; };
  struct row_t { operand q[RQ], dy[RQ]; float m[RQ], inv[RQ]; };
  struct part { float pt[W], p[W], d; };  // of a query head: sums of P t k, P k and P t

  static __device__ __forceinline__ int head(const att_args& a, const lane_t& ln, int r) { return ln.hk * a.group + (int)blockIdx.z * RQ + r; }
  static __device__ __forceinline__ void clear(part& s) {
    s.d = 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) s.pt[j] = s.p[j] = 0.f;
  }
  static __device__ __forceinline__ source sources(const att_args& a, const lane_t& ln) {
    const int at = ln.col(ln.hk, a.dh);
    return {static_cast<const T*>(a.k) + at, static_cast<const T*>(a.v) + at};
  }
  static __device__ __forceinline__ void gather(const att_args& a, const source& o, int col, gathered& x) {
    x.k = att_load<T, W, TINY>(att_row<T>(o.k, col, a.pk), a.dh);
    x.v = att_load<T, W, TINY>(att_row<T>(o.v, col, a.pv), a.dh);
  }
  static __device__ __forceinline__ void request(const att_args& a, const lane_t& ln, int row, requested& o) {
    const int h = head(a, ln, 0), at = ln.col(h, a.dh);
    const T *p = att_row<T>(a.q, row, a.pq) + at, *d = att_row<T>(a.dy, row, a.pdy) + at;
    const float2* ml = reinterpret_cast<const float2*>(a.stats) + ((uint64_t)(uint32_t)row * (uint32_t)a.heads + (uint32_t)h);
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      o.q[r] = att_load<T, W, TINY>(p + r * a.dh, a.dh);
      o.dy[r] = att_load<T, W, TINY>(d + r * a.dh, a.dh);
      o.ml[r] = ml[r];
    }
  }
  static __device__ __forceinline__ void row(const att_args& a, const lane_t& ln, const requested& o, row_t& w) {
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      w.q[r].set(o.q[r], ln.mask, true);
      w.dy[r].set(o.dy[r], ln.mask, false);
      w.m[r] = o.ml[r].x;
      w.inv[r] = att_inverse(o.ml[r].y);
    }
  }
  template <int LPG, int BIAS>
  static __device__ __forceinline__ void edge(const att_args& a, const lane_t& ln, float bias, const gathered& g, const row_t& w, part (&s)[PARTS]) {
    float k[W], z[2 * RQ];
    to_float<T, W>(g.k, k);
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      z[r] = att_dot(w.q[r], g.k);
      z[RQ + r] = att_dot(w.dy[r], g.v);
    }
    att_sums<LPG, 2 * RQ>(z, ln.lph);
    const float f = att_scores<operand, BIAS, RQ>(a, z, bias, [&](bool out) {
#pragma unroll
      for (int r = 0; r < RQ; ++r) z[RQ + r] = out ? 0.f : z[RQ + r];
#pragma unroll
      for (int j = 0; j < W; ++j) k[j] = out ? 0.f : k[j];
    });
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      const float p = fast_exp(att_gap<operand>(z[r], f, w.m[r])) * w.inv[r], pt = p * z[RQ + r];  // (at most 1: what fits the operands' range fits the sums)
      s[r].d += pt;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        s[r].pt[j] = fmaf(pt, k[j], s[r].pt[j]);
        s[r].p[j] = fmaf(p, k[j], s[r].p[j]);
      }
    }
  }
  static __device__ __forceinline__ void join(part& s, const part& o) {
    s.d += o.d;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      s.pt[j] += o.pt[j];
      s.p[j] += o.p[j];
    }
  }
  static __device__ __forceinline__ void store_head(const att_args& a, const lane_t& ln, int row, int h, const part& s, float m, float inv) {
    float o[W];
#pragma unroll
    for (int j = 0; j < W; ++j) o[j] = (s.pt[j] - s.d * s.p[j]) * a.scale;
    if (a.y) att_store<T, W, TINY>(static_cast<T*>(a.y) + (int64_t)row * a.ldy + ln.col(h, a.dh), a.dh, o);
    if (ln.first) a.stat[(int64_t)row * a.heads + h] = {m, inv, s.d, 0.f};
  }
  static __device__ __forceinline__ void store(const att_args& a, const lane_t& ln, int row, const part (&s)[PARTS]) {
    if (!ln.live) return;
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      const float* st = a.stats + ((int64_t)row * a.heads + head(a, ln, r)) * 2;
      store_head(a, ln, row, head(a, ln, r), s[r], st[0], att_inverse(st[1]));
    }
  }
  // (the row at work: its numbers are here, and loading them would wait for every gather in flight)
  static __device__ __forceinline__ void store(const att_args& a, const lane_t& ln, int row, const part (&s)[PARTS], const row_t& w) {
    if (!ln.live) return;
#pragma unroll
    for (int r = 0; r < RQ; ++r) store_head(a, ln, row, head(a, ln, r), s[r], w.m[r], w.inv[r]);
  }
  static __device__ __forceinline__ void store_empty(const att_args& a, const lane_t& ln, int row, const part (&)[PARTS]) {
    if (!ln.live || !a.y) return;  // (nobody asks for the numbers of a row without entries)
    const float o[W] = {};
#pragma unroll
    for (int r = 0; r < RQ; ++r) att_store<T, W, TINY>(static_cast<T*>(a.y) + (int64_t)row * a.ldy + ln.col(head(a, ln, r), a.dh), a.dh, o);
  }
  // a segment's partial row: heads * dh sums of P t k, as many of P k, heads of P t
  static __device__ __forceinline__ void store_part(const att_args& a, const lane_t& ln, int seg, const part (&s)[PARTS]) {
    if (!ln.live) return;
    const int width = a.heads * a.dh;
    float* p = a.part + (int64_t)seg * a.heads * (2 * a.dh + 1);
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      const int h = head(a, ln, r);
      att_store<float, W, TINY>(p + ln.col(h, a.dh), a.dh, s[r].pt);
      att_store<float, W, TINY>(p + width + ln.col(h, a.dh), a.dh, s[r].p);
      if (ln.first) p[2 * width + h] = s[r].d;
    }
  }
};

// An element of dk / dv: what the passes over other query heads have left (fp32), and the sum of all with the last one's.
template <class T>
__device__ __forceinline__ void att_out(const att_args& a, float* carry, T* out, int64_t at_carry, int64_t at, float v) {
  if (a.pass > 0) v += carry[at_carry];
  if (a.pass < a.passes - 1) carry[at_carry] = v;
  else out[at] = (T)v;
}

// over A^T's rows: dk and dv.  Query heads [pass * RQ, (pass + 1) * RQ) of each key head's; blockIdx.z is not used.
template <class T_, int W_, int RQ_, bool TINY_>
struct att_bwd_col {
  using T = T_;
  static constexpr int W = W_, RQ = RQ_, RING = RQ == 1 && W == 4 ? 4 : 2, PARTS = 1, MOST = 4;
  static constexpr bool WIDE = sizeof(T) == 2;
  static constexpr bool TINY = TINY_;
  using lane_t = att_lane<T, W, TINY>;
  using operand = att_operand<T, W>;
  struct gathered { raw_t<T, W> q[RQ], dy[RQ]; att_num st[RQ]; };
  struct source { const T *q, *dy; const att_num* st; };
  struct requested { raw_t<T, W> k, v; };
  struct row_t { operand k, v; };
  struct part { float dk[W], dv[W]; };

  static __device__ __forceinline__ void clear(part& s) {
#pragma unroll
    for (int j = 0; j < W; ++j) s.dk[j] = s.dv[j] = 0.f;
  }
  static __device__ __forceinline__ source sources(const att_args& a, const lane_t& ln) {
    const int h0 = ln.hk * a.group + a.pass * RQ, at = ln.col(h0, a.dh);
    return {static_cast<const T*>(a.q) + at, static_cast<const T*>(a.dy) + at, a.stat + h0};
  }
  static __device__ __forceinline__ void gather(const att_args& a, const source& o, int col, gathered& x) {
    const T *p = att_row<T>(o.q, col, a.pq), *d = att_row<T>(o.dy, col, a.pdy);
    const att_num* st = att_row<att_num>(o.st, col, (uint32_t)a.heads * (uint32_t)sizeof(att_num));
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      x.q[r] = att_load<T, W, TINY>(p + r * a.dh, a.dh);
      x.dy[r] = att_load<T, W, TINY>(d + r * a.dh, a.dh);
      x.st[r] = st[r];
    }
  }
  static __device__ __forceinline__ void request(const att_args& a, const lane_t& ln, int row, requested& o) {
    const int at = ln.col(ln.hk, a.dh);
    o.k = att_load<T, W, TINY>(att_row<T>(a.k, row, a.pk) + at, a.dh);
    o.v = att_load<T, W, TINY>(att_row<T>(a.v, row, a.pv) + at, a.dh);
  }
  static __device__ __forceinline__ void row(const att_args& a, const lane_t& ln, const requested& o, row_t& w) {
    w.k.set(o.k, ln.mask, true);
    w.v.set(o.v, ln.mask, false);
  }
  template <int LPG, int BIAS>
  static __device__ __forceinline__ void edge(const att_args& a, const lane_t& ln, float bias, const gathered& g, const row_t& w, part (&s)[PARTS]) {
    float q[RQ][W], dy[RQ][W], z[2 * RQ], inv[RQ], d[RQ];
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      inv[r] = g.st[r].inv;
      d[r] = g.st[r].d;
      to_float<T, W>(g.q[r], q[r]);
      to_float<T, W>(g.dy[r], dy[r]);
      z[r] = att_dot(w.k, g.q[r]);
      z[RQ + r] = att_dot(w.v, g.dy[r]);
    }
    att_sums<LPG, 2 * RQ>(z, ln.lph);
    const float f = att_scores<operand, BIAS, RQ>(a, z, bias, [&](bool out) {
#pragma unroll
      for (int r = 0; r < RQ; ++r) {
        z[RQ + r] = out ? 0.f : z[RQ + r];
        inv[r] = out ? 0.f : inv[r];  // (the row's numbers are not finite where one of its other entries is not)
        d[r] = out ? 0.f : d[r];
#pragma unroll
        for (int j = 0; j < W; ++j) {
          q[r][j] = out ? 0.f : q[r][j];
          dy[r][j] = out ? 0.f : dy[r][j];
        }
      }
    });
#pragma unroll
    for (int r = 0; r < RQ; ++r) {
      const float p = fast_exp(att_gap<operand>(z[r], f, g.st[r].m)) * inv[r], ds = p * (z[RQ + r] - d[r]);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        s[0].dk[j] = fmaf(ds, q[r][j], s[0].dk[j]);
        s[0].dv[j] = fmaf(p, dy[r][j], s[0].dv[j]);
      }
    }
  }
  static __device__ __forceinline__ void join(part& s, const part& o) {
#pragma unroll
    for (int j = 0; j < W; ++j) {
      s.dk[j] += o.dk[j];
      s.dv[j] += o.dv[j];
    }
  }
  static __device__ __forceinline__ void store(const att_args& a, const lane_t& ln, int row, const part (&s)[PARTS]) {
    if (!ln.live) return;
    const int at = ln.col(ln.hk, a.dh), width = a.kv_heads * a.dh;
    float o[2][W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      o[0][j] = s[0].dk[j] * a.scale;
      o[1][j] = s[0].dv[j];
    }
    if (a.passes == 1) {
      att_store<T, W, TINY>(static_cast<T*>(a.y) + (int64_t)row * a.ldy + at, a.dh, o[0]);
      att_store<T, W, TINY>(static_cast<T*>(a.y2) + (int64_t)row * a.ldy2 + at, a.dh, o[1]);
    } else {  // (own elements only: a moved-back vector's are the other lane's to add)
#pragma unroll
      for (int j = 0; j < W; ++j)
        if (j >= ln.lo && j < ln.hi) {
          att_out(a, a.carry, static_cast<T*>(a.y), (int64_t)row * width + at + j, (int64_t)row * a.ldy + at + j, o[0][j]);
          att_out(a, a.carry2, static_cast<T*>(a.y2), (int64_t)row * width + at + j, (int64_t)row * a.ldy2 + at + j, o[1][j]);
        }
    }
  }
  static __device__ __forceinline__ void store(const att_args& a, const lane_t& ln, int row, const part (&s)[PARTS], const row_t&) { store(a, ln, row, s); }
  static __device__ __forceinline__ void store_empty(const att_args& a, const lane_t& ln, int row, const part (&s)[PARTS]) { store(a, ln, row, s); }
  // a segment's partial row: dk, then dv
  static __device__ __forceinline__ void store_part(const att_args& a, const lane_t& ln, int seg, const part (&s)[PARTS]) {
    if (!ln.live) return;
    const int width = a.kv_heads * a.dh;
    float* p = a.part + (int64_t)seg * 2 * width + ln.col(ln.hk, a.dh);
    float o[W];
#pragma unroll
    for (int j = 0; j < W; ++j) o[j] = s[0].dk[j] * a.scale;
    att_store<float, W, TINY>(p, a.dh, o);
    att_store<float, W, TINY>(p + width, a.dh, s[0].dv);
  }
};

// ---- a pass ----------------------------------------------------------------------------------------------------------
template <class P, int LPG>
__global__ void __launch_bounds__(ISP_WG) k_att(isp_view A, const int64_t* __restrict__ indptr, const int32_t* __restrict__ indices,
                                                const float* __restrict__ bias, att_args a) {
  __shared__ rn_lds lds;
  constexpr int G = ISP_WAVE / LPG, RING = P::RING, CHUNK = RING % 4 == 0 ? 2 : 1;
  using part = typename P::part;
  constexpr int PARTS = P::PARTS, N = sizeof(part) / sizeof(float);
  static_assert(ISP_WAVE * sizeof(part) <= sizeof(lds.w[0].ent), "the runs' sums fit the entries' place, a part at a time");
  const int lane = threadIdx.x & (ISP_WAVE - 1), w = threadIdx.x >> 6;
  const int item = __builtin_amdgcn_readfirstlane((int)blockIdx.x * ISP_WAVES_PER_WG + w);
  if (item >= A.n_blocks + A.n_seg) return;
  const item_range it = locate_item(A, indptr, item);
  if (it.skip) return;
  auto& L = lds.w[w];
  const rn_run R = rn_prepare<G>(it, indptr, indices, bias, nullptr, L, lane);
  const int g = lane / LPG;
  const typename P::lane_t ln(a, lane % LPG, LPG / a.lph);

  part st[PARTS], head[PARTS];  // head: the end of a row that began in an earlier run
#pragma unroll
  for (int k = 0; k < PARTS; ++k) {
    P::clear(st[k]);
    P::clear(head[k]);
  }
  for (int i = g; i < R.n_empty; i += G) P::store_empty(a, ln, L.dst[RN_EMPTY0 - i], st);

  if (R.steps == 0) return;  // (no entries: the operands may not be there)

  bool carried = R.mid, ended = false;
  const typename P::source src = P::sources(a, ln);
  auto run = [&](auto seg_tag, auto bias_tag) {
    constexpr bool SEG = decltype(seg_tag)::value;
    typename P::gathered x[RING];
    typename P::requested next;  // the row after the one at work, requested when that one began
    typename P::row_t cur;
    P::request(a, ln, SEG ? it.src_row : L.dst[R.k], next);
    P::row(a, ln, next, cur);
    if constexpr (!SEG) P::request(a, ln, L.dst[R.k + 1], next);
    rn_stream<RING, !SEG, false, CHUNK>(
        L, R, [&](int u, int c, int, int, bool) { P::gather(a, src, c, x[u]); },
        [&](auto u, float b, int) { P::template edge<LPG, decltype(bias_tag)::value>(a, ln, b, x[u], cur, st); },
        [&](int k, int row) {
          if (!carried) P::store(a, ln, row, st, cur);
          if (__any(carried)) {  // (once per run)
#pragma unroll
            for (int i = 0; i < PARTS; ++i)
              if (carried) head[i] = st[i];
          }
#pragma unroll
          for (int i = 0; i < PARTS; ++i) P::clear(st[i]);
          carried = false;
          ended = true;
          P::row(a, ln, next, cur);
          P::request(a, ln, L.dst[k + 2], next);
        });
  };
  auto both = [&](auto bias_tag) {
    if (it.is_seg) run(std::true_type{}, bias_tag);
    else run(std::false_type{}, bias_tag);
  };
  if constexpr (P::W == 4) both(std::integral_constant<int, ATT_ASK>{});
  else if (a.bias) both(std::integral_constant<int, ATT_BIAS>{});
  else both(std::integral_constant<int, ATT_PLAIN>{});

  if (it.is_seg) {  // one row: the groups' parts
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      const float* v = reinterpret_cast<const float*>(&st[k]);
#pragma unroll
      for (int o = LPG; o < ISP_WAVE; o <<= 1) {
        part other;
        float* t = reinterpret_cast<float*>(&other);
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = __shfl_xor(v[i], o);
        P::join(st[k], other);
      }
    }
    if (g == 0) P::store_part(a, ln, it.row, st);
    return;
  }
  if constexpr (G > 1) {  // rows cut by a run boundary: the run in which such a row ends joins the earlier runs' parts
    const unsigned long long m_end = __ballot(ended), m_mid = __ballot(R.mid);
    const unsigned long long m_head = m_end & m_mid;
    if (m_head == 0) return;
    float* __restrict__ tail = reinterpret_cast<float*>(L.ent);
    const bool mine = (m_head >> lane) & 1ull;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      wave_lds_sync();  // (every entry, or the part before, has been read)
      const float* v = reinterpret_cast<const float*>(&st[k]);
#pragma unroll
      for (int i = 0; i < N; ++i) tail[lane * N + i] = v[i];
      wave_lds_sync();
      if (mine) {
        int j = lane - LPG;
        for (;;) {
          part other;
          float* t = reinterpret_cast<float*>(&other);
#pragma unroll
          for (int i = 0; i < N; ++i) t[i] = tail[j * N + i];
          P::join(head[k], other);
          if (((m_end >> j) & 1ull) || !((m_mid >> j) & 1ull)) break;  // the row began in that run
          j -= LPG;
        }
      }
    }
    if (mine) P::store(a, ln, L.dst[R.k], head);
  }
}

// Split rows: their segments' partial rows put together.  A workgroup per row and 64 columns, a wavefront per quarter of the segments,
// in order; then the quarters, in order.
template <class T>
__global__ void __launch_bounds__(ISP_WG) k_att_fwd_fixup(isp_view A, att_args a) {
  __shared__ float part[ISP_WAVES_PER_WG][3][ISP_WAVE];
  const int lane = threadIdx.x & (ISP_WAVE - 1), w = threadIdx.x >> 6;
  const int s0 = A.hub_seg_ptr[blockIdx.x], s1 = A.hub_seg_ptr[blockIdx.x + 1], row = A.hub_rows[blockIdx.x];
  const int width = a.heads * a.dh, col = (int)blockIdx.y * ISP_WAVE + lane;
  const int h = col < width ? col / a.dh : 0;
  const int64_t pitch = (int64_t)a.heads * (a.dh + 2);
  const int q = (s1 - s0 + ISP_WAVES_PER_WG - 1) / ISP_WAVES_PER_WG;
  const int lo = s0 + w * q < s1 ? s0 + w * q : s1, hi = lo + q < s1 ? lo + q : s1;
  float m = ATT_NONE, l = 0.f, y = 0.f;
  if (col < width) {
#pragma unroll 4
    for (int s = lo; s < hi; ++s) m = fmaxf(m, a.part[s * pitch + width + 2 * h]);
#pragma unroll 4
    for (int s = lo; s < hi; ++s) {
      const float ms = a.part[s * pitch + width + 2 * h], ls = a.part[s * pitch + width + 2 * h + 1], ys = a.part[s * pitch + col];
      const float f = ms == m ? 1.f : fast_exp(ms - m);
      l = fmaf(ls, f, l);
      y = fmaf(ys, f, y);
    }
  }
  part[w][0][lane] = m;
  part[w][1][lane] = l;
  part[w][2][lane] = y;
  __syncthreads();
  if (w > 0 || col >= width) return;
#pragma unroll
  for (int i = 1; i < ISP_WAVES_PER_WG; ++i) m = fmaxf(m, part[i][0][lane]);
  l = y = 0.f;
#pragma unroll
  for (int i = 0; i < ISP_WAVES_PER_WG; ++i) {
    const float mi = part[i][0][lane], f = mi == m ? 1.f : fast_exp(mi - m);
    l = fmaf(part[i][1][lane], f, l);
    y = fmaf(part[i][2][lane], f, y);
  }
  static_cast<T*>(a.y)[(int64_t)row * a.ldy + col] = (T)(y * att_inverse(l));
  if (a.stats && col == h * a.dh) {
    float* st = a.stats + ((int64_t)row * a.heads + h) * 2;
    st[0] = m;
    st[1] = l;
  }
}

// The sum of column `col` of a split row's partial rows, `pitch` floats each, over the wavefront's quarter of its segments.
__device__ __forceinline__ float att_quarter(const att_args& a, int lo, int hi, int64_t pitch, int col) {
  float y = 0.f;
#pragma unroll 8
  for (int s = lo; s < hi; ++s) y += a.part[s * pitch + col];
  return y;
}
template <class T>
__global__ void __launch_bounds__(ISP_WG) k_att_row_fixup(isp_view A, att_args a) {
  __shared__ float part[ISP_WAVES_PER_WG][3][ISP_WAVE];
  const int lane = threadIdx.x & (ISP_WAVE - 1), w = threadIdx.x >> 6;
  const int s0 = A.hub_seg_ptr[blockIdx.x], s1 = A.hub_seg_ptr[blockIdx.x + 1], row = A.hub_rows[blockIdx.x];
  const int width = a.heads * a.dh, col = (int)blockIdx.y * ISP_WAVE + lane;
  const int h = col < width ? col / a.dh : 0;
  const int64_t pitch = (int64_t)a.heads * (2 * a.dh + 1);
  const int q = (s1 - s0 + ISP_WAVES_PER_WG - 1) / ISP_WAVES_PER_WG;
  const int lo = s0 + w * q < s1 ? s0 + w * q : s1, hi = lo + q < s1 ? lo + q : s1;
  if (col < width) {
    part[w][0][lane] = att_quarter(a, lo, hi, pitch, col);
    part[w][1][lane] = att_quarter(a, lo, hi, pitch, width + col);
    part[w][2][lane] = att_quarter(a, lo, hi, pitch, 2 * width + h);
  }
  __syncthreads();
  if (w > 0 || col >= width) return;
  float t[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    t[k] = part[0][k][lane];
#pragma unroll
    for (int i = 1; i < ISP_WAVES_PER_WG; ++i) t[k] += part[i][k][lane];
  }
  const int64_t at = (int64_t)row * a.heads + h;
  if (a.y) static_cast<T*>(a.y)[(int64_t)row * a.ldy + col] = (T)((t[0] - t[2] * t[1]) * a.scale);
  if (col == h * a.dh) a.stat[at] = {a.stats[2 * at], att_inverse(a.stats[2 * at + 1]), t[2], 0.f};
}
template <class T>
__global__ void __launch_bounds__(ISP_WG) k_att_col_fixup(isp_view A, att_args a) {
  __shared__ float part[ISP_WAVES_PER_WG][ISP_WAVE];
  const int lane = threadIdx.x & (ISP_WAVE - 1), w = threadIdx.x >> 6;
  const int s0 = A.hub_seg_ptr[blockIdx.x], s1 = A.hub_seg_ptr[blockIdx.x + 1], row = A.hub_rows[blockIdx.x];
  const int half = a.kv_heads * a.dh, width = 2 * half, col = (int)blockIdx.y * ISP_WAVE + lane;
  const int q = (s1 - s0 + ISP_WAVES_PER_WG - 1) / ISP_WAVES_PER_WG;
  const int lo = s0 + w * q < s1 ? s0 + w * q : s1, hi = lo + q < s1 ? lo + q : s1;
  float y = col < width ? att_quarter(a, lo, hi, width, col) : 0.f;
  part[w][lane] = y;
  __syncthreads();
  if (w > 0 || col >= width) return;
#pragma unroll
  for (int i = 1; i < ISP_WAVES_PER_WG; ++i) y += part[i][lane];
  if (col < half) att_out(a, a.carry, static_cast<T*>(a.y), (int64_t)row * half + col, (int64_t)row * a.ldy + col, y);
  else att_out(a, a.carry2, static_cast<T*>(a.y2), (int64_t)row * half + col - half, (int64_t)row * a.ldy2 + col - half, y);
}

// K's and V's rows next to each other in rows of whole lines: 16 bytes a thread.
template <class T>
__global__ void __launch_bounds__(ISP_WG) k_att_pack(att_args a, uint32_t pitch) {
  constexpr int W = 16 / sizeof(T);
  const uint32_t per_row = pitch / 16;
  const int width = a.kv_heads * a.dh;
  const int64_t total = a.n_cols * per_row;
  for (int64_t i = (int64_t)blockIdx.x * ISP_WG + threadIdx.x; i < total; i += (int64_t)gridDim.x * ISP_WG) {
    const int64_t row = i / per_row;
    const int e = (int)(i - row * per_row) * W;
    const T *k = att_row<T>(a.k, (uint32_t)row, a.pk), *v = att_row<T>(a.v, (uint32_t)row, a.pv);
    raw_t<T, W> o;
    if (e + W <= width) o = load_raw<T, W>(k + e);
    else if (e >= width && e + W <= 2 * width) o = load_raw<T, W>(v + (e - width));
    else
#pragma unroll
      for (int j = 0; j < W; ++j) o[j] = e + j < width ? k[e + j] : e + j < 2 * width ? v[e + j - width] : (T)0.f;
    *reinterpret_cast<raw_t<T, W>*>(static_cast<char*>(a.packed) + row * pitch + (int64_t)e * sizeof(T)) = o;
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------
// chunks: of a key head's query heads, side by side (blockIdx.z)
template <class P, int LPG>
isp_status att_launch(const isp_view& v, const att_args& a, int chunks, hipStream_t s) {
  const int items = v.n_blocks + v.n_seg, hb = LPG / a.lph;
  if (items == 0) return ISP_OK;
  const dim3 grid((unsigned)((items + ISP_WAVES_PER_WG - 1) / ISP_WAVES_PER_WG), (unsigned)((a.kv_heads + hb - 1) / hb), (unsigned)chunks);
  k_att<P, LPG><<<grid, ISP_WG, 0, s>>>(v, v.indptr, v.indices, a.bias ? v.values : nullptr, a);
  ISP_LAUNCH_CHECK();
  return ISP_OK;
}
// Lanes to a group: as many of the heads as 64 lanes hold.
template <template <class, int, int, bool> class P, class T, int W, int RQ>
isp_status att_lanes(const isp_view& v, const att_args& a, int chunks, hipStream_t s) {
  if constexpr (W == 4)
    if (a.dh < W) return att_launch<P<T, W, RQ, true>, 4>(v, a, chunks, s);
  int lanes = 4;
  while (lanes < ISP_WAVE && lanes < a.lph * a.kv_heads) lanes *= 2;
  switch (lanes) {
    case 4: return att_launch<P<T, W, RQ, false>, 4>(v, a, chunks, s);
    case 8: return att_launch<P<T, W, RQ, false>, 8>(v, a, chunks, s);
    case 16: return att_launch<P<T, W, RQ, false>, 16>(v, a, chunks, s);
    case 32: return att_launch<P<T, W, RQ, false>, 32>(v, a, chunks, s);
    default: return att_launch<P<T, W, RQ, false>, 64>(v, a, chunks, s);
  }
}
template <template <class, int, int, bool> class P, class T>
isp_status att_pass(const isp_view& v, att_args a, int rq, int chunks, bool wide, hipStream_t s) {
  a.lph = att_lanes_per_head(a.dh, wide ? 8 : 4);
  if constexpr (P<T, 4, 1, false>::WIDE)
    if (wide) return att_lanes<P, T, 8, 1>(v, a, chunks, s);
  if constexpr (P<T, 4, 1, false>::MOST == 4)
    if (rq == 4) return att_lanes<P, T, 4, 4>(v, a, chunks, s);
  if (rq == 2) return att_lanes<P, T, 4, 2>(v, a, chunks, s);
  return att_lanes<P, T, 4, 1>(v, a, chunks, s);
}

template <class T>
bool att_takes_wide(const isp_csr* A, const att_args& a) {
  return att_wide(sizeof(T), a.group, a.kv_heads, a.dh, A->info.nnz, A->info.n_rows - A->info.bin_rows[0]);
}

template <class T>
isp_status att_forward(const isp_csr* A, att_args a, hipStream_t s) {
  const isp_view& v = A->v;
  const int rq = att_share(a.group, 4);
  if (a.packed) {
    const int64_t row_bytes = (int64_t)a.kv_heads * a.dh * sizeof(T);
    const uint32_t pitch = (uint32_t)att_packed_pitch(row_bytes);
    const int64_t groups = (a.n_cols * (pitch / 16) + ISP_WG - 1) / ISP_WG;
    k_att_pack<T><<<(unsigned)(groups < 65536 ? groups : 65536), ISP_WG, 0, s>>>(a, pitch);
    ISP_LAUNCH_CHECK();
    a.k = a.packed;
    a.v = static_cast<const char*>(a.packed) + row_bytes;
    a.pk = a.pv = pitch;
  }
  isp_status st = att_pass<att_fwd, T>(v, a, rq, a.group / rq, att_takes_wide<T>(A, a), s);
  if (st != ISP_OK || v.n_hub == 0) return st;
  k_att_fwd_fixup<T><<<dim3((unsigned)v.n_hub, (unsigned)((a.heads * a.dh + ISP_WAVE - 1) / ISP_WAVE)), ISP_WG, 0, s>>>(v, a);
  ISP_LAUNCH_CHECK();
  return ISP_OK;
}

template <class T>
isp_status att_backward(const isp_csr* A, att_args a, const att_grads& o, hipStream_t s) {
  const isp_view &v = A->v, &vt = A->At ? A->At->v : A->v;
  const int rq_row = att_share(a.group, 2), rq = att_share(a.group, 4), passes = a.group / rq;
  a.y = o.dq;
  a.ldy = o.lddq;
  isp_status st = att_pass<att_bwd_row, T>(v, a, rq_row, a.group / rq_row, att_takes_wide<T>(A, a), s);
  if (st != ISP_OK) return st;
  if (v.n_hub > 0) {
    k_att_row_fixup<T><<<dim3((unsigned)v.n_hub, (unsigned)((a.heads * a.dh + ISP_WAVE - 1) / ISP_WAVE)), ISP_WG, 0, s>>>(v, a);
    ISP_LAUNCH_CHECK();
  }
  if (!o.dk) return ISP_OK;
  a.y = o.dk;
  a.ldy = o.lddk;
  a.y2 = o.dv;
  a.ldy2 = o.lddv;
  a.passes = passes;
  const bool wide = att_takes_wide<T>(A->At, a);
  for (a.pass = 0; a.pass < passes; ++a.pass) {
    if ((st = att_pass<att_bwd_col, T>(vt, a, rq, 1, wide, s)) != ISP_OK) return st;
    if (vt.n_hub > 0) {
      k_att_col_fixup<T><<<dim3((unsigned)vt.n_hub, (unsigned)((2 * a.kv_heads * a.dh + ISP_WAVE - 1) / ISP_WAVE)), ISP_WG, 0, s>>>(vt, a);
      ISP_LAUNCH_CHECK();
    }
  }
  return ISP_OK;
}

}  // namespace
