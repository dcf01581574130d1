// What the scores of stored logits and of the head share: element types, the
// running statistics of a softmax and how two of them join.
#pragma once

#include <type_traits>

#include "../../include/toktier_model.h"
#include "tt_internal.h"

namespace tt {

using bf16_t = __bf16;
using f16_t = _Float16;

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float NEG_INF = -__builtin_inff();

// The larger (smaller) of two, NaN if either is: a row's maximum carries its NaNs.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return __builtin_elementwise_minimum(a, b); }

// Statistics of a part of a row, in powers of two: m the largest logit, and over
// all entries but one of those that m is of, s the sum of e_j = 2^d_j and u the
// sum of e_j d_j.  That one entry is left out so that what the others come to
// keeps its bits where the row is nearly sure of it (next to a 1, a sum of 1e-5
// would keep 7 of its 24 bits).
// d_j = x_j c - R with c = scale / log 2 and R the rounded product m c.  How far
// R is off m c is made up for wherever sums of different m meet (rounded_off), so
// that one fused multiply-add an entry gives d_j.  Where m c is too large for that
// (masks of the type's lowest value overflow), d_j = (x_j - m) c.
struct Stats {
  float m, s, u;
};
constexpr float PLAIN_MOST = 1048576.f;
constexpr float LEAST_EXPONENT = -126.f;  // 2^d is 0 or next to it below

__device__ __forceinline__ Stats empty_stats() { return {NEG_INF, 0.f, 0.f}; }

// d_j = (x_j - base) c + off; base is 0 for all but huge m
struct Reference {
  float base, off;
};
__device__ __forceinline__ bool is_plain(float m, float c) { return m == NEG_INF || fabsf(m * c) < PLAIN_MOST; }
__device__ __forceinline__ Reference reference(float m, float c) {
  if (m == NEG_INF) return {0.f, 0.f};
  return is_plain(m, c) ? Reference{0.f, -(m * c)} : Reference{m, 0.f};
}
// R - m c
__device__ __forceinline__ float rounded_off(float m, float c) {
  return m != NEG_INF && is_plain(m, c) ? -fmaf(m, c, -(m * c)) : 0.f;
}
// PLAIN: base is known to be 0.  (-inf adds 0: d is held for the product alone)
template <bool PLAIN>
__device__ __forceinline__ void add_entry(Stats& st, float x, const Reference& r, float c) {
  const float d = fmaf(PLAIN ? x : x - r.base, c, r.off), e = __builtin_amdgcn_exp2f(d);
  st.s += e;
  st.u = fmaf(e, fmaxf(d, LEAST_EXPONENT), st.u);
}
// Two entries and the largest before them: the largest of the three goes on in
// `top`, the other two are added.
template <bool PLAIN>
__device__ __forceinline__ void add_two(Stats& st, float& top, float x, float y, const Reference& r, float c) {
  const float low = smaller(smaller(top, x), y), mid = __builtin_amdgcn_fmed3f(top, x, y);
  top = larger(larger(top, x), y);
  add_entry<PLAIN>(st, low, r, c);
  add_entry<PLAIN>(st, mid, r, c);
}

// e d for e = 2^d: 0 where e is 0, also for d = -inf; NaN stays.
__device__ __forceinline__ float weigh(float e, float d) { return e * fmaxf(d, -1e30f); }

// a's sums moved to the larger maximum m.  The entry that a left out is not
// among them: it is the caller's to add, or to go on leaving out.
__device__ __forceinline__ void lower(Stats& a, float m, float c) {
  if (a.m == m) return;
  if (a.m == NEG_INF) {
    a = {m, 0.f, 0.f};
    return;
  }
  const float d = (a.m - m) * c + (rounded_off(a.m, c) - rounded_off(m, c)), f = __builtin_amdgcn_exp2f(d);
  a.u = fmaf(f, a.u, weigh(f, d) * a.s);
  a.s *= f;
  a.m = m;
}

__device__ __forceinline__ Stats join(Stats a, Stats b, float c) {
  const float m = larger(a.m, b.m), less = smaller(a.m, b.m);
  lower(a, m, c);
  lower(b, m, c);
  Stats all = {m, a.s + b.s, a.u + b.u};
  add_entry<false>(all, less, reference(m, c), c);
  return all;
}

// The wave's statistics in every lane: one move to the wave's maximum, then sums.
// Each lane left out `held`, and some lane's is the wave's maximum.
__device__ __forceinline__ Stats wave_join(Stats a, float held, float c) {
  float m = a.m;
#pragma unroll
  for (int d = 32; d; d >>= 1) m = larger(m, __shfl_xor(m, d));
  lower(a, m, c);
  // every lane but the first of those that hold the maximum adds what it left out
  const uint64_t top = __ballot(held == m);
  if ((top & (~top + 1)) != 1ull << (threadIdx.x & 63)) add_entry<false>(a, held, reference(m, c), c);
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    a.s += __shfl_xor(a.s, d);
    a.u += __shfl_xor(a.u, d);
  }
  return a;
}

// A row's results from the statistics of the whole row.
struct RowScores {
  float m, log_s, entropy;
};
__device__ __forceinline__ RowScores row_scores(const Stats& a, float c) {
  if (a.m == NEG_INF) return {NEG_INF, NEG_INF, 0.f};  // nothing but -inf
  if (a.m != a.m || a.m == __builtin_inff()) {
    const float nan = __builtin_nanf("");
    return {nan, nan, nan};
  }
  // the sums as of m c itself; the entry left out is a 1 whose exponent is 0
  const float off = rounded_off(a.m, c), f = __builtin_amdgcn_exp2f(off), s = a.s * f, u = f * fmaf(off, a.s, a.u);
  const float log_s = log1pf(s);
  return {a.m, log_s, fmaf(-LN2, u / (1.f + s), log_s)};
}

// log p of logit x in a row with these results.
__device__ __forceinline__ float log_prob(float x, const RowScores& r, float scale) {
  if (r.log_s == NEG_INF) return NEG_INF;
  return (x - r.m) * scale - r.log_s;
}

__device__ __forceinline__ float given_log_prob(int32_t target, int64_t vocab, float x, const RowScores& r, float scale) {
  if (target < 0) return 0.f;
  return target < vocab ? log_prob(x, r, scale) : __builtin_nanf("");
}

// The gradient of a row with respect to its logits, G_j = a p_j + b p_j d_j with
// p_j = 2^d_j and d_j = (x_j - m) c - log2 s.  At the given token a p_j + g would
// cancel where p_j is near 1 (a sure token: 1 - p_j of 3e-4 would keep 11 bits),
// so there it is h p_j + b p_j d_j - g (p_j - 1): h is the entropy's share of a.
struct RowGrad {
  float m, l2, a, b, g, h;
  int32_t target;
  bool zero;
};
__device__ __forceinline__ RowGrad row_grad(const int32_t* targets, const float* stats, const float* entropy,
                                            const float* grad_logprobs, const float* grad_entropy, int64_t row,
                                            int64_t vocab, float scale) {
  RowGrad r;
  r.target = targets ? targets[row] : -1;
  r.m = stats[2 * row];
  const float log_s = stats[2 * row + 1];
  const float gl = grad_logprobs && r.target >= 0 ? grad_logprobs[row] : 0.f;
  const float ge = grad_entropy ? grad_entropy[row] : 0.f;
  const float h = grad_entropy ? entropy[row] : 0.f;
  r.l2 = log_s * LOG2E;
  r.a = -scale * (gl + ge * h);
  r.b = -scale * ge * LN2;
  r.g = scale * gl;
  r.h = -scale * ge * h;
  r.zero = (gl == 0.f && ge == 0.f) || log_s == NEG_INF;
  if (r.target >= vocab) r.a = __builtin_nanf("");
  return r;
}
// (p is 0 long before d reaches -1e4, where d is held so that 0 times -inf does not arise)
__device__ __forceinline__ float grad_of(float x, float c, const RowGrad& r) {
  const float d = fmaf(x - r.m, c, -r.l2);
  return __builtin_amdgcn_exp2f(d) * fmaf(fmaxf(d, -1e4f), r.b, r.a);
}
// A logit that is computed again (by tiles of another shape) differs from the
// statistics' in its last bits, which next to a small log s are not small.  But
// where log2 s is below 0.36 all others come to less than 0.29 of the largest
// entry: one within a factor of 2^-0.7 of it is itself the largest, and d is -log2 s.
__device__ __forceinline__ float grad_of_given(float x, float c, const RowGrad& r) {
  const bool largest = r.l2 < 0.36f && (x - r.m) * c > -0.7f;
  const float d = largest ? -r.l2 : fmaf(x - r.m, c, -r.l2);
  return fmaf(__builtin_amdgcn_exp2f(d), fmaf(fmaxf(d, -1e4f), r.b, r.h), -r.g * expm1f(d * LN2));
}

inline bool score_type(int32_t type) { return type == TT_F32 || type == TT_BF16 || type == TT_F16; }
inline bool good_scale(float scale) { return scale > 0.f && scale < __builtin_inff(); }

}  // namespace tt
