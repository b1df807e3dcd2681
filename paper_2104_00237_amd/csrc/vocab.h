// Row statistics, targets and tiles that the vocabulary losses' kernels share.
//
//   s = X W^T, z = s or cap tanh(s / cap), u = z / T, lse = log sum_v exp u_v
//   cross-entropy  loss = lse - z_y + c lse^2              dz_v = g (p_v (1 + 2 c lse) - [v = y])
//   distillation   loss = T^2 sum_j q_j (log q_j - u_j + lse)   dz_v = g T (p_v - sum of q_j with id_j = v)
//   ds = dz (1 - (z / cap)^2)
// Cross-entropy is distillation from one entry with q = 1 (T = 1, log q = 0) but for c.
#pragma once

#include "gemm_common.h"

namespace opfuse {

// Statistics are a maximum and the sum of exponentials below it.  A maximum of -infinity: nothing yet, or
// logits of -infinity only; a NaN logit makes the sum NaN (a maximum alone would pass over it).
__device__ __forceinline__ float stat_shift(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = __fadd_rn(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// tanh(x) for |x| <= 0.75 as x + x^3 R(x^2), fitted in float64 for the least relative error (3.2e-8; with fp32
// rounding at most 9.7e-8).
constexpr float kTanhNear = 0.75f;
__device__ __forceinline__ float vocab_tanh_near(float x) {
  const float u = __fmul_rn(x, x);
  float r = -4.76950407e-03f;
  r = __fmaf_rn(r, u, 1.96649302e-02f);
  r = __fmaf_rn(r, u, -5.33902645e-02f);
  r = __fmaf_rn(r, u, 1.33265212e-01f);
  r = __fmaf_rn(r, u, -3.33330691e-01f);
  return __fmaf_rn(__fmul_rn(x, u), r, x);
}
// Anywhere: beyond 0.75 as 1 - 2 e / (1 + e) with e = exp(-2 |x|), which never exceeds 1 (at most 1.9e-7 of it off,
// an ulp of the exponential and of the reciprocal counted; half a step of fp32 from |x| = 3 on).  4096 rows over 32768
// of width 1024 with logits spread by a cap of 15, this / a quotient of polynomials that exceeds 1: forward 320 / 311
// us, backward 801 / 772.
__device__ __forceinline__ float tanh_exp(float x) { return __builtin_amdgcn_exp2f(__fmul_rn(fabsf(x), -2.88539008f)); }
__device__ __forceinline__ float vocab_tanh(float x) {
  const float e = tanh_exp(x), far = __fmaf_rn(__fmul_rn(-2.f, e), __builtin_amdgcn_rcpf(__fadd_rn(1.f, e)), 1.f);
  float near = vocab_tanh_near(x);
  asm("" : "+v"(near));   // (both and a choice: the compiler makes a branch for every element of it)
  return fabsf(x) <= kTanhNear ? near : copysignf(far, x);   // (a NaN stays: e is one)
}
// 1 - tanh(x)^2 with t = tanh(x), never negative.  Beyond 0.75 from x as 4 e / (1 + e)^2 (1.8e-6 of it off): what
// a saturated t has left of 1 - t^2 is its rounding (2 % of it at x = 7, all of it from 9 on).
__device__ __forceinline__ float tanh_slope(float x, float t) {
  const float e = tanh_exp(x), r = __builtin_amdgcn_rcpf(__fadd_rn(1.f, e));
  return fabsf(x) <= kTanhNear ? __fmaf_rn(-t, t, 1.f) : __fmul_rn(__fmul_rn(4.f * e, r), r);
}
// In full precision, for fp32 operands: a relative error of 1e-7 in a logit of 10 is one of 1e-6 in its
// probability.  slope: the cap's derivative there.
__device__ __forceinline__ float vocab_cap_exact(float s, float cap, float* slope = nullptr) {
  if (slope) *slope = 1.f;
  if (cap <= 0.f) return s;
  const float x = __fdiv_rn(s, cap), t = tanhf(x);
  if (slope) *slope = tanh_slope(x, t);
  return __fmul_rn(cap, t);
}

// A row's target as a wavefront sees it: entry j has weight exp(t_j / T - top) / total.
// Entries with a negative id are left out whatever their logit; a row none of whose entries has a
// weight (none at all, or logits of -infinity only) does not count; an id past the vocabulary
// makes the row's loss NaN and its gradient zero, as does nothing else.
struct RowTarget {
  float top, total;
  bool counts, bad;
  __device__ __forceinline__ float weight(float t) const { return __fdiv_rn(expf(t - top), total); }
};
__device__ __forceinline__ float teacher_logit(const VocabArgs& a, int64_t i) {
  const float t = a.tbf ? __uint_as_float((uint32_t)((const uint16_t*)a.teacher)[i] << 16) : ((const float*)a.teacher)[i];
  return __fdiv_rn(t, a.T);
}

// A distillation row's entries, the lanes' first E each in registers: f(n, j, has, t) for entry j with its
// logit over T, n its number in the registers or -1 behind them.
template <int E>
struct RowEntries {
  float t[E];
  bool has[E], bad[E];
  __device__ __forceinline__ void load(const VocabArgs& a, int64_t row, int lane) {
    const int64_t at = row * a.k;
    int64_t id[E];
#pragma unroll
    for (int e = 0; e < E; ++e) id[e] = lane + e * 64 < a.k ? a.ids[at + lane + e * 64] : -1;
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] = lane + e * 64 < a.k ? teacher_logit(a, at + lane + e * 64) : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) has[e] = id[e] >= 0, bad[e] = id[e] >= a.V;
  }
  template <class F>
  __device__ __forceinline__ void all(const VocabArgs& a, int64_t row, int lane, F&& f) const {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (has[e]) f(e, lane + e * 64, bad[e], t[e]);
    for (int j = lane + E * 64; j < a.k; j += 64) {
      const int64_t id = a.ids[row * a.k + j];
      if (id >= 0) f(-1, j, id >= a.V, teacher_logit(a, row * a.k + j));
    }
  }
  __device__ __forceinline__ RowTarget target(const VocabArgs& a, int64_t row, int lane) const {
    RowTarget r{0.f, 1.f, false, false};
    float top = -INFINITY;
    bool past = false, nan = false;
    all(a, row, lane, [&](int, int, bool b, float x) {
      past |= b;
      nan |= x != x;
      top = fmaxf(top, x);
    });
    r.top = wave_max(top);
    r.bad = __any(past);
    r.counts = r.top != -INFINITY || __any(nan);
    r.top = stat_shift(r.top);
    float total = 0.f;
    all(a, row, lane, [&](int, int, bool, float x) { total += expf(x - r.top); });
    total = wave_sum(total);
    r.total = total == 0.f ? 1.f : total;
    return r;
  }
};
constexpr int kRowEntries = 4;   // 256 entries a row without a second load

__device__ __forceinline__ RowTarget row_target(const VocabArgs& a, int64_t row, int lane) {
  if (a.teacher == nullptr) {
    const int64_t y = a.ids[row];
    return RowTarget{0.f, 1.f, y >= 0, y >= a.V};
  }
  RowEntries<kRowEntries> e;
  e.load(a, row, lane);
  return e.target(a, row, lane);
}

// A distillation row's loss from its lse and the (capped) logits of its entries; every lane gets it.
__device__ __forceinline__ float row_loss(const VocabArgs& a, int64_t row, float lse, int lane, bool* counts) {
  RowEntries<kRowEntries> e;
  float z[kRowEntries];
#pragma unroll
  for (int n = 0; n < kRowEntries; ++n) z[n] = lane + n * 64 < a.k ? a.zt[row * a.k + lane + n * 64] : 0.f;
  e.load(a, row, lane);
  const RowTarget r = e.target(a, row, lane);
  *counts = r.counts;
  if (!r.counts) return 0.f;
  if (r.bad) return NAN;
  float loss = 0.f;
  const float log_total = logf(r.total);
  e.all(a, row, lane, [&](int n, int j, bool, float t) {
    float zt = 0.f;
    if (n < 0) zt = a.zt[row * a.k + j];
#pragma unroll
    for (int u = 0; u < kRowEntries; ++u) zt = n == u ? z[u] : zt;
    const float q = r.weight(t);
    // (an entry of weight 0 adds nothing, also where its logarithm or logit is infinite)
    if (q != 0.f) loss = __fmaf_rn(q, (t - r.top - log_total) - (__fdiv_rn(zt, a.T) - lse), loss);
  });
  return a.T * a.T * wave_sum(loss);
}

// The gradient at a place with logit z (capped): cp p - ct q, times the cap's slope there; that of an entry from its
// capped logit, which is all that the forward keeps.
__device__ __forceinline__ float place_grad(float T, float z, float slope, float lse, float cp, float ct, float q) {
  const float p = expf(__fsub_rn(__fdiv_rn(z, T), lse));
  return __fmul_rn(__fmaf_rn(cp, p, -__fmul_rn(ct, q)), slope);
}
__device__ __forceinline__ float entry_grad(float T, float cap, float z, float lse, float cp, float ct, float q) {
  const float r = cap > 0.f ? __fdiv_rn(z, cap) : 0.f;
  return place_grad(T, z, __fmaf_rn(-r, r, 1.f), lse, cp, ct, q);
}
// A label's logit for it: the forward's own where the one computed again agrees with it up to rounding.  Where a
// label has most of the probability, a rounding of its logit is in lse too and leaves p - q alone; another
// product's rounding would not (fp32 forwards and backwards change kernels at different sizes: 7701 rows over 190
// of width 3904 were 8.5e-6 from float64 instead of 2.4e-6).  A W that has moved on from the forward's has its own.
// (Distillation's entries have the forward's at every size: tiles store no logits to look at.)
__device__ __forceinline__ float entry_logit(float z, float forward) {
  return fabsf(z - forward) <= 0x1p-16f * (1.f + fabsf(forward)) ? forward : z;
}

// Statistics [parts][M] joined: lse, losses, their mean (vocab_tiles.hip).  sums: vocab_join_bytes; done: 0.
size_t vocab_join_bytes(const VocabArgs& a);
hipError_t vocab_join_launch(const VocabArgs& a, const float2* part, int parts, void* sums, int* done, hipStream_t s);

}  // namespace opfuse
