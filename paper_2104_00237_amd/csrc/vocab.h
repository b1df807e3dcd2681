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

// tanh(x) as x P(x^2) / Q(x^2), fitted in float64 for the least relative error on (0, 9] (2.1e-8; with fp32
// rounding at most 3.2e-7, rms 5.3e-8, near 0 too, where 1 - 2 / (e^2x + 1) has nothing left); beyond 9 it
// is 1 within half a step.  A third of tanhf's instructions: a capped tile of logits takes 65536 of them.
__device__ __forceinline__ float vocab_tanh(float x) {
  x = fabsf(x) > 9.f ? copysignf(9.f, x) : x;   // (a NaN stays)
  const float u = __fmul_rn(x, x);
  float p = 1.33548417e-08f, q = 7.77663388e-07f;
  p = __fmaf_rn(p, u, 2.06092191e-05f), q = __fmaf_rn(q, u, 3.28564871e-04f);
  p = __fmaf_rn(p, u, 3.49559658e-03f), q = __fmaf_rn(q, u, 2.58770157e-02f);
  p = __fmaf_rn(p, u, 1.33810326e-01f), q = __fmaf_rn(q, u, 4.67143476e-01f);
  p = __fmaf_rn(p, u, 1.f), q = __fmaf_rn(q, u, 1.f);
  return __fmul_rn(__fmul_rn(x, p), __builtin_amdgcn_rcpf(q));
}
// The same for |x| <= 0.75 as x + x^3 R(x^2), fitted likewise (3.2e-8; with rounding at most 9.7e-8): half the
// instructions again.
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
// In full precision, for fp32 operands: a relative error of 1e-7 in a logit of 10 is one of 1e-6 in its
// probability.
__device__ __forceinline__ float vocab_cap_exact(float s, float cap) { return cap > 0.f ? __fmul_rn(cap, tanhf(__fdiv_rn(s, cap))) : s; }

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

// The gradient at a place with logit z (capped): cp p - ct q, through the cap.
__device__ __forceinline__ float place_grad(float T, float cap, float z, float lse, float cp, float ct, float q) {
  const float p = expf(__fsub_rn(__fdiv_rn(z, T), lse));
  const float d = __fmaf_rn(cp, p, -__fmul_rn(ct, q));
  if (cap <= 0.f) return d;
  const float r = __fdiv_rn(z, cap);
  return __fmul_rn(d, __fmaf_rn(-r, r, 1.f));
}
// An entry's logit for it: the forward's own where the one computed again agrees with it up to rounding.  Where an
// entry has most of the probability, a rounding of its logit is in lse too and leaves p - q alone; another
// product's rounding would not (fp32 forwards and backwards change kernels at different sizes: 7701 rows over 190
// of width 3904 were 8.5e-6 from float64 instead of 2.4e-6).  A W that has moved on from the forward's has its own.
__device__ __forceinline__ float entry_logit(float z, float forward) {
  return fabsf(z - forward) <= 0x1p-16f * (1.f + fabsf(forward)) ? forward : z;
}

// Statistics [parts][M] joined: lse, losses, their mean (vocab_tiles.hip).  sums: vocab_join_bytes; done: 0.
size_t vocab_join_bytes(const VocabArgs& a);
hipError_t vocab_join_launch(const VocabArgs& a, const float2* part, int parts, void* sums, int* done, hipStream_t s);

}  // namespace opfuse
