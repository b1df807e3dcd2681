// Vocabulary losses on the bf16 matrix cores: the logits' product ends in the rows' statistics (forward)
// or in the logits' gradient (backward), so that logits exist in accumulators only.
//
// Forward: distillation's entries sorted by the tile of logits that holds them; the logits' product, whose
// tiles leave a maximum and a sum of exponentials a row and the entries' logits; the statistics joined,
// losses and their mean.
// Backward: the rows that get a gradient, gathered (what others hold is never read, and they cost no
// work); then per piece of the vocabulary the logits' product again, stored as their gradient in bf16,
// dX summed over the pieces in fp32, dW (or the update) of the piece's rows; at the end dX rounded and
// put back to its rows.  A common factor (T over the rows that count) is left out of the stored gradient
// and applied to the sums: p - 1 near -1 then rounds to itself, and what rounding the label's still leaves is
// added to dX's sums in fp32.
// Six products' worth of flops for M V K instead of the four that stored logits would need.
//
// fp32 operands take the same way as three bf16 planes each (vocab_tile.h), made beforehand: X once, W
// and the logits' gradient a piece at a time.

#include <algorithm>
#include <cstring>

#include "vocab_tile.h"

namespace opfuse {

namespace {

// Tiles (rows x columns, in wavefronts of 4x2, 2x2 and 1x1 blocks): a 256x256 tile a CU with two
// wavefronts a SIMD, 128x128 where those would not fill the chip, 32 wide for few rows.
using Big = TileShape<4, 2, 2, 4, 32, 4, 2>;
using Mid = TileShape<2, 2, 2, 2, 32, 4, 2>;
using Half = TileShape<4, 2, 2, 2, 32, 3, 2>;   // 256x128, two workgroups a CU
using FewQ = TileShape<1, 1, 4, 1, 64, 4, 2>;   // 128 x 32
using FewP = TileShape<1, 1, 1, 4, 64, 4, 2>;   // 32 x 128

constexpr int kFew = 32;                     // rows up to which a product's tiles are 32 wide

typedef uint32_t au32x4 __attribute__((ext_vector_type(4)));

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int64_t per(int64_t n, int64_t each) { return (n + each - 1) / each; }
bool odd_rows(const void* p, int64_t ld, int64_t K) { return !aligned16(p) || ld % 8 != 0 || K % 8 != 0; }

// The nearest bf16s of two values, which keep what that leaves.  What rounds to infinity leaves infinity or NaN: such a
// gradient shows.
__device__ __forceinline__ uint32_t take_part(float& x, float& y) {
  const uint32_t w = pack2(x, y);
  x = __fsub_rn(x, __uint_as_float(w << 16));
  y = __fsub_rn(y, __uint_as_float(w & 0xffff0000u));
  return w;
}
// An operand's, at most the largest bf16 (the largest fp32 values keep the rest).  An infinite value is all in its last
// part, the others are 0: that part meets only the other operand's first, whose sign and whether it is 0 are its own,
// so that the products are those of fp32 (with an infinite first part, the other operand's zeros and lower parts would
// make NaNs of them).  Two infinite factors meet nowhere: NaN.
__device__ __forceinline__ uint32_t take_operand_part(float& x, float& y, bool last) {
  if (last) return pack2(x, y);
  constexpr float most = 3.38953139e38f;
  auto part = [&](float v) { return fabsf(v) == INFINITY ? 0.f : fabsf(v) > most ? copysignf(most, v) : v; };   // (a NaN stays)
  const uint32_t w = pack2(part(x), part(y));
  x = __fsub_rn(x, __uint_as_float(w << 16));
  y = __fsub_rn(y, __uint_as_float(w & 0xffff0000u));
  return w;
}

// This wavefront's LDS writes are there for all its lanes.
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------------- forward
// Rows' entries by tile, a wavefront's rows (a group) at a time: off[group][vocabulary tile] .. of
// list[group], each entry its row in the group, its place in the tile and its number in the row.
struct Entries {
  int* off;            // [groups][vtiles + 1]
  uint32_t* list;      // [groups][rows of a group * k]
  int vtiles;
};

template <int BP, int GROUP>
__global__ __launch_bounds__(1024) void vocab_sort_kernel(VocabArgs a, Entries en, FastDiv dk, int* done) {
  extern __shared__ int bins[];   // [vtiles]
  __shared__ int waves[16];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int64_t row0 = (int64_t)blockIdx.x * GROUP;
  const int n = (int)min((int64_t)GROUP, a.M - row0) * a.k;
  const int64_t* ids = a.ids + row0 * a.k;
  if (blockIdx.x == 0 && t == 0) *done = 0;
  for (int i = t; i < en.vtiles; i += 1024) bins[i] = 0;
  __syncthreads();
  constexpr int U = 8;   // ids of a thread at a time; one batch (64 rows of 128) stays in registers
  int id[U];
  auto load = [&](int i0) {   // -1: no entry
    int64_t y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) y[u] = i0 + u * 1024 < n ? ids[i0 + u * 1024] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = y[u] >= 0 && y[u] < a.V ? (int)y[u] : -1;
  };
  for (int i0 = t; i0 < n; i0 += 1024 * U) {
    load(i0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * 1024;
      if (i >= n) continue;
      if (id[u] >= 0) atomicAdd(&bins[id[u] / BP], 1);
      else a.zt[row0 * a.k + i] = 0.f;
    }
  }
  __syncthreads();
  // exclusive sums: a run of bins each thread, then the runs' totals
  const int run = (en.vtiles + 1023) / 1024, b0 = min(en.vtiles, t * run), b1 = min(en.vtiles, b0 + run);
  int sum = 0;
  for (int b = b0; b < b1; ++b) sum += bins[b];
  int at = sum;
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(at, d);
    if (lane >= d) at += v;
  }
  if (lane == 63) waves[w] = at;
  __syncthreads();
  at -= sum;
  int all = 0;
  for (int i = 0; i < 16; ++i) {
    if (i < w) at += waves[i];
    all += waves[i];
  }
  int* off = en.off + (int64_t)blockIdx.x * (en.vtiles + 1);
  for (int b = b0; b < b1; ++b) {
    const int c = bins[b];
    off[b] = at;
    bins[b] = at;
    at += c;
  }
  if (t == 0) off[en.vtiles] = all;
  __syncthreads();
  // (the order of a tile's entries may differ from run to run: each goes to a place of its own)
  uint32_t* list = en.list + (int64_t)blockIdx.x * GROUP * a.k;
  for (int i0 = t; i0 < n; i0 += 1024 * U) {
    if (n > 1024 * U) load(i0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * 1024;
      if (i >= n || id[u] < 0) continue;
      const int tile = id[u] / BP, row = fdiv(i, dk);
      list[atomicAdd(&bins[tile], 1)] = (uint32_t)row | (uint32_t)(id[u] - tile * BP) << 8 | (uint32_t)(i - row * a.k) << 16;
    }
  }
}

constexpr float kLog2E = 1.44269504088896341f;

// Two statistics: a maximum of the (capped) logits, and the sum of exp((z - maximum) / T).  c: log2(e) / T.
// Differences are taken before they are scaled: a maximum in units of log2 would be rounded by as much
// as all the rest of lse.
__device__ __forceinline__ float2 stat2_join(float2 x, float2 y, float c) {
  const float m = fmaxf(x.x, y.x), s = stat_shift(m);
  return make_float2(m, __fmaf_rn(x.y, __builtin_amdgcn_exp2f(__fmul_rn(x.x - s, c)),
                                  __fmul_rn(y.y, __builtin_amdgcn_exp2f(__fmul_rn(y.x - s, c)))));
}

// tanh of a block's logits over their cap, and its slope there if asked for.  Trained logits stay well inside it: a
// wavefront whose 1024 all lie within 0.75 of it takes the short form.
__device__ __forceinline__ void tanh_block(vacc_t& v, float rcap, float* slope = nullptr) {
  float m = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) m = fmaxf(m, fabsf(v[r]));
  if (__all(m * rcap <= kTanhNear)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      v[r] = vocab_tanh_near(__fmul_rn(v[r], rcap));
      if (slope) slope[r] = __fmaf_rn(-v[r], v[r], 1.f);
    }
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float x = __fmul_rn(v[r], rcap);
      v[r] = vocab_tanh(x);
      if (slope) slope[r] = tanh_slope(x, v[r]);
      if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (no more of them at a time than there are registers for)
    }
  }
}
// A block's logits capped.
template <int PL>
__device__ __forceinline__ void cap_block(vacc_t& v, float cap, float rcap) {
  if constexpr (PL == 1) tanh_block(v, rcap);
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = PL == 1 ? __fmul_rn(cap, v[r]) : vocab_cap_exact(v[r], cap);
}

// A = W, B = X: a lane's accumulators are one row's logits, for statistics within the lane.
template <class T, int PL>
struct StatEpi {
  static constexpr int ROWS = ROWS_NONE;
  const int64_t* labels;   // cross-entropy: found by the tiles themselves; distillation: NULL, entries are sorted
  int64_t V;
  int* done;               // the join's count, cleared here for cross-entropy
  float2* part;        // [vtiles][M]
  float* zt;
  Entries en;
  int tile0;           // the piece's first vocabulary tile
  int64_t M;
  int k;
  float cap, rcap, c;  // c = log2(e) / T
  template <class Acc>
  __device__ __forceinline__ void operator()(const TilePlace& t, Acc& acc, const Ring& ring, int lane, int wave, int wp,
                                             int wq) const {
    constexpr int IP = T::IP, IQ = T::IQ;
    const int h4 = (lane >> 5) * 4, l32 = lane & 31;
    const int np = t.np - wp * IP * 32;   // vocabulary entries from this wavefront's first
    if (cap > 0.f) {
      each(std::make_integer_sequence<int, IP * IQ>{}, [&](auto B_) __attribute__((always_inline)) {
        cap_block<PL>(acc[decltype(B_)::value / IQ][decltype(B_)::value % IQ], cap, rcap);
      });
    }
    constexpr int GROUP = IQ * 32;
    const int tile = tile0 + t.p0 / T::BP;
    const int64_t group = t.q0 / GROUP + wq;
    int e0 = 0, e1 = 0;
    if (labels) {
      if (blockIdx.x == 0 && tile0 == 0 && wave == 0 && lane == 0) *done = 0;
      each(std::make_integer_sequence<int, IQ>{}, [&](auto J_) __attribute__((always_inline)) {
        constexpr int j = decltype(J_)::value;
        const int q = (wq * IQ + j) * 32 + l32;
        const int64_t y = q < t.nq ? labels[t.q0 + q] : -1;
        if (tile == 0 && wp == 0 && lane < 32 && q < t.nq && (y < 0 || y >= V)) zt[t.q0 + q] = 0.f;
        const int64_t far = y - ((int64_t)tile * T::BP + wp * IP * 32 + h4);
        const int label = y >= 0 && y < V && far >= 0 && far < IP * 32 ? (int)far : -1;   // from this lane's first entry
        each(std::make_integer_sequence<int, IP>{}, [&](auto I_) __attribute__((always_inline)) {
          constexpr int i = decltype(I_)::value;
          if (!__any(label >= i * 32 && label < i * 32 + 32)) return;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (i * 32 + 8 * (r >> 2) + (r & 3) == label) zt[t.q0 + q] = acc[i][j][r];
        });
      });
    } else if (wq * GROUP < t.nq) {
      const int* off = en.off + group * (en.vtiles + 1) + tile;
      e0 = off[0], e1 = off[1];
    }
    if (e1 > e0) {
      const uint32_t* list = en.list + group * GROUP * k;
      float* lds = (float*)ring_part<T, PL, 4096, T::NW>(ring, wave);
      constexpr int U = 4;   // entries of a lane at a time
      for (int b = e0; b < e1; b += 64 * U) {
        uint32_t x[U];
        int block[U];          // that of this wavefront's which holds the entry
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int e = b + u * 64 + lane;
          x[u] = e < e1 ? list[e] : 0;
          const int i = ((x[u] >> 13) & 7) - wp * IP, j = (x[u] >> 5) & 7;
          block[u] = e < e1 && i >= 0 && i < IP ? i * IQ + j : -1;
        }
#pragma unroll
        for (int i = 0; i < IP; ++i)
#pragma unroll
          for (int j = 0; j < IQ; ++j) {
            bool mine = false;
#pragma unroll
            for (int u = 0; u < U; ++u) mine |= block[u] == i * IQ + j;
            if (!__any(mine)) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) lds[(8 * (r >> 2) + h4 + (r & 3)) * 32 + l32] = acc[i][j][r];
            wave_lds_sync();
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (block[u] == i * IQ + j)
                zt[(group * GROUP + (x[u] & 255)) * k + (x[u] >> 16)] = lds[((x[u] >> 8) & 31) * 32 + (x[u] & 31)];
            wave_lds_sync();
          }
      }
    }
    float m[IQ], s[IQ];
    auto in = [&](int i, int r) { return i * 32 + 8 * (r >> 2) + h4 + (r & 3) < np; };
    if (np < IP * 32) {   // the last tile: what lies past the vocabulary has no probability
#pragma unroll
      for (int i = 0; i < IP; ++i)
#pragma unroll
        for (int j = 0; j < IQ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] = in(i, r) ? acc[i][j][r] : -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < IQ; ++j) {
      m[j] = -INFINITY;
#pragma unroll
      for (int i = 0; i < IP; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) m[j] = fmaxf(m[j], acc[i][j][r]);
      m[j] = fmaxf(m[j], __shfl_xor(m[j], 32));
      const float shift = stat_shift(m[j]);
      s[j] = 0.f;
#pragma unroll
      for (int i = 0; i < IP; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[j] = __fadd_rn(s[j], __builtin_amdgcn_exp2f(__fmul_rn(__fsub_rn(acc[i][j][r], shift), c)));
      s[j] = __fadd_rn(s[j], __shfl_xor(s[j], 32));
    }
    // the wavefronts of a row's vocabulary entries join in LDS
    static_assert(T::WP * T::BQ * 8 <= kRingBytes<T, PL>, "room for the join");
    float2* sh = (float2*)ring_part<T, PL, T::WP * T::BQ * 8, 1>(ring, 0);   // [WP][BQ]
    __syncthreads();
    if (lane < 32) {
#pragma unroll
      for (int j = 0; j < IQ; ++j) sh[wp * T::BQ + (wq * IQ + j) * 32 + l32] = make_float2(m[j], s[j]);
    }
    __syncthreads();
    const int q = wave * 64 + lane;
    if (q < T::BQ && q < t.nq) {
      float2 v = sh[q];
#pragma unroll
      for (int w = 1; w < T::WP; ++w) v = stat2_join(v, sh[w * T::BQ + q], c);
      part[(int64_t)tile * M + t.q0 + q] = v;
    }
  }
};

// Rows' statistics joined, RB rows a workgroup, and their losses.  With few workgroups the last one takes the
// mean from the workgroups' sums, in their order: a launch less; with many, each one's fence (it writes the
// XCD's L2 back) costs more than that launch (1024 of them: 31 us).
// (one row a workgroup up to kJoinFew rows; distillation: a wavefront for each row's entries)
constexpr int kJoinRows = 8, kJoinRowsTop = 4, kJoinFew = 256, kMeanFew = 32;
template <int RB>
__global__ __launch_bounds__(256) void vocab_join_kernel(VocabArgs a, const float2* part, int parts, float* counts_out,
                                                         bool in_kernel_mean, double2* sums, int* done) {
  __shared__ float2 sh[256];
  __shared__ float ll[RB], cc[RB];
  __shared__ int last;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t row0 = (int64_t)blockIdx.x * RB, row = row0 + t % RB;
  const float k = kLog2E / a.T;
  float2 v = make_float2(-INFINITY, 0.f);
  constexpr int U = 8, STEP = 256 / RB;
  for (int p = t / RB; p < parts; p += STEP * U) {
    float2 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      x[u] = p + u * STEP < parts && row < a.M ? part[(int64_t)(p + u * STEP) * a.M + row] : make_float2(-INFINITY, 0.f);
    // (one maximum for the eight: a chain of joins would be two exponentials long each)
    float m = v.x;
#pragma unroll
    for (int u = 0; u < U; ++u) m = fmaxf(m, x[u].x);
    const float shift = stat_shift(m);
    float s = __fmul_rn(v.y, __builtin_amdgcn_exp2f(__fmul_rn(v.x - shift, k)));
#pragma unroll
    for (int u = 0; u < U; ++u) s = __fmaf_rn(x[u].y, __builtin_amdgcn_exp2f(__fmul_rn(x[u].x - shift, k)), s);
    v = make_float2(m, s);
  }
  sh[t] = v;
  __syncthreads();
  for (int d = 128; d >= RB; d >>= 1) {
    if (t < d) sh[t] = stat2_join(sh[t], sh[t + d], k);
    __syncthreads();
  }
  auto lse_of = [&](int r) { return __fadd_rn(__fdiv_rn(sh[r].x, a.T), logf(sh[r].y)); };
  if (a.teacher == nullptr) {   // a row's loss by one lane
    if (t < RB) {
      float loss = 0.f;
      bool counts = false;
      if (row < a.M) {
        const float lse = lse_of(t);
        const int64_t y = a.ids[row];
        counts = y >= 0;
        if (counts) loss = y >= a.V ? NAN : __fmaf_rn(__fmul_rn(a.z_loss, lse), lse, __fsub_rn(lse, a.zt[row]));
        a.lse[row] = lse;
        a.loss[row] = loss;
      }
      ll[t] = loss;
      cc[t] = counts ? 1.f : 0.f;
      if (row < a.M) counts_out[row] = cc[t];
    }
  } else {
    for (int r = wave; r < RB; r += 4) {
      float loss = 0.f;
      bool counts = false;
      if (row0 + r < a.M) {
        const float lse = lse_of(r);
        loss = row_loss(a, row0 + r, lse, lane, &counts);
        if (lane == 0) {
          a.lse[row0 + r] = lse;
          a.loss[row0 + r] = loss;
          counts_out[row0 + r] = counts ? 1.f : 0.f;
        }
      }
      if (lane == 0) {
        ll[r] = loss;
        cc[r] = counts ? 1.f : 0.f;
      }
    }
  }
  if (!in_kernel_mean) return;
  __syncthreads();
  if (t == 0) {
    double l = 0.0, c = 0.0;
    for (int r = 0; r < RB; ++r) l += (double)ll[r], c += (double)cc[r];
    sums[blockIdx.x] = make_double2(l, c);
    __threadfence();
    last = atomicAdd(done, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  if (t == 0) {
    double l = 0.0, c = 0.0;
    for (int i = 0; i < (int)gridDim.x; ++i) l += sums[i].x, c += sums[i].y;
    *a.mean = (float)(l / fmax(c, 1.0));
  }
}

// The mean of many rows: their losses over the number that count, in float64 and one order.
__global__ __launch_bounds__(1024) void vocab_mean_kernel(const float* loss, const float* counts, int64_t M, float* mean) {
  __shared__ double sh[2][16];
  const int t = threadIdx.x;
  double l = 0.0, c = 0.0;
  constexpr int U = 8;
  for (int64_t i = t; i < M; i += 1024 * U) {
    float x[U], y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = i + u * 1024 < M ? loss[i + u * 1024] : 0.f, y[u] = i + u * 1024 < M ? counts[i + u * 1024] : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) l += (double)x[u], c += (double)y[u];
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d), c += __shfl_xor(c, d);
  if ((t & 63) == 0) sh[0][t >> 6] = l, sh[1][t >> 6] = c;
  __syncthreads();
  if (t) return;
  for (int i = 1; i < 16; ++i) l += sh[0][i], c += sh[1][i];
  *mean = (float)(l / fmax(c, 1.0));
}

// --------------------------------------------------------------------- backward
// Which rows have a gradient (2), or count without one (1); distillation: the weights' shift and sum.
__global__ __launch_bounds__(256) void vocab_flag_kernel(VocabArgs a, uint8_t* flag, float2* weight) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.M) return;
  const RowTarget r = row_target(a, row, lane);
  if (lane) return;
  flag[row] = r.counts ? r.bad ? 1 : 2 : 0;
  weight[row] = make_float2(r.top, r.total);
}

// The rows with a gradient in order: at[i] is the i-th, place[row] its number or -1, n[0] how many;
// scale: what the stored gradient leaves out.  rows[i]: lse, the factors of the probabilities and
// of the targets, the label and its logit.
struct RowCoef {
  float lse, cp, ct;
  int label;           // cross-entropy; distillation: -1
  float zt;
};
__device__ __forceinline__ RowCoef row_coef(const VocabArgs& a, int64_t row, float lse, float ct, int label) {
  // (an infinite factor makes the row's gradient NaN: a loss scale's overflow must show)
  float cp = __fmul_rn(ct, __fmaf_rn(2.f * a.z_loss, lse, 1.f));
  if (fabsf(cp) == INFINITY || fabsf(ct) == INFINITY) cp = ct = NAN;
  return RowCoef{lse, cp, ct, label, label >= 0 ? a.zt[row] : 0.f};
}
__global__ __launch_bounds__(1024) void vocab_index_kernel(VocabArgs a, const uint8_t* flag, int* at, int* place, int* n,
                                                           float* scale, RowCoef* rows) {
  __shared__ int waves[16], counted[16];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  constexpr int U = 8;   // 64 rows each at a time
  // (a run of rows each wavefront: one scan of the workgroup, not one every 1024 rows)
  const int64_t run = ((a.M + 15) / 16 + 63) / 64 * 64, r0 = min(a.M, w * run), r1 = min(a.M, r0 + run);
  auto kinds = [&](int64_t r, int (&f)[U], int (&label)[U]) {   // of rows r + 64 u + lane
    if (a.teacher) {
#pragma unroll
      for (int u = 0; u < U; ++u) f[u] = r + u * 64 + lane < r1 ? flag[r + u * 64 + lane] : 0, label[u] = -1;
    } else {
      int64_t y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) y[u] = r + u * 64 + lane < r1 ? a.ids[r + u * 64 + lane] : -1;
#pragma unroll
      for (int u = 0; u < U; ++u) f[u] = y[u] < 0 ? 0 : y[u] >= a.V ? 1 : 2, label[u] = (int)y[u];
    }
  };
  int mine = 0, counts = 0, f[U], label[U];
  for (int64_t r = r0; r < r1; r += 64 * U) {
    kinds(r, f, label);
#pragma unroll
    for (int u = 0; u < U; ++u) mine += __popcll(__ballot(f[u] == 2)), counts += __popcll(__ballot(f[u] != 0));
  }
  if (lane == 0) waves[w] = mine, counted[w] = counts;
  __syncthreads();
  int before = 0, all = 0, c = 0;
  for (int i = 0; i < 16; ++i) {
    if (i < w) before += waves[i];
    all += waves[i];
    c += counted[i];
  }
  if (t == 0) {
    *n = all;
    *scale = a.dloss ? 1.f : (float)((double)a.T / (double)max(c, 1));
  }
  for (int64_t r = r0; r < r1; r += 64 * U) {
    kinds(r, f, label);
    float lse[U], g[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = r + u * 64 + lane;
      lse[u] = row < r1 ? a.lse[row] : 0.f;
      g[u] = row < r1 && a.dloss ? __fmul_rn(a.dloss[row], a.T) : 1.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = r + u * 64 + lane;
      const uint64_t b = __ballot(f[u] == 2);
      const int to = before + __popcll(b & ((1ull << lane) - 1));
      before += __popcll(b);
      if (row >= r1) continue;
      place[row] = f[u] == 2 ? to : -1;
      if (f[u] != 2) continue;
      at[to] = (int)row;
      rows[to] = row_coef(a, row, lse[u], g[u], label[u]);
    }
  }
}

// dst[i] = rows at[i] of src (at NULL: row i), n of them, widened to ldd with zeros; fp32 rows as three
// planes, `plane` elements apart.
template <int PL>
__global__ __launch_bounds__(256) void vocab_gather_kernel(const void* srcp, int64_t lds, const int* at, const int* n,
                                                           int64_t rows, int64_t K, uint16_t* dst, int64_t ldd, int64_t plane,
                                                           int vec) {
  const int64_t count = n ? *n : rows, each = ldd / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count * each; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / each, c = (i - r * each) * 8, from = (at ? at[r] : r) * lds + c;
    uint16_t* d = dst + r * ldd + c;
    if constexpr (PL == 1) {
      const uint16_t* s = (const uint16_t*)srcp + from;
      uint4 v;
      if (vec) {
        v = *reinterpret_cast<const uint4*>(s);
      } else {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = c + e < K ? s[e] : 0;
        v = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
      }
      *reinterpret_cast<uint4*>(d) = v;
    } else {
      const float* s = (const float*)srcp + from;
      float x[8];
      if (vec) {
        const float4 a = ld4(s), b = ld4(s + 4);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = c + e < K ? s[e] : 0.f;
      }
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = take_operand_part(x[2 * e], x[2 * e + 1], p == 2);
        *reinterpret_cast<uint4*>(d + p * plane) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}

// Up to kPrepared rows: all of the above in one launch, a workgroup a row.  Rows without a gradient stay, as
// zeros; counts is for the mean's scale, which the logits' product takes.  Gathered / prepared, whole backward in
// us with a tenth of the rows left out: 137 rows over 5003 of width 320 28.6 / 26.4, 300 over 8192 of 512 49.8 /
// 46.6, 579 over 338 of 4160 51.3 / 52.8, 1024 over 32768 of 1024 216 / 219.
constexpr int kPrepared = 384;
template <int PL>
__global__ __launch_bounds__(256) void vocab_prepared_kernel(VocabArgs a, int* at, int* place, int* n, float* scale, float* counts,
                                                             RowCoef* rows, float2* weight, uint16_t* x, int64_t ldd,
                                                             int64_t plane, int twice) {
  __shared__ int on;
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  if (t < 64) {
    const RowTarget r = row_target(a, row, t);
    if (t == 0) {
      const bool live = r.counts && !r.bad;
      const float lse = a.lse[row], ct = a.dloss ? __fmul_rn(a.dloss[row], a.T) : 1.f;
      rows[row] = live ? row_coef(a, row, lse, ct, a.teacher ? -1 : (int)a.ids[row]) : RowCoef{0.f, 0.f, 0.f, -1, 0.f};
      weight[row] = make_float2(r.top, r.total);
      at[row] = (int)row;
      place[row] = live ? (int)row : -1;
      counts[row] = r.counts ? 1.f : 0.f;
      if (row == 0) {
        n[0] = (int)a.M;
        n[1] = 2 * n[0];
        if (a.dloss) *scale = 1.f;
      }
      on = live;
    }
  }
  __syncthreads();
  const bool live = on != 0;
  for (int64_t c = t * 2; c < ldd; c += 512) {
    float v[2] = {0.f, 0.f};
    uint16_t* d = x + row * ldd + c;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (!live || c + e >= a.K) continue;
      const int64_t i = row * a.ldx + c + e;
      v[e] = PL == 1 ? __uint_as_float((uint32_t)((const uint16_t*)a.x)[i] << 16) : ((const float*)a.x)[i];
    }
    if constexpr (PL == 1) {
      const uint32_t two = __float_as_uint(v[0]) >> 16 | (__float_as_uint(v[1]) & 0xffff0000u);
      *reinterpret_cast<uint32_t*>(d) = two;
      if (twice) *reinterpret_cast<uint32_t*>(d + plane) = two;
    } else {
#pragma unroll
      for (int p = 0; p < 3; ++p) *reinterpret_cast<uint32_t*>(d + p * plane) = take_operand_part(v[0], v[1], p == 2);
    }
  }
}

// A = W, B = X again: the gradient of a row's logits (distillation: but for its entries), rounded to bf16 or
// in three planes, stored [row][vocabulary] through the ring, in 16-byte pieces of whole rows.
// A row's gradient is mostly its label's, and one rounding of that to bf16 (up to 2^-8) is a common factor of the
// row's dX, where the others' roundings average out: what it leaves is kept (rest: id, value) and taken with W's
// row when dX is stored.  dW adds rows up, which averages too unless they are few: up
// to kTwo of them have a second plane, which dW's reduction takes as more rows (backward, one plane / two, us: 64
// rows over 5003 of width 320 26.5 / 27.2, over 32768 of 1024 61.9 / 65.1, 128 of those 82.3 / 97.9).
constexpr int kTwo = 64;
static_assert(kTwo <= kPrepared, "the second plane's rows follow the first's");
template <class Shape_, int PL, bool TWO>
struct GradEpi {
  static constexpr int NP = TWO ? 2 : PL;
  static constexpr int ROWS = ROWS_Q;
  const RowCoef* rows;
  uint16_t* dz;
  int64_t ldz, plane;
  float cap, rcap, rT;
  int v0;              // the piece's first vocabulary entry
  const float* counts; // of prepared rows without given gradients, for the scale; else NULL
  int M;
  float* scale;
  float T;
  int2* rest;          // bf16 cross-entropy; else NULL
  template <class Acc>
  __device__ __forceinline__ void operator()(const TilePlace& t, Acc& acc, const Ring& ring, int lane, int wave, int wp,
                                             int wq) const {
    constexpr int IP = Shape_::IP, IQ = Shape_::IQ, SLOTS = IP * 4;   // 16-byte pieces of a row in LDS
    const int h = lane >> 5, l32 = lane & 31;
    const int np = t.np - wp * IP * 32, nq = t.nq - wq * IQ * 32;
    if (counts && blockIdx.x == 0 && wave == 0 && v0 == 0) {
      float c = 0.f;
      for (int i = lane; i < M; i += 64) c += counts[i];
      c = wave_sum(c);   // (whole numbers: exact)
      if (lane == 0) *scale = T / fmaxf(c, 1.f);
    }
    RowCoef rc[IQ];
#pragma unroll
    for (int j = 0; j < IQ; ++j) {
      rc[j] = RowCoef{0.f, 0.f, 0.f, -1, 0.f};
      if (j * 32 + l32 < nq) rc[j] = rows[t.q0 + (wq * IQ + j) * 32 + l32];
    }
    auto fill = [&](auto J_, auto Capped) __attribute__((always_inline)) {
      constexpr int j = decltype(J_)::value;
      // a row without a gradient (a prepared one that does not count, of zeros) keeps nothing of an infinite W
      const bool none = rc[j].cp == 0.f && rc[j].ct == 0.f, some_none = __any(none);
      each(std::make_integer_sequence<int, IP>{}, [&](auto I_) __attribute__((always_inline)) {
        constexpr int i = decltype(I_)::value;
        // the label among this block's entries
        const int label = rc[j].label < 0 ? -1 : rc[j].label - v0 - t.p0 - (wp * IP + i) * 32 - h * 4;
        const bool here = __any(label >= 0 && label < 32);
        constexpr bool capped = decltype(Capped)::value;
        // bf16 operands: what is left of the logit is tanh alone, and lse is taken off in units of log2 (its
        // rounding there is one of lse's own size, |lse| 2^-24 of a probability: 1e-6 at 16)
        float slope[16];
        if constexpr (capped && PL == 1) tanh_block(acc[i][j], rcap, slope);
        float at_label = 0.f;
        const float c2 = rT * kLog2E * (capped ? cap : 1.f), lse2 = rc[j].lse * kLog2E;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float d, z;
          if constexpr (PL == 1) {
            const float x = acc[i][j][r];   // the logit over its cap
            z = capped ? __fmul_rn(cap, x) : x;
            d = __builtin_amdgcn_exp2f(__fmaf_rn(x, c2, -lse2));
          } else {
            z = vocab_cap_exact(acc[i][j][r], capped ? cap : 0.f, &slope[r]);
            d = __builtin_amdgcn_exp2f(__fmul_rn(kLog2E, __fmaf_rn(z, rT, -rc[j].lse)));
          }
          d = __fmul_rn(d, rc[j].cp);
          d = capped ? __fmul_rn(d, slope[r]) : d;
          acc[i][j][r] = d;
          if (here) at_label = 8 * (r >> 2) + (r & 3) == label ? z : at_label;
        }
        if (some_none) {
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] = none ? 0.f : acc[i][j][r];
        }
        if (here) {
          const float d = none ? 0.f : entry_grad(T, cap, entry_logit(at_label, rc[j].zt), rc[j].lse, rc[j].cp, rc[j].ct, 1.f);
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] = 8 * (r >> 2) + (r & 3) == label ? d : acc[i][j][r];
          if (rest && label >= 0 && label < 32 && !(label & 4)) {
            float left = d, none = 0.f;
            take_part(left, none);
            rest[t.q0 + (wq * IQ + j) * 32 + l32] = make_int2(rc[j].label, __float_as_int(left));
          }
        }
        if (np < IP * 32) {   // the piece's last tile: zeros to the end of its 16-byte pieces
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] = i * 32 + 8 * (r >> 2) + h * 4 + (r & 3) < np ? acc[i][j][r] : 0.f;
        }
      });
    };
    // 32 rows at a time, by turns in two parts of the ring: lanes of a store take SLOTS pieces each of 64 / SLOTS rows
    const int s16 = lane % SLOTS, q0 = lane / SLOTS;
    const uint32_t off = s16 * 8 < np ? (uint32_t)((q0 * ldz + s16 * 8) * 2) : kOOB;
    const uint32_t step = (uint32_t)(64 / SLOTS * ldz * 2);
    each(std::make_integer_sequence<int, IQ>{}, [&](auto J_) __attribute__((always_inline)) {
      constexpr int j = decltype(J_)::value;
      if (cap > 0.f) fill(J_, std::true_type{});
      else fill(J_, std::false_type{});
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        char* lds = ring_part<Shape_, PL, IP * 2048, Shape_::NW * 2>(ring, wave * 2 + ((j * NP + p) & 1));
#pragma unroll
        for (int i = 0; i < IP; ++i)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int slot = (i * 4 + g) ^ (l32 & (SLOTS - 1));
            uint2 w;
            if constexpr (NP == 1) {
              w = make_uint2(pack2(acc[i][j][4 * g], acc[i][j][4 * g + 1]), pack2(acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]));
            } else {
              float x[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = acc[i][j][4 * g + e];
              w.x = take_part(x[0], x[1]);
              w.y = take_part(x[2], x[3]);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][j][4 * g + e] = x[e];
            }
            *reinterpret_cast<uint2*>(lds + l32 * (IP * 64) + slot * 16 + h * 8) = w;
          }
        wave_lds_sync();
        // (rows up to 2^21 elements apart, 32 of them)
        const rsrc_t out = make_rsrc(dz + p * plane + ((int64_t)t.q0 + (wq * IQ + j) * 32) * ldz + t.p0 + wp * IP * 32);
#pragma unroll
        for (int u = 0; u < 32 * SLOTS / 64; ++u) {
          const int q = u * (64 / SLOTS) + q0;
          const au32x4 v = *reinterpret_cast<const au32x4*>(lds + q * (IP * 64) + (s16 ^ (q & (SLOTS - 1))) * 16);
          __builtin_amdgcn_raw_buffer_store_b128(v, out, j * 32 + q < nq ? off + u * step : kOOB, 0, 0);
        }
      }
    });
  }
};

// Distillation, the entries' places in a piece: p less the weights of all the row's entries that name it, by
// the first of them, from the logit that the forward kept.
// rest (bf16): as GradEpi's, of the entry with the largest so far.
template <int NP>
__global__ __launch_bounds__(256) void vocab_entry_kernel(VocabArgs a, const int* at, const int* n, const RowCoef* rows,
                                                          const float2* weight, int64_t v0, int64_t nv, uint16_t* dz,
                                                          int64_t ldz, int64_t plane, int2* rest) {
  __shared__ __attribute__((aligned(16))) int places[4][kTopMax];   // in the piece, or -1
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int i = blockIdx.x * 4 + w;
  if (i >= *n) return;
  const int64_t row = at[i], first = row * a.k;
  const int k4 = (a.k + 3) & ~3;
  for (int j = lane; j < k4; j += 64) {
    const int64_t id = j < a.k ? a.ids[first + j] : -1;
    places[w][j] = id >= v0 && id < v0 + nv ? (int)(id - v0) : -1;
  }
  wave_lds_sync();
  const RowTarget r{weight[row].x, weight[row].y, true, false};
  const RowCoef rc = rows[i];
  int2 most = rest && v0 > 0 && lane == 0 ? rest[i] : make_int2(-1, 0);
  if (rc.cp == 0.f && rc.ct == 0.f) {   // (zeros already)
    if (rest && lane == 0) rest[i] = most;
    return;
  }
  for (int j0 = 0; j0 < a.k; j0 += 64) {
    const int j = j0 + lane, place = j < a.k ? places[w][j] : -1;
    if (!__any(place >= 0)) continue;
    // (entries that name one place twice are rare: four compares an LDS read, weights only where one matches)
    float q = place >= 0 ? r.weight(teacher_logit(a, first + j)) : 0.f;
    bool lead = place >= 0;
    for (int e = 0; e < k4; e += 4) {
      const int4 p = *reinterpret_cast<const int4*>(&places[w][e]);
      const int x[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (x[u] != place || place < 0 || e + u == j) continue;
        lead &= e + u > j;
        q = __fadd_rn(q, r.weight(teacher_logit(a, first + e + u)));
      }
    }
    if (!lead) continue;
    uint16_t* d = dz + (int64_t)i * ldz + place;
    float x = entry_grad(a.T, a.cap, a.zt[first + j], rc.lse, rc.cp, rc.ct, q), y = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      d[p * plane] = (uint16_t)take_part(x, y);
      if (p == 0 && fabsf(x) > fabsf(__int_as_float(most.y))) most = make_int2((int)v0 + place, __float_as_int(x));
    }
  }
  if (!rest) return;
  const float big = wave_max(fabsf(__int_as_float(most.y)));
  const uint64_t who = __ballot(most.x >= 0 && fabsf(__int_as_float(most.y)) == big);
  if (who ? lane == __ffsll((unsigned long long)who) - 1 : lane == 0) rest[i] = most;
}

// Sums of a part of the reduction: stored, or added to those of the pieces before.
template <class T, int ROWS_DIM>
struct PartEpi {
  static constexpr int ROWS = ROWS_DIM;
  float* out;          // [S][rows][ld]
  int64_t rows, ld;
  int add;
  template <class Acc>
  __device__ __forceinline__ void operator()(const TilePlace& t, Acc& acc, const Ring&, int lane, int, int wp, int wq) const {
    const int np = t.np - wp * T::IP * 32, nq = t.nq - wq * T::IQ * 32, h4 = (lane >> 5) * 4, l32 = lane & 31;
    float* o = out + ((int64_t)t.split * rows + t.p0 + wp * T::IP * 32) * ld + t.q0 + wq * T::IQ * 32;
    auto store = [&](auto Add) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < T::IP; ++i)
#pragma unroll
        for (int j = 0; j < T::IQ; ++j) {
          const bool in = j * 32 + l32 < nq;
          float v[16];
          if constexpr (decltype(Add)::value) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int p = i * 32 + 8 * (r >> 2) + h4 + (r & 3);
              v[r] = in && p < np ? o[p * ld + j * 32 + l32] : 0.f;
            }
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int p = i * 32 + 8 * (r >> 2) + h4 + (r & 3);
            if (in && p < np) o[p * ld + j * 32 + l32] = decltype(Add)::value ? __fadd_rn(v[r], acc[i][j][r]) : acc[i][j][r];
          }
        }
    };
    if (add) store(std::true_type{});
    else store(std::false_type{});
  }
};

// dW of a piece's rows: a gradient stored (or added), or the update.
struct HeadGrad {
  const float* scale;
  void* dw;            // NULL: update
  int gbf, accumulate;
  int64_t K;
  of_param W;
  const float* gW;
  OptK opt;
  __device__ __forceinline__ void store(int64_t i, float g) const {
    if (gbf) {
      uint16_t* d = (uint16_t*)dw + i;
      *d = f32_to_bf16(accumulate ? __fadd_rn(__uint_as_float((uint32_t)*d << 16), g) : g);
    } else {
      float* d = (float*)dw + i;
      *d = accumulate ? __fadd_rn(*d, g) : g;
    }
  }
};

template <class T, bool UPDATE>
struct HeadEpi {
  static constexpr int ROWS = ROWS_R;
  HeadGrad g;
  template <class Acc>
  __device__ __forceinline__ void operator()(const TilePlace& t, Acc& acc, const Ring&, int lane, int, int wp, int wq) const {
    if constexpr (UPDATE) {
      // (the optimizer tested once, not at each element: update of 32768 x 1024 over 1024 fp32 rows 1184 -> 1166 us)
      OptK o = g.opt;
      opt_prepare(o);
      if (o.kind == OF_OPT_ADAMW) run<OF_OPT_ADAMW>(t, acc, o, lane, wp, wq);
      else if (o.kind == OF_OPT_ADAM) run<OF_OPT_ADAM>(t, acc, o, lane, wp, wq);
      else run<-1>(t, acc, o, lane, wp, wq);
    } else {
      run<-1>(t, acc, g.opt, lane, wp, wq);
    }
  }
  template <int KIND, class Acc>
  __device__ __forceinline__ void run(const TilePlace& t, Acc& acc, OptK o, int lane, int wp, int wq) const {
    if constexpr (KIND >= 0) o.kind = KIND;
    const int np = t.np - wp * T::IP * 32, nq = (int)min((int64_t)t.nq, g.K - t.q0) - wq * T::IQ * 32;
    const int h4 = (lane >> 5) * 4, l32 = lane & 31;
    const int64_t org = (int64_t)(t.p0 + wp * T::IP * 32) * g.K + t.q0 + wq * T::IQ * 32;
    const float scale = *g.scale;
    // bf16: lanes 2l and 2l + 1 trade a value so that each stores two columns of a row
    const bool pair = !UPDATE && g.gbf && !g.accumulate && g.K % 2 == 0 && ((uintptr_t)g.dw & 3u) == 0;
    auto at = [&](int r) { return 8 * (r >> 2) + h4 + (r & 3); };
    constexpr int N = 8;
    OptState1 st[2][N];
    float e[2][N];
    auto fetch = [&](auto G_) __attribute__((always_inline)) {   // the states of elements N G .. of this lane
      constexpr int G = decltype(G_)::value, r0 = G % (16 / N) * N, i = G / (16 / N) / T::IQ, j = G / (16 / N) % T::IQ;
#pragma unroll
      for (int r = 0; r < N; ++r) {
        if (j * 32 + l32 >= nq || at(r0 + r) >= np - i * 32) continue;
        const int64_t x = org + (i * 32 + at(r0 + r)) * g.K + j * 32 + l32;
        st[G & 1][r] = opt_load1(o, g.W, x);
        e[G & 1][r] = g.gW ? g.gW[x] : 0.f;
      }
    };
    if constexpr (UPDATE) fetch(std::integral_constant<int, 0>{});
    each(std::make_integer_sequence<int, T::IP * T::IQ>{}, [&](auto B_) __attribute__((always_inline)) {
      constexpr int i = decltype(B_)::value / T::IQ, j = decltype(B_)::value % T::IQ;
      const int q = j * 32 + l32, n = np - i * 32;
      const int64_t o0 = org + (int64_t)i * 32 * g.K + q;
      if constexpr (UPDATE) {
        // (the states of the next elements are asked for before these are updated)
        each(std::make_integer_sequence<int, 16 / N>{}, [&](auto R_) __attribute__((always_inline)) {
          constexpr int g0 = decltype(B_)::value * (16 / N) + decltype(R_)::value;
          if constexpr (g0 + 1 < T::IP * T::IQ * (16 / N)) fetch(std::integral_constant<int, g0 + 1>{});
#pragma unroll
          for (int r = 0; r < N; ++r) {
            constexpr int r0 = decltype(R_)::value * N;
            if (q >= nq || at(r0 + r) >= n) continue;
            const float d = __fmul_rn(acc[i][j][r0 + r], scale);
            opt_apply1(o, g.W, st[g0 & 1][r], g.gW ? __fadd_rn(e[g0 & 1][r], d) : d, o0 + at(r0 + r) * g.K);
          }
        });
      } else if (pair) {
        const bool odd = lane & 1;
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const float x = __fmul_rn(acc[i][j][r], scale), y = __fmul_rn(acc[i][j][r + 1], scale);
          const float mine = odd ? y : x, give = odd ? x : y;
          const float got = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(give), 0xb1, 0xf, 0xf, true));   // lane ^ 1
          const int p = at(r) + (odd ? 1 : 0);
          if (q < nq && p < n)
            *reinterpret_cast<uint32_t*>((uint16_t*)g.dw + (o0 - (odd ? 1 : 0) + p * g.K)) = odd ? pack2(got, mine) : pack2(mine, got);
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (q < nq && at(r) < n) g.store(o0 + at(r) * g.K, __fmul_rn(acc[i][j][r], scale));
      }
    });
  }
};

// The same from parts [S][rows][ld], summed in order.
__global__ __launch_bounds__(256) void vocab_head_kernel(HeadGrad g, const float* part, int S, int64_t rows, int64_t ld) {
  const float scale = *g.scale;
  OptK o = g.opt;
  if (!g.dw) opt_prepare(o);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * g.K; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / g.K, c = i - r * g.K;
    const float* p = part + r * ld + c;
    float v = p[0];
    for (int s = 1; s < S; s += 8) {   // eight loads in flight
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = s + u < S ? p[(s + u) * rows * ld] : 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (s + u < S) v = __fadd_rn(v, x[u]);
    }
    v = __fmul_rn(v, scale);
    if (g.dw) g.store(i, v);
    else update1(o, g.W, g.gW ? __fadd_rn(g.gW[i], v) : v, i);
  }
}

// W's rows of a piece that dX still takes (rest), before the update.
__global__ __launch_bounds__(256) void vocab_rest_kernel(const int2* rest, const int* n, int64_t v0, int64_t nv, const uint16_t* w,
                                                         int64_t K, uint16_t* kept, int64_t ld) {
  const int64_t count = *n;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count * K; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / K, c = i - r * K, id = rest[r].x;
    if (id >= v0 && id < v0 + nv) kept[r * ld + c] = w[id * K + c];
  }
}

// dX from its parts [S][M][ld]: their sum in order and the rest (of W, or kept rows of it), scaled, at its row;
// zeros where a row has none.
template <int V>
__global__ __launch_bounds__(256) void vocab_dx_kernel(const float* part, int S, int64_t M, int64_t ld, const int* place,
                                                       const float* scale, int64_t K, void* dx, int64_t ldx, int gbf, const int2* rest,
                                                       const uint16_t* w, int64_t ldw, int kept) {
  const float f = *scale;
  const int64_t each = K / V;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * each; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / each, c = (i - row * each) * V;
    const int r = place[row];
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
    if (r >= 0) {
      const float* p = part + (int64_t)r * ld + c;
      for (int s = 0; s < S; s += 8) {   // eight loads in flight
        float x[8][V];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          if constexpr (V == 4) {
            const float4 y = s + u < S ? ld4(p + (s + u) * M * ld) : make_float4(0.f, 0.f, 0.f, 0.f);
            x[u][0] = y.x, x[u][1] = y.y, x[u][2] = y.z, x[u][3] = y.w;
          } else {
            x[u][0] = s + u < S ? p[(s + u) * M * ld] : 0.f;
          }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = __fadd_rn(v[e], x[u][e]);
      }
      const int2 left = rest ? rest[r] : make_int2(-1, 0);
      if (left.x >= 0) {
        const uint16_t* y = w + (kept ? r : left.x) * ldw + c;
        uint32_t x[V];
        if constexpr (V == 4) {
          const uint2 z = *reinterpret_cast<const uint2*>(y);
          x[0] = z.x << 16, x[1] = z.x & 0xffff0000u, x[2] = z.y << 16, x[3] = z.y & 0xffff0000u;
        } else {
          x[0] = (uint32_t)y[0] << 16;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = __fmaf_rn(__int_as_float(left.y), __uint_as_float(x[e]), v[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = __fmul_rn(v[e], f);
    if constexpr (V == 4) {
      if (gbf) *reinterpret_cast<uint2*>((uint16_t*)dx + row * ldx + c) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
      else st4((float*)dx + row * ldx + c, make_float4(v[0], v[1], v[2], v[3]));
    } else {
      if (gbf) ((uint16_t*)dx)[row * ldx + c] = f32_to_bf16(v[0]);
      else ((float*)dx)[row * ldx + c] = v[0];
    }
  }
}

// ------------------------------------------------------------------------ plans
enum Shape { BIG = 0, MID = 1, FEW = 2 };
struct Choice {
  Shape shape;
  int S;               // parts of the reduction
};

// Time of a product of P x Q tiles over R: rounds of workgroups, each its stages of 32 elements and an
// epilogue; parts are written and read again.  us, fitted to products of 512 to 32768 rows and columns.
// few_p, few_q: the 32-wide tiles' rows and columns where they may be taken (bf16): they read operands more often, and
// are the only ones to fill the chip with a few hundred rows over a small vocabulary (backward of 579 rows over
// 338 of width 4160: 77 -> 52 us).  grads: the gradient's epilogue, whose code a large tile runs through once
// (29 KB with 128 x 128, 11 with 128 x 32; whole backward, 128 x 128 / 128 x 32, us: 301 rows over 12345 of width
// 257 70.2 / 60.9, 300 over 8192 of 512 47.6 / 38.1; 512 over 32768 of 1024, 256 x 256 / 128 x 32: 148 / 169).
Choice choose(int64_t P, int64_t Q, int64_t R, int planes, bool split, int few_p = 0, int few_q = 0, bool grads = false) {
  Choice best{MID, 1};
  double least = 1e300;
  for (const Shape s : {BIG, MID, FEW}) {
    if (s == FEW && (!few_p || planes == 3)) continue;
    const int64_t bp = s == BIG ? 256 : s == MID ? 128 : few_p, bq = s == BIG ? 256 : s == MID ? 128 : few_q;
    const int64_t tiles = per(P, bp) * per(Q, bq);
    for (int S = 1; S <= (split ? 64 : 1); S += S < 4 ? 1 : S / 2) {
      if (S > 1 && R / S < 128) break;
      const int64_t wg = tiles * S;
      const double stages = (double)up(per(per(R, 32), S) * (planes == 3 ? 6 : 1), s == FEW ? 8 : 4);
      const double one = s == BIG   ? stages * 0.85 + (grads ? 30 : 8)
                         : s == MID ? stages * (wg > 256 ? 0.58 : 0.36) + (grads ? 16 : 4)
                                    : stages * (wg > 256 ? 0.3 : 0.18) + (grads ? 3 : 4);
      const double time = per(wg, s == BIG ? 256 : 512) * one + (S > 1 ? 2 + (double)P * Q * S * 8 / 4e6 : 0);
      if (time < least) least = time, best = Choice{s, S};
    }
  }
  return best;
}

// Parts of dX's reduction for few rows: enough workgroups for the chip, at least 256 entries each.
int few_parts(int64_t K, int64_t V) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({64, per(512, per(K, 128)), V / 256}));
}

struct TilesPlan {
  int PL;                           // planes of an operand
  int64_t Kp, piece, copied, ldz;   // widened rows; vocabulary entries of a piece, and of one whose W is copied
  Choice logits, dx, dw;
  int BP, group;                    // the logits' tiles: vocabulary entries, and rows of a wavefront
  int64_t vtiles, groups;
  int64_t px, pw, pz;               // elements of a plane of X, W and the gradient
  size_t x, w, off, list, part, sums, done;
  bool two;                         // two planes of a bf16 gradient, for dW
  size_t flag, weight, at, place, n, scale, rows, rest, kept, dz, pdx, pdw, total;
};

TilesPlan tiles_plan(const VocabArgs& a, bool bwd) {
  TilesPlan p{};
  p.PL = a.bf16 ? 1 : 3;
  p.Kp = up(a.K, 8);
  size_t here = 0;
  auto take = [&](int64_t bytes) {
    const size_t at = here;
    here += (size_t)up(bytes, 256);
    return at;
  };
  p.logits = a.M <= kFew && a.bf16 ? Choice{FEW, 1} : choose(a.V, a.M, a.K, p.PL, false, FewQ::BP, FewQ::BQ, bwd && a.bf16);
  p.BP = p.logits.shape == BIG ? 256 : 128;
  p.group = 32 * (p.logits.shape == BIG ? Big::IQ : p.logits.shape == MID ? Mid::IQ : FewQ::IQ);
  p.vtiles = per(a.V, p.BP), p.groups = per(a.M, p.group);
  // fp32 W, and W whose rows are not whole 16-byte pieces, is copied: up to 512 MB at a time, in copies of
  // one size
  const int64_t room = std::max<int64_t>(256, (1LL << 28) / (p.Kp * p.PL) / 256 * 256);
  p.copied = std::min(up(per(a.V, per(a.V, room)), 256), up(a.V, 8));
  p.two = bwd && a.bf16 && a.M <= kTwo;
  p.px = a.M * p.Kp;
  const bool whole = a.bf16 && a.aligned && a.K % 8 == 0;   // W's rows need no copy
  if (!bwd) {
    p.x = take(whole && a.ldx % 8 == 0 ? 0 : p.px * p.PL * 2);
    p.pw = p.copied * p.Kp;
    p.w = take(whole ? 0 : p.pw * p.PL * 2);
    p.off = take(a.entries ? p.groups * (p.vtiles + 1) * 4 : 0);
    p.list = take(a.entries ? p.groups * p.group * a.k * 4 : 0);
    p.part = take(p.vtiles * a.M * 8);
    p.sums = take((int64_t)vocab_join_bytes(a));
    p.done = take(4);
    p.total = here;
    return p;
  }
  // a piece's gradient takes up to 512 MB; pieces of one size
  const int64_t most = std::max<int64_t>(256, (1LL << 28) / (a.M * p.PL) / 256 * 256);
  p.piece = std::min(up(per(a.V, per(a.V, most)), 256), up(a.V, 8));
  p.copied = std::min(p.copied, p.piece);
  p.pw = p.copied * p.Kp;
  p.x = take(p.px * (p.two ? 2 : p.PL) * 2);
  p.w = take(whole ? 0 : p.pw * p.PL * 2);
  p.ldz = p.piece;
  p.pz = a.M * p.ldz;
  p.dx = a.M <= kFew && a.bf16 ? Choice{FEW, few_parts(a.K, p.piece)} : choose(a.M, a.K, p.piece, p.PL, true, FewP::BP, FewP::BQ);
  p.dw = choose(p.piece, a.K, p.two ? 2 * a.M : a.M, p.PL, true);

  p.flag = take(a.M <= kPrepared ? a.M * 4 : a.M);   // flags, or prepared rows' counts
  p.weight = take(a.M * 8);
  p.at = take(a.M * 4);
  p.place = take(a.M * 4);
  p.n = take(8);
  p.scale = take(4);
  p.rows = take(a.M * (int64_t)sizeof(RowCoef));
  p.rest = take(a.bf16 ? a.M * 8 : 0);
  p.kept = take(a.bf16 ? p.px * 2 : 0);
  p.dz = take(p.pz * (p.two ? 2 : p.PL) * 2);
  p.pdx = take((int64_t)p.dx.S * a.M * p.Kp * 4);
  p.pdw = take(p.dw.S > 1 ? (int64_t)p.dw.S * p.piece * p.Kp * 4 : 0);
  p.total = here;
  return p;
}

// An operand: its first plane, row stride and planes' distance.
struct Operand {
  const uint16_t* p;
  int64_t ld, plane;
};

template <class T, int PL, bool A, bool B, class Epi>
hipError_t product(const Operand& a, const Operand& b, int64_t P, int64_t Q, int64_t R, const int* rows, int S, const Epi& e,
                   hipStream_t s) {
  const TileProblem pr{a.p, b.p, a.ld, b.ld, (int)P, (int)Q, (int)R, rows, (int)per(P, T::BP), (int)per(Q, T::BQ), S,
                       a.plane, b.plane};
  hipLaunchKernelGGL((tile_kernel<T, PL, A, B, Epi>), dim3((unsigned)(pr.gp * pr.gq * S)), dim3(T::NT), 0, s, pr, e);
  return hipGetLastError();
}

#define TRY(x)                                    \
  do {                                            \
    const hipError_t e_ = (x);                    \
    if (e_ != hipSuccess) return e_;              \
  } while (0)

int grid_of(int64_t n) { return (int)std::min<int64_t>(8192, std::max<int64_t>(1, per(n, 256))); }

// A call's plan, workspace and stream.
template <int PL>
struct Tiles {
  const VocabArgs& a;
  TilesPlan p;
  char* ws;
  hipStream_t s;

  template <class U>
  U* at(size_t off) const { return (U*)(ws + off); }

  hipError_t gather(const void* src, int64_t lds, const int* rows_at, const int* n, int64_t rows, uint16_t* dst, int64_t plane) const {
    const int vec = PL == 1 ? !odd_rows(src, lds, a.K) : aligned16(src) && lds % 4 == 0 && a.K % 8 == 0;
    hipLaunchKernelGGL(vocab_gather_kernel<PL>, dim3(grid_of(rows * p.Kp / 8)), dim3(256), 0, s, src, lds, rows_at, n, rows, a.K,
                       dst, p.Kp, plane, vec);
    return hipGetLastError();
  }
  bool prepared() const { return a.M <= kPrepared; }
  bool copies_w() const { return PL == 3 || odd_rows(a.W.w_bf16, a.K, a.K); }
  hipError_t head(int64_t v0, int64_t n, Operand* w) const {   // W's rows [v0, v0 + n)
    if (!copies_w()) {
      *w = Operand{a.W.w_bf16 + v0 * a.K, a.K, 0};
      return hipSuccess;
    }
    *w = Operand{at<uint16_t>(p.w), p.Kp, p.pw};
    const void* src = PL == 1 ? (const void*)(a.W.w_bf16 + v0 * a.K) : (const void*)(a.W.w + v0 * a.K);
    return gather(src, a.K, nullptr, nullptr, n, at<uint16_t>(p.w), p.pw);
  }

  template <class T>
  hipError_t sort_entries() const {
    const Entries en{at<int>(p.off), at<uint32_t>(p.list), (int)p.vtiles};
    hipLaunchKernelGGL((vocab_sort_kernel<T::BP, T::IQ * 32>), dim3((unsigned)p.groups), dim3(1024), (size_t)p.vtiles * 4, s, a, en,
                       make_fastdiv((uint32_t)a.k), at<int>(p.done));
    return hipGetLastError();
  }
  template <class T>
  hipError_t stats(const Operand& x, const Operand& w, int64_t v0, int64_t n) const {
    const Entries en{at<int>(p.off), at<uint32_t>(p.list), (int)p.vtiles};
    const StatEpi<T, PL> e{a.teacher ? nullptr : a.ids, a.V, at<int>(p.done), at<float2>(p.part), a.zt, en, (int)(v0 / T::BP), a.M, a.k, a.cap, a.rcap, kLog2E / a.T};
    return product<T, PL, true, true>(w, x, n, a.M, a.K, nullptr, 1, e, s);
  }
  int2* rest() const { return PL == 1 ? at<int2>(p.rest) : nullptr; }
  template <class T, bool TWO = false>
  hipError_t grads(const Operand& w, int64_t v0, int64_t n) const {
    const GradEpi<T, PL, TWO> e{at<RowCoef>(p.rows), at<uint16_t>(p.dz), p.ldz, p.pz, a.cap, a.rcap, 1.f / a.T, (int)v0,
                           prepared() && !a.dloss ? at<const float>(p.flag) : nullptr, (int)a.M, at<float>(p.scale), a.T, a.teacher ? nullptr : rest()};
    return product<T, PL, true, true>(w, Operand{at<uint16_t>(p.x), p.Kp, p.px}, n, a.M, a.K, at<int>(p.n), 1, e, s);
  }
  template <bool TWO>
  hipError_t shaped_grads(const Operand& w, int64_t v0, int64_t nv) const {
    if constexpr (PL == 3 && TWO) {
      return hipErrorInvalidValue;
    } else {
      switch (p.logits.shape) {
        case BIG: return grads<Big, TWO>(w, v0, nv);
        case MID: return grads<Mid, TWO>(w, v0, nv);
        default:
          if constexpr (PL == 1) return grads<FewQ, TWO>(w, v0, nv);
          return hipErrorInvalidValue;
      }
    }
  }
  template <class T>
  hipError_t data_grad(const Operand& w, int64_t n, bool first) const {
    const PartEpi<T, ROWS_P> e{at<float>(p.pdx), a.M, p.Kp, first ? 0 : 1};
    return product<T, PL, true, false>(Operand{at<uint16_t>(p.dz), p.ldz, p.pz}, w, a.M, p.Kp, n, at<int>(p.n), p.dx.S, e, s);
  }
  template <class T>
  hipError_t head_grad(const HeadGrad& g, int64_t n) const {
    const Operand dz{at<uint16_t>(p.dz), p.ldz, p.pz}, x{at<uint16_t>(p.x), p.Kp, p.px};
    const int* rows = at<int>(p.n) + (p.two ? 1 : 0);
    const int64_t R = p.two ? 2 * a.M : a.M;
    if (p.dw.S > 1) {
      const PartEpi<T, ROWS_R> e{at<float>(p.pdw), n, p.Kp, 0};
      TRY((product<T, PL, false, false>(dz, x, n, p.Kp, R, rows, p.dw.S, e, s)));
      hipLaunchKernelGGL(vocab_head_kernel, dim3(grid_of(n * a.K)), dim3(256), 0, s, g, at<const float>(p.pdw), p.dw.S, n, p.Kp);
      return hipGetLastError();
    }
    if (g.dw) return product<T, PL, false, false>(dz, x, n, p.Kp, R, rows, 1, HeadEpi<T, false>{g}, s);
    // An update's tiles are smaller, two workgroups a CU.  Whole calls in us, 256x256 / these: fp32 1024 rows over 32768
    // of width 1024 1290 / 1250, 4096 over 16384 1962 / 2000; bf16 (fp32 dX) 512 rows over 32768 482 / 495, 4096
    // 1109 / 1111, of width 4096 4007 / 3942.  Both workgroups of a CU reach their updates together: the products
    // do not hide them (MFMAs 37 % busy in fp32).
    using U = std::conditional_t<std::is_same_v<T, Big>, std::conditional_t<PL == 1, Half, Mid>, T>;
    return product<U, PL, false, false>(dz, x, n, p.Kp, R, rows, 1, HeadEpi<U, true>{g}, s);
  }

  hipError_t fwd() const {
    Operand x{(const uint16_t*)a.x, a.ldx, 0};
    if (PL == 3 || odd_rows(a.x, a.ldx, a.K)) {
      TRY(gather(a.x, a.ldx, nullptr, nullptr, a.M, at<uint16_t>(p.x), p.px));
      x = Operand{at<uint16_t>(p.x), p.Kp, p.px};
    }
    if (a.teacher) {
      switch (p.logits.shape) {
        case BIG: TRY(sort_entries<Big>()); break;
        case MID: TRY(sort_entries<Mid>()); break;
        default: TRY(sort_entries<FewQ>()); break;
      }
    }
    const int64_t piece = copies_w() ? p.copied : a.V;
    for (int64_t v0 = 0; v0 < a.V; v0 += piece) {
      const int64_t n = std::min(piece, a.V - v0);
      Operand w;
      TRY(head(v0, n, &w));
      switch (p.logits.shape) {
        case BIG: TRY(stats<Big>(x, w, v0, n)); break;
        case MID: TRY(stats<Mid>(x, w, v0, n)); break;
        default:
          if constexpr (PL == 1) TRY(stats<FewQ>(x, w, v0, n));
      }
    }
    return vocab_join_launch(a, at<const float2>(p.part), (int)p.vtiles, at<double2>(p.sums), at<int>(p.done), s);
  }

  hipError_t bwd() const {
    int *rows_at = at<int>(p.at), *place = at<int>(p.place), *n = at<int>(p.n);
    float* scale = at<float>(p.scale);
    if (prepared()) {
      hipLaunchKernelGGL(vocab_prepared_kernel<PL>, dim3((unsigned)a.M), dim3(256), 0, s, a, rows_at, place, n, scale,
                         at<float>(p.flag), at<RowCoef>(p.rows), at<float2>(p.weight), at<uint16_t>(p.x), p.Kp, p.px,
                         p.two ? 1 : 0);
      TRY(hipGetLastError());
    } else {
      if (a.teacher) {
        hipLaunchKernelGGL(vocab_flag_kernel, dim3((unsigned)per(a.M, 4)), dim3(256), 0, s, a, at<uint8_t>(p.flag), at<float2>(p.weight));
        TRY(hipGetLastError());
      }
      hipLaunchKernelGGL(vocab_index_kernel, dim3(1), dim3(1024), 0, s, a, at<const uint8_t>(p.flag), rows_at, place, n, scale,
                         at<RowCoef>(p.rows));
      TRY(hipGetLastError());
      TRY(gather(a.x, a.ldx, rows_at, n, a.M, at<uint16_t>(p.x), p.px));
    }
    const int64_t piece = copies_w() ? p.copied : p.piece;
    for (int64_t v0 = 0; v0 < a.V; v0 += piece) {
      const int64_t nv = std::min(piece, a.V - v0);
      Operand w;
      TRY(head(v0, nv, &w));
      TRY(p.two ? shaped_grads<true>(w, v0, nv) : shaped_grads<false>(w, v0, nv));
      if (a.teacher) {
        auto entries = [&](auto* kernel) {
          hipLaunchKernelGGL(kernel, dim3((unsigned)per(a.M, 4)), dim3(256), 0, s, a, rows_at, n, at<const RowCoef>(p.rows),
                             at<const float2>(p.weight), v0, nv, at<uint16_t>(p.dz), p.ldz, p.pz, rest());
        };
        if (p.two) entries(vocab_entry_kernel<2>);
        else entries(vocab_entry_kernel<PL>);
        TRY(hipGetLastError());
      }
      if (a.dx) {
        switch (p.dx.shape) {
          case BIG: TRY(data_grad<Big>(w, nv, v0 == 0)); break;
          case MID: TRY(data_grad<Mid>(w, nv, v0 == 0)); break;
          default:
            if constexpr (PL == 1) TRY(data_grad<FewP>(w, nv, v0 == 0));
        }
      }
      if (a.fused && a.dx && rest()) {
        hipLaunchKernelGGL(vocab_rest_kernel, dim3(grid_of(a.M * a.K)), dim3(256), 0, s, rest(), n, v0, nv, a.W.w_bf16, a.K,
                           at<uint16_t>(p.kept), p.Kp);
        TRY(hipGetLastError());
      }
      if (!a.fused && !a.dw) continue;
      HeadGrad g{};
      g.scale = scale;
      g.K = a.K;
      g.gbf = a.gbf;
      g.accumulate = a.accumulate;
      const int64_t o = v0 * a.K;
      if (a.fused) {
        g.W = a.W;
        g.W.w += o;
        if (g.W.m) g.W.m += o;
        if (g.W.v) g.W.v += o;
        if (g.W.w_bf16) g.W.w_bf16 += o;
        g.gW = a.gW ? a.gW + o : nullptr;
        g.opt = a.opt;
      } else {
        g.dw = a.gbf ? (void*)((uint16_t*)a.dw + o) : (void*)((float*)a.dw + o);
      }
      TRY(p.dw.shape == BIG ? head_grad<Big>(g, nv) : head_grad<Mid>(g, nv));
    }
    if (!a.dx) return hipSuccess;
    const uint16_t* rw = a.fused ? at<uint16_t>(p.kept) : a.W.w_bf16;
    const bool vec = a.K % 4 == 0 && a.ldx % 4 == 0 && ((uintptr_t)a.dx) % (a.gbf ? 8 : 16) == 0 && (PL == 3 || ((uintptr_t)rw) % 8 == 0);
    const auto go = [&](auto* kernel, int each) {
      hipLaunchKernelGGL(kernel, dim3(grid_of(a.M * a.K / each)), dim3(256), 0, s, at<const float>(p.pdx), p.dx.S, a.M, p.Kp, place,
                         scale, a.K, a.dx, a.ldx, a.gbf ? 1 : 0, rest(), rw, a.fused ? p.Kp : a.K, a.fused ? 1 : 0);
    };
    if (vec) go(vocab_dx_kernel<4>, 4);
    else go(vocab_dx_kernel<1>, 1);
    return hipGetLastError();
  }
};

}  // namespace

hipError_t vocab_join_launch(const VocabArgs& a, const float2* part, int parts, void* sums, int* done, hipStream_t s) {
  // sums: the rows' counts, or up to kMeanFew workgroups' sums
  float* counts = (float*)((char*)sums + kMeanFew * sizeof(double2));
  const bool few = a.mean && a.M <= kMeanFew;
  auto go = [&](auto* kernel, int64_t rows) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)per(a.M, rows)), dim3(256), 0, s, a, part, parts, counts, few, (double2*)sums, done);
  };
  if (a.M <= kJoinFew) go(vocab_join_kernel<1>, 1);
  else if (a.teacher) go(vocab_join_kernel<kJoinRowsTop>, kJoinRowsTop);
  else go(vocab_join_kernel<kJoinRows>, kJoinRows);
  TRY(hipGetLastError());
  if (a.mean && !few) hipLaunchKernelGGL(vocab_mean_kernel, dim3(1), dim3(1024), 0, s, a.loss, counts, a.M, a.mean);
  return hipGetLastError();
}
size_t vocab_join_bytes(const VocabArgs& a) { return kMeanFew * sizeof(double2) + (size_t)a.M * 4; }

// fp32 W is made into planes first, which few rows do not pay for, and small calls lose to launches.  Pieces of
// the library's fp32 products / tiles, us: 32768 x 1024 forward 256 rows 139 / 161, 512 244 / 214, backward 128
// rows 255 / 281, 192 366 / 346, 512 796 / 557; 2048 x 512 forward 1024 rows 40 / 50, 4096 99 / 80, backward 512
// 62 / 77, 2048 153 / 118.
bool vocab_tiles_ok(const VocabArgs& a, bool bwd) {
  return a.bf16 || (bwd ? a.M >= 192 && a.M * a.V >= (1 << 21) : a.M > 400 && a.M * a.V >= (1 << 22));
}

size_t vocab_tiles_ws_bytes(const VocabArgs& a, bool bwd) { return tiles_plan(a, bwd).total; }

hipError_t vocab_tiles_fwd(const VocabArgs& a, void* ws, hipStream_t s) {
  if (a.bf16) return Tiles<1>{a, tiles_plan(a, false), (char*)ws, s}.fwd();
  return Tiles<3>{a, tiles_plan(a, false), (char*)ws, s}.fwd();
}

hipError_t vocab_tiles_bwd(const VocabArgs& a, void* ws, hipStream_t s) {
  if (a.bf16) return Tiles<1>{a, tiles_plan(a, true), (char*)ws, s}.bwd();
  return Tiles<3>{a, tiles_plan(a, true), (char*)ws, s}.bwd();
}

}  // namespace opfuse
