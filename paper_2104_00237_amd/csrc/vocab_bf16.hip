// Vocabulary losses on bf16 operands: the logits' product ends in the rows' statistics (forward) or in
// the logits' gradient (backward), so that logits exist in accumulators only.
//
// Forward, three launches: the rows' entries sorted by the tile of logits that holds them; the logits'
// product, whose tiles leave a maximum and a sum of exponentials a row and the entries' logits; the
// statistics joined, losses and their mean.
// Backward: the rows that get a gradient, gathered (what others hold is never read, and they cost no
// work); then per piece of the vocabulary the logits' product again, stored as their gradient in bf16,
// the entries' places put right, dX summed over the pieces in fp32, dW (or the update) of the piece's
// rows; at the end dX rounded and put back to its rows.  A common factor (T over the rows that count) is
// left out of the stored gradient and applied to the sums: p - 1 near -1 then rounds to itself.
// Six products' worth of flops for M V K instead of the four that stored logits would need.

#include <algorithm>
#include <cstring>

#include "vocab_tile.h"

namespace opfuse {

namespace {

// Tiles (rows x columns, in wavefronts of 4x2, 2x2 and 1x1 blocks): a 256x256 tile a CU with two
// wavefronts a SIMD, 128x128 where those would not fill the chip, 32 wide for few rows.
using Big = TileShape<4, 2, 2, 4, 32, 2>;
using Mid = TileShape<2, 2, 2, 2, 32, 2>;
using FewQ = TileShape<1, 1, 4, 1, 64, 2>;   // 128 x 32
using FewP = TileShape<1, 1, 1, 4, 64, 2>;   // 32 x 128

constexpr int kFew = 32;                     // rows up to which a product's tiles are 32 wide

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int64_t per(int64_t n, int64_t each) { return (n + each - 1) / each; }
bool odd_rows(const void* p, int64_t ld, int64_t K) { return !aligned16(p) || ld % 8 != 0 || K % 8 != 0; }

// A wavefront's own part of the ring once the main loop is done: BYTES each.
template <class T, int BYTES>
__device__ __forceinline__ char* own_lds(char* const (&ring)[4], int wave) {
  constexpr int EACH = (T::ABYTES + T::BBYTES) / BYTES;
  static_assert(EACH * 4 >= T::NW, "room for every wavefront");
  const int r = wave / EACH;
  return (r == 0 ? ring[0] : r == 1 ? ring[1] : r == 2 ? ring[2] : ring[3]) + (wave % EACH) * BYTES;
}
// This wavefront's LDS writes are there for all its lanes.
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------------- forward
// A row's entries by tile: off[row tile][vocabulary tile] .. of list[row tile], each entry its row and
// its column in the tile and its number in the row.
struct Entries {
  int* off;            // [row tiles][vtiles + 1]
  uint32_t* list;      // [row tiles][BQ * k]
  int vtiles;
};

template <int BP, int BQ>
__global__ __launch_bounds__(1024) void vocab_sort_kernel(VocabArgs a, Entries en, int* done) {
  extern __shared__ int bins[];   // [vtiles]
  __shared__ int part[1024];
  const int t = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * BQ;
  const int n = (int)min((int64_t)BQ, a.M - row0) * a.k;
  const int64_t* ids = a.ids + row0 * a.k;
  if (blockIdx.x == 0 && t == 0) *done = 0;
  for (int i = t; i < en.vtiles; i += 1024) bins[i] = 0;
  __syncthreads();
  for (int i = t; i < n; i += 1024) {
    const int64_t id = ids[i];
    if (id >= 0 && id < a.V) atomicAdd(&bins[(int)id / BP], 1);
    else a.zt[row0 * a.k + i] = 0.f;
  }
  __syncthreads();
  // exclusive sums: a run of bins each thread, the runs' totals in steps of doubling
  const int run = (en.vtiles + 1023) / 1024, b0 = min(en.vtiles, t * run), b1 = min(en.vtiles, b0 + run);
  int sum = 0;
  for (int b = b0; b < b1; ++b) sum += bins[b];
  part[t] = sum;
  __syncthreads();
  for (int d = 1; d < 1024; d <<= 1) {
    const int v = t >= d ? part[t - d] : 0;
    __syncthreads();
    part[t] += v;
    __syncthreads();
  }
  int at = part[t] - sum;
  int* off = en.off + (int64_t)blockIdx.x * (en.vtiles + 1);
  for (int b = b0; b < b1; ++b) {
    const int c = bins[b];
    off[b] = at;
    bins[b] = at;
    at += c;
  }
  if (t == 1023) off[en.vtiles] = part[1023];
  __syncthreads();
  // (the order of a tile's entries may differ from run to run: each goes to a place of its own)
  uint32_t* list = en.list + (int64_t)blockIdx.x * BQ * a.k;
  for (int i = t; i < n; i += 1024) {
    const int64_t id = ids[i];
    if (id < 0 || id >= a.V) continue;
    const int tile = (int)id / BP, row = i / a.k;
    list[atomicAdd(&bins[tile], 1)] = (uint32_t)row | (uint32_t)((int)id - tile * BP) << 8 | (uint32_t)(i - row * a.k) << 16;
  }
}

// A = W, B = X: a lane's accumulators are one row's logits, for statistics within the lane.
template <class T>
struct StatEpi {
  static constexpr int ROWS = ROWS_NONE;
  float2* part;        // [vtiles * WP][M]: maximum (in units of log2) and sum
  float* zt;
  Entries en;
  int tile0;           // the piece's first vocabulary tile
  int64_t M;
  int k;
  float cap, c;        // c = log2(e) / T
  template <class Acc>
  __device__ __forceinline__ void operator()(const TilePlace& t, Acc& acc, char* const (&ring)[4], int lane, int wave, int wp,
                                             int wq) const {
    constexpr int IP = T::IP, IQ = T::IQ;
    const int h4 = (lane >> 5) * 4, l32 = lane & 31;
    const int np = t.np - wp * IP * 32;   // vocabulary entries from this wavefront's first
    if (cap > 0.f) {
#pragma unroll
      for (int i = 0; i < IP; ++i)
#pragma unroll
        for (int j = 0; j < IQ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] = vocab_cap(acc[i][j][r], cap);
    }
    const int tile = tile0 + t.p0 / T::BP, rt = t.q0 / T::BQ;
    const int* off = en.off + (int64_t)rt * (en.vtiles + 1) + tile;
    const int e0 = off[0], e1 = off[1];
    if (e1 > e0) {
      const uint32_t* list = en.list + (int64_t)rt * T::BQ * k;
      float* lds = (float*)own_lds<T, (IP * IQ * 2048 > 4096 ? IP * IQ * 2048 : 4096)>(ring, wave);
#pragma unroll
      for (int i = 0; i < IP; ++i)
#pragma unroll
        for (int j = 0; j < IQ; ++j) {
          bool there = false;
          for (int b = e0; b < e1; b += 64) {
            const uint32_t x = b + lane < e1 ? list[b + lane] : 0;
            const int tr = x & 255, tv = (x >> 8) & 255;
            const bool mine = b + lane < e1 && (tr >> 5) == wq * IQ + j && (tv >> 5) == wp * IP + i;
            if (!__any(mine)) continue;
            if (!there) {
#pragma unroll
              for (int r = 0; r < 16; ++r) lds[(8 * (r >> 2) + h4 + (r & 3)) * 32 + l32] = acc[i][j][r];
              wave_lds_sync();
              there = true;
            }
            if (mine) zt[((int64_t)t.q0 + tr) * k + (x >> 16)] = lds[(tv & 31) * 32 + (tr & 31)];
          }
          if (there) wave_lds_sync();
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
      const float shift = __fmul_rn(stat_shift(m[j]), c);
      s[j] = 0.f;
#pragma unroll
      for (int i = 0; i < IP; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[j] = __fadd_rn(s[j], __builtin_amdgcn_exp2f(__fmaf_rn(acc[i][j][r], c, -shift)));
      s[j] = __fadd_rn(s[j], __shfl_xor(s[j], 32));
      m[j] = m[j] == -INFINITY ? m[j] : shift;
    }
    if (lane < 32) {
#pragma unroll
      for (int j = 0; j < IQ; ++j) {
        const int q = (wq * IQ + j) * 32 + l32;
        if (q < t.nq) part[((int64_t)tile * T::WP + wp) * M + t.q0 + q] = make_float2(m[j], s[j]);
      }
    }
  }
};

// Rows' statistics joined, 16 rows a workgroup; their losses; the last workgroup takes the mean from
// the workgroups' sums, in their order.
constexpr int kJoinRows = 16;
__global__ __launch_bounds__(256) void vocab_join_kernel(VocabArgs a, const float2* part, int parts, double2* sums, int* done) {
  __shared__ float2 sh[256];
  __shared__ float ll[kJoinRows], cc[kJoinRows];
  __shared__ int last;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t row0 = (int64_t)blockIdx.x * kJoinRows, row = row0 + t % kJoinRows;
  auto join = [](float2 x, float2 y) {   // in units of log2
    const float m = fmaxf(x.x, y.x), s = stat_shift(m);
    return make_float2(m, __fadd_rn(__fmul_rn(x.y, __builtin_amdgcn_exp2f(x.x - s)), __fmul_rn(y.y, __builtin_amdgcn_exp2f(y.x - s))));
  };
  float2 v = make_float2(-INFINITY, 0.f);
  constexpr int U = 8, STEP = 256 / kJoinRows;
  for (int p = t / kJoinRows; p < parts; p += STEP * U) {
    float2 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      x[u] = p + u * STEP < parts && row < a.M ? part[(int64_t)(p + u * STEP) * a.M + row] : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int u = 0; u < U; ++u) v = join(v, x[u]);
  }
  sh[t] = v;
  __syncthreads();
  for (int d = 128; d >= kJoinRows; d >>= 1) {
    if (t < d) sh[t] = join(sh[t], sh[t + d]);
    __syncthreads();
  }
  for (int r = wave; r < kJoinRows; r += 4) {
    if (row0 + r >= a.M) {
      if (lane == 0) ll[r] = cc[r] = 0.f;
      continue;
    }
    const float lse = __fmul_rn(__fadd_rn(sh[r].x, log2f(sh[r].y)), 0.693147180559945309f);
    bool counts;
    const float loss = row_loss(a, row0 + r, lse, lane, &counts);
    if (lane == 0) {
      a.lse[row0 + r] = lse;
      a.loss[row0 + r] = loss;
      ll[r] = loss;
      cc[r] = counts ? 1.f : 0.f;
    }
  }
  if (a.mean == nullptr) return;
  __syncthreads();
  if (t == 0) {
    double l = 0.0, c = 0.0;
    for (int r = 0; r < kJoinRows; ++r) l += (double)ll[r], c += (double)cc[r];
    sums[blockIdx.x] = make_double2(l, c);
    __threadfence();
    last = atomicAdd(done, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  __shared__ double2 tot[256];
  double l = 0.0, c = 0.0;
  for (int i = t; i < (int)gridDim.x; i += 256) l += sums[i].x, c += sums[i].y;
  tot[t] = make_double2(l, c);
  __syncthreads();
  for (int d = 128; d > 0; d >>= 1) {
    if (t < d) tot[t].x += tot[t + d].x, tot[t].y += tot[t + d].y;
    __syncthreads();
  }
  if (t == 0) *a.mean = (float)(tot[0].x / fmax(tot[0].y, 1.0));
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
// scale: what the stored gradient leaves out.  rows[i]: lse in units of log2, and the factors of the
// probabilities and of the targets.
struct RowCoef {
  float lse2, cp, ct;
};
__global__ __launch_bounds__(1024) void vocab_index_kernel(VocabArgs a, const uint8_t* flag, int* at, int* place, int* n,
                                                           float* scale, RowCoef* rows) {
  __shared__ int waves[16], counted[16], base;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  if (t == 0) base = 0;
  int counts = 0;
  for (int64_t r0 = 0; r0 < a.M; r0 += 1024) {
    const int64_t row = r0 + t;
    int f = 0;
    if (row < a.M) {
      if (a.teacher) {
        f = flag[row];
      } else {
        const int64_t y = a.ids[row];
        f = y < 0 ? 0 : y >= a.V ? 1 : 2;
      }
    }
    counts += f != 0;
    const uint64_t b = __ballot(f == 2);
    if (lane == 0) waves[w] = __popcll(b);
    __syncthreads();
    int before = base, all = base;
    for (int i = 0; i < 16; ++i) {
      if (i < w) before += waves[i];
      all += waves[i];
    }
    before += __popcll(b & ((1ull << lane) - 1));
    if (row < a.M) place[row] = f == 2 ? before : -1;
    if (f == 2) {
      at[before] = (int)row;
      const float ct = a.dloss ? __fmul_rn(a.dloss[row], a.T) : 1.f;
      rows[before] = RowCoef{__fmul_rn(a.lse[row], 1.44269504088896341f), __fmul_rn(ct, __fmaf_rn(2.f * a.z_loss, a.lse[row], 1.f)), ct};
    }
    __syncthreads();
    if (t == 0) base = all;
    __syncthreads();
  }
  for (int d = 32; d > 0; d >>= 1) counts += __shfl_xor(counts, d);
  if (lane == 0) counted[w] = counts;
  __syncthreads();
  if (t) return;
  int c = 0;
  for (int i = 0; i < 16; ++i) c += counted[i];
  *n = base;
  *scale = a.dloss ? 1.f : (float)((double)a.T / (double)max(c, 1));
}

// dst[i] = rows at[i] of src (at NULL: row i), n of them, widened to ldd with zeros.
__global__ __launch_bounds__(256) void vocab_gather_kernel(const uint16_t* src, int64_t lds, const int* at, const int* n,
                                                           int64_t rows, int64_t K, uint16_t* dst, int64_t ldd, int vec) {
  const int64_t count = n ? *n : rows, each = ldd / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count * each; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / each, c = (i - r * each) * 8;
    const uint16_t* s = src + (at ? at[r] : r) * lds + c;
    uint4 v;
    if (vec) {
      v = *reinterpret_cast<const uint4*>(s);
    } else {
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = c + e < K ? s[e] : 0;
      v = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    }
    *reinterpret_cast<uint4*>(dst + r * ldd + c) = v;
  }
}

// A = W, B = X again: the gradient of a row's logits but for its entries, rounded to bf16 and stored
// [row][vocabulary] through the ring, in 16-byte pieces of whole rows.
template <class T>
struct GradEpi {
  static constexpr int ROWS = ROWS_Q;
  const RowCoef* rows;
  uint16_t* dz;
  int64_t ldz;
  float cap, c;
  template <class Acc>
  __device__ __forceinline__ void operator()(const TilePlace& t, Acc& acc, char* const (&ring)[4], int lane, int wave, int wp,
                                             int wq) const {
    constexpr int IP = T::IP, IQ = T::IQ, SLOTS = IP * 4;   // 16-byte pieces of a row in LDS
    const int h = lane >> 5, l32 = lane & 31;
    const int np = t.np - wp * IP * 32, nq = t.nq - wq * IQ * 32;
    char* lds = own_lds<T, (IP * IQ * 2048 > 4096 ? IP * IQ * 2048 : 4096)>(ring, wave);
#pragma unroll
    for (int j = 0; j < IQ; ++j) {
      const int q = j * 32 + l32;
      RowCoef rc{0.f, 0.f, 0.f};
      if (q < nq) rc = rows[t.q0 + wq * IQ * 32 + q];
      const float f = cap > 0.f ? 1.f / cap : 0.f;
#pragma unroll
      for (int i = 0; i < IP; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float d[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float z = acc[i][j][g * 4 + r], more = rc.cp;
            if (cap > 0.f) {
              z = vocab_cap(z, cap);
              const float x = __fmul_rn(z, f);
              more = __fmul_rn(more, __fmaf_rn(-x, x, 1.f));
            }
            d[r] = __fmul_rn(__builtin_amdgcn_exp2f(__fmaf_rn(z, c, -rc.lse2)), more);
            if (i * 32 + g * 8 + h * 4 + r >= np) d[r] = 0.f;
          }
          const int slot = (i * 4 + g) ^ (q & (SLOTS - 1));
          *reinterpret_cast<uint2*>(lds + q * (IP * 64) + slot * 16 + h * 8) = make_uint2(pack2(d[0], d[1]), pack2(d[2], d[3]));
        }
    }
    wave_lds_sync();
    uint16_t* out = dz + ((int64_t)t.q0 + wq * IQ * 32) * ldz + t.p0 + wp * IP * 32;
#pragma unroll
    for (int u = 0; u < IQ * 32 * SLOTS / 64; ++u) {
      const int x = u * 64 + lane, q = x / SLOTS, s = x % SLOTS;
      const uint4 v = *reinterpret_cast<const uint4*>(lds + q * (IP * 64) + (s ^ (q & (SLOTS - 1))) * 16);
      if (q < nq && s * 8 < np) *reinterpret_cast<uint4*>(out + q * ldz + s * 8) = v;
    }
  }
};

// The entries' places in a piece: p less the weights of all the row's entries that name it, by the first
// of them, from the logit that the forward kept.
__device__ __forceinline__ uint16_t entry_grad(const VocabArgs& a, const RowCoef& rc, float z, float q) {
  const float p = __builtin_amdgcn_exp2f(__fmaf_rn(z, 1.44269504088896341f / a.T, -rc.lse2));
  float d = __fmaf_rn(rc.cp, p, -__fmul_rn(rc.ct, q));
  if (a.cap > 0.f) {
    const float x = z / a.cap;
    d = __fmul_rn(d, __fmaf_rn(-x, x, 1.f));
  }
  return f32_to_bf16(d);
}
__global__ __launch_bounds__(256) void vocab_label_kernel(VocabArgs a, const int* at, const int* n, const RowCoef* rows,
                                                          int64_t v0, int64_t nv, uint16_t* dz, int64_t ldz) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= *n) return;
  const int64_t row = at[i], id = a.ids[row] - v0;
  if (id >= 0 && id < nv) dz[(int64_t)i * ldz + id] = entry_grad(a, rows[i], a.zt[row], 1.f);
}
__global__ __launch_bounds__(256) void vocab_entry_kernel(VocabArgs a, const int* at, const int* n, const RowCoef* rows,
                                                          const float2* weight, int64_t v0, int64_t nv, uint16_t* dz,
                                                          int64_t ldz) {
  __shared__ int64_t ids[4][kTopMax];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int i = blockIdx.x * 4 + w;
  if (i >= *n) return;
  const int64_t row = at[i], first = row * a.k;
  for (int j = lane; j < a.k; j += 64) ids[w][j] = a.ids[first + j];
  wave_lds_sync();
  const RowTarget r{weight[row].x, weight[row].y, true, false};
  const RowCoef rc = rows[i];
  for (int j = lane; j < a.k; j += 64) {
    const int64_t id = ids[w][j];
    if (id < v0 || id >= v0 + nv) continue;
    float q = 0.f;
    bool lead = true;
    for (int e = 0; e < a.k; ++e) {
      if (ids[w][e] != id) continue;
      lead &= e >= j;
      q = __fadd_rn(q, r.weight(teacher_logit(a, first + e)));
    }
    if (lead) dz[(int64_t)i * ldz + (id - v0)] = entry_grad(a, rc, a.zt[first + j], q);
  }
}

// Sums of a part of the reduction: stored, or added to those of the pieces before.
template <class T, int ROWS_DIM>
struct PartEpi {
  static constexpr int ROWS = ROWS_DIM;
  float* out;          // [S][rows][ld]
  int64_t rows, ld;
  int add;
  template <class Acc>
  __device__ __forceinline__ void operator()(const TilePlace& t, Acc& acc, char* const (&)[4], int lane, int, int wp, int wq) const {
    const int np = t.np - wp * T::IP * 32, nq = t.nq - wq * T::IQ * 32, h4 = (lane >> 5) * 4, l32 = lane & 31;
    float* o = out + ((int64_t)t.split * rows + t.p0 + wp * T::IP * 32) * ld + t.q0 + wq * T::IQ * 32;
#pragma unroll
    for (int i = 0; i < T::IP; ++i)
#pragma unroll
      for (int j = 0; j < T::IQ; ++j) {
        const bool in = j * 32 + l32 < nq;
        float v[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int p = i * 32 + 8 * (r >> 2) + h4 + (r & 3);
          v[r] = add && in && p < np ? o[p * ld + j * 32 + l32] : 0.f;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int p = i * 32 + 8 * (r >> 2) + h4 + (r & 3);
          if (in && p < np) o[p * ld + j * 32 + l32] = __fadd_rn(v[r], acc[i][j][r]);
        }
      }
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
  __device__ __forceinline__ void operator()(const TilePlace& t, Acc& acc, char* const (&)[4], int lane, int, int wp, int wq) const {
    const int np = t.np - wp * T::IP * 32, nq = (int)min((int64_t)t.nq, g.K - t.q0) - wq * T::IQ * 32;
    const int h4 = (lane >> 5) * 4, l32 = lane & 31;
    const int64_t org = (int64_t)(t.p0 + wp * T::IP * 32) * g.K + t.q0 + wq * T::IQ * 32;
    const float scale = *g.scale;
    OptK o = g.opt;
    if constexpr (UPDATE) opt_prepare(o);
    // bf16: lanes 2l and 2l + 1 trade a value so that each stores two columns of a row
    const bool pair = !UPDATE && g.gbf && !g.accumulate && g.K % 2 == 0 && ((uintptr_t)g.dw & 3u) == 0;
#pragma unroll
    for (int i = 0; i < T::IP; ++i)
#pragma unroll
      for (int j = 0; j < T::IQ; ++j) {
        const int q = j * 32 + l32;
        auto at = [&](int r) { return i * 32 + 8 * (r >> 2) + h4 + (r & 3); };
        if constexpr (UPDATE) {
          if (q >= nq) continue;
          OptState1 st[16];
          float e[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            if (at(r) >= np) continue;
            st[r] = opt_load1(o, g.W, org + at(r) * g.K + q);
            e[r] = g.gW ? g.gW[org + at(r) * g.K + q] : 0.f;
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            if (at(r) >= np) continue;
            const float d = __fmul_rn(acc[i][j][r], scale);
            opt_apply1(o, g.W, st[r], g.gW ? __fadd_rn(e[r], d) : d, org + at(r) * g.K + q);
          }
        } else if (pair) {
          const bool odd = lane & 1;
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            const float x = __fmul_rn(acc[i][j][r], scale), y = __fmul_rn(acc[i][j][r + 1], scale);
            const float mine = odd ? y : x, give = odd ? x : y;
            const float got = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(give), 0xb1, 0xf, 0xf, true));   // lane ^ 1
            const int p = at(r) + (odd ? 1 : 0);
            if (q < nq && p < np)
              *reinterpret_cast<uint32_t*>((uint16_t*)g.dw + org + p * g.K + (q & ~1)) = odd ? pack2(got, mine) : pack2(mine, got);
          }
        } else {
          if (q >= nq) continue;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (at(r) < np) g.store(org + at(r) * g.K + q, __fmul_rn(acc[i][j][r], scale));
        }
      }
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
    for (int s = 1; s < S; ++s) v = __fadd_rn(v, p[s * rows * ld]);
    v = __fmul_rn(v, scale);
    if (g.dw) g.store(i, v);
    else update1(o, g.W, g.gW ? __fadd_rn(g.gW[i], v) : v, i);
  }
}

// dX from its parts [S][M][ld]: their sum in order, scaled, at its row; zeros where a row has none.
template <int V>
__global__ __launch_bounds__(256) void vocab_dx_kernel(const float* part, int S, int64_t M, int64_t ld, const int* place,
                                                       const float* scale, int64_t K, void* dx, int64_t ldx, int gbf) {
  const float f = *scale;
  const int64_t each = K / V;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * each; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / each, c = (i - row * each) * V;
    const int r = place[row];
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
    if (r >= 0) {
      for (int s = 0; s < S; ++s) {
        const float* p = part + ((int64_t)s * M + r) * ld + c;
        if constexpr (V == 4) {
          const float4 x = ld4(p);
          v[0] = __fadd_rn(v[0], x.x), v[1] = __fadd_rn(v[1], x.y), v[2] = __fadd_rn(v[2], x.z), v[3] = __fadd_rn(v[3], x.w);
        } else {
          v[0] = __fadd_rn(v[0], *p);
        }
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
Choice choose(int64_t P, int64_t Q, int64_t R, bool split) {
  Choice best{MID, 1};
  double least = 1e300;
  for (const Shape s : {BIG, MID}) {
    const int64_t b = s == BIG ? 256 : 128, tiles = per(P, b) * per(Q, b);
    for (int S = 1; S <= (split ? 64 : 1); S += S < 4 ? 1 : S / 2) {
      if (S > 1 && R / S < 128) break;
      const int64_t wg = tiles * S;
      const double stages = (double)up(per(per(R, 32), S), 4);
      const double one = s == BIG ? stages * 0.85 + 8 : stages * (wg > 256 ? 0.58 : 0.36) + 4;
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

struct Bf16Plan {
  int64_t Kp, piece, ldz;           // widened rows; vocabulary entries of a piece
  Choice logits, dx, dw;
  int BP, BQ, WP;                   // the logits' tiles
  int64_t vtiles, rtiles;
  size_t x, w, off, list, part, sums, done;
  size_t flag, weight, at, place, n, scale, rows, dz, pdx, pdw, total;
};

Bf16Plan bf16_plan(const VocabArgs& a, bool bwd) {
  Bf16Plan p{};
  p.Kp = up(a.K, 8);
  size_t here = 0;
  auto take = [&](int64_t bytes) {
    const size_t at = here;
    here += (size_t)up(bytes, 256);
    return at;
  };
  p.logits = a.M <= kFew ? Choice{FEW, 1} : choose(a.V, a.M, a.K, false);
  p.BP = p.logits.shape == BIG ? 256 : 128;
  p.BQ = p.logits.shape == BIG ? 256 : p.logits.shape == MID ? 128 : 32;
  p.WP = p.logits.shape == FEW ? 4 : 2;
  p.vtiles = per(a.V, p.BP), p.rtiles = per(a.M, p.BQ);
  // W's rows are copied where they are not whole 16-byte pieces: 64 MB at a time
  const int64_t copied = std::max<int64_t>(256, (1 << 25) / p.Kp / 256 * 256);
  if (!bwd) {
    p.x = take(a.M * p.Kp * 2);
    p.w = take(std::min(copied, a.V) * p.Kp * 2);
    p.off = take(p.rtiles * (p.vtiles + 1) * 4);
    p.list = take(p.rtiles * p.BQ * a.k * 4);
    p.part = take(p.vtiles * p.WP * a.M * 8);
    p.sums = take(per(a.M, kJoinRows) * 16);
    p.done = take(4);
    p.total = here;
    p.piece = copied;
    return p;
  }
  // a piece's gradient takes up to 512 MB; pieces of one size
  const int64_t most = std::max<int64_t>(256, (1LL << 28) / a.M / 256 * 256);
  p.piece = std::min(up(per(a.V, per(a.V, most)), 256), up(a.V, 8));
  p.ldz = p.piece;
  p.dx = a.M <= kFew ? Choice{FEW, few_parts(a.K, p.piece)} : choose(a.M, a.K, p.piece, true);
  p.dw = choose(p.piece, a.K, a.M, true);
  p.x = take(a.M * p.Kp * 2);
  p.w = take(std::min(copied, p.piece) * p.Kp * 2);
  p.flag = take(a.M);
  p.weight = take(a.M * 8);
  p.at = take(a.M * 4);
  p.place = take(a.M * 4);
  p.n = take(4);
  p.scale = take(4);
  p.rows = take(a.M * (int64_t)sizeof(RowCoef));
  p.dz = take(a.M * p.ldz * 2);
  p.pdx = take((int64_t)p.dx.S * a.M * p.Kp * 4);
  p.pdw = take(p.dw.S > 1 ? (int64_t)p.dw.S * p.piece * p.Kp * 4 : 0);
  p.total = here;
  return p;
}

template <class T, bool A, bool B, class Epi>
hipError_t product(const uint16_t* a, int64_t lda, const uint16_t* b, int64_t ldb, int64_t P, int64_t Q, int64_t R,
                   const int* rows, int S, const Epi& e, hipStream_t s) {
  const TileProblem pr{a, b, lda, ldb, (int)P, (int)Q, (int)R, rows, (int)per(P, T::BP), (int)per(Q, T::BQ), S};
  hipLaunchKernelGGL((tile_kernel<T, A, B, Epi>), dim3((unsigned)(pr.gp * pr.gq * S)), dim3(T::NT), 0, s, pr, e);
  return hipGetLastError();
}

#define TRY(x)                                    \
  do {                                            \
    const hipError_t e_ = (x);                    \
    if (e_ != hipSuccess) return e_;              \
  } while (0)

int grid_of(int64_t n) { return (int)std::min<int64_t>(8192, std::max<int64_t>(1, per(n, 256))); }

hipError_t gather(const uint16_t* src, int64_t lds, const int* at, const int* n, int64_t rows, int64_t K, uint16_t* dst,
                  int64_t ldd, hipStream_t s) {
  hipLaunchKernelGGL(vocab_gather_kernel, dim3(grid_of(rows * ldd / 8)), dim3(256), 0, s, src, lds, at, n, rows, K, dst, ldd,
                     odd_rows(src, lds, K) ? 0 : 1);
  return hipGetLastError();
}

template <class T>
hipError_t stats(const VocabArgs& a, const Bf16Plan& p, char* ws, const uint16_t* x, int64_t ldx, const uint16_t* w, int64_t v0,
                 int64_t n, hipStream_t s) {
  const Entries en{(int*)(ws + p.off), (uint32_t*)(ws + p.list), (int)p.vtiles};
  const StatEpi<T> e{(float2*)(ws + p.part), a.zt, en, (int)(v0 / T::BP), a.M, a.k, a.cap, 1.44269504088896341f / a.T};
  return product<T, true, true>(w, p.Kp, x, ldx, n, a.M, a.K, nullptr, 1, e, s);
}

template <class T>
hipError_t sort_entries(const VocabArgs& a, const Bf16Plan& p, char* ws, hipStream_t s) {
  const Entries en{(int*)(ws + p.off), (uint32_t*)(ws + p.list), (int)p.vtiles};
  hipLaunchKernelGGL((vocab_sort_kernel<T::BP, T::BQ>), dim3((unsigned)p.rtiles), dim3(1024), (size_t)p.vtiles * 4, s, a, en,
                     (int*)(ws + p.done));
  return hipGetLastError();
}

template <class T>
hipError_t grads(const VocabArgs& a, const Bf16Plan& p, char* ws, const uint16_t* w, int64_t n, hipStream_t s) {
  const GradEpi<T> e{(RowCoef*)(ws + p.rows), (uint16_t*)(ws + p.dz), p.ldz, a.cap, 1.44269504088896341f / a.T};
  return product<T, true, true>(w, p.Kp, (uint16_t*)(ws + p.x), p.Kp, n, a.M, a.K, (int*)(ws + p.n), 1, e, s);
}

template <class T>
hipError_t data_grad(const VocabArgs& a, const Bf16Plan& p, char* ws, const uint16_t* w, int64_t n, bool first, hipStream_t s) {
  const PartEpi<T, ROWS_P> e{(float*)(ws + p.pdx), a.M, p.Kp, first ? 0 : 1};
  return product<T, true, false>((uint16_t*)(ws + p.dz), p.ldz, w, p.Kp, a.M, p.Kp, n, (int*)(ws + p.n), p.dx.S, e, s);
}

template <class T>
hipError_t head_grad(const VocabArgs& a, const Bf16Plan& p, char* ws, const HeadGrad& g, int64_t n, hipStream_t s) {
  const uint16_t *dz = (uint16_t*)(ws + p.dz), *x = (uint16_t*)(ws + p.x);
  const int* rows = (int*)(ws + p.n);
  if (p.dw.S > 1) {
    const PartEpi<T, ROWS_R> e{(float*)(ws + p.pdw), n, p.Kp, 0};
    TRY((product<T, false, false>(dz, p.ldz, x, p.Kp, n, p.Kp, a.M, rows, p.dw.S, e, s)));
    hipLaunchKernelGGL(vocab_head_kernel, dim3(grid_of(n * a.K)), dim3(256), 0, s, g, (const float*)(ws + p.pdw), p.dw.S, n, p.Kp);
    return hipGetLastError();
  }
  if (g.dw) return product<T, false, false>(dz, p.ldz, x, p.Kp, n, p.Kp, a.M, rows, 1, HeadEpi<T, false>{g}, s);
  return product<T, false, false>(dz, p.ldz, x, p.Kp, n, p.Kp, a.M, rows, 1, HeadEpi<T, true>{g}, s);
}

}  // namespace

size_t vocab_bf16_ws_bytes(const VocabArgs& a, bool bwd) { return bf16_plan(a, bwd).total; }

hipError_t vocab_bf16_fwd(const VocabArgs& a, void* wsp, hipStream_t s) {
  const Bf16Plan p = bf16_plan(a, false);
  char* ws = (char*)wsp;
  const uint16_t* x = (const uint16_t*)a.x;
  int64_t ldx = a.ldx;
  if (odd_rows(x, ldx, a.K)) {
    TRY(gather(x, ldx, nullptr, nullptr, a.M, a.K, (uint16_t*)(ws + p.x), p.Kp, s));
    x = (uint16_t*)(ws + p.x), ldx = p.Kp;
  }
  switch (p.logits.shape) {
    case BIG: TRY(sort_entries<Big>(a, p, ws, s)); break;
    case MID: TRY(sort_entries<Mid>(a, p, ws, s)); break;
    default: TRY(sort_entries<FewQ>(a, p, ws, s)); break;
  }
  const bool copy = odd_rows(a.W.w_bf16, a.K, a.K);
  const int64_t piece = copy ? p.piece : a.V;
  for (int64_t v0 = 0; v0 < a.V; v0 += piece) {
    const int64_t n = std::min(piece, a.V - v0);
    const uint16_t* w = a.W.w_bf16 + v0 * a.K;
    if (copy) {
      TRY(gather(w, a.K, nullptr, nullptr, n, a.K, (uint16_t*)(ws + p.w), p.Kp, s));
      w = (uint16_t*)(ws + p.w);
    }
    switch (p.logits.shape) {
      case BIG: TRY(stats<Big>(a, p, ws, x, ldx, w, v0, n, s)); break;
      case MID: TRY(stats<Mid>(a, p, ws, x, ldx, w, v0, n, s)); break;
      default: TRY(stats<FewQ>(a, p, ws, x, ldx, w, v0, n, s)); break;
    }
  }
  hipLaunchKernelGGL(vocab_join_kernel, dim3((unsigned)per(a.M, kJoinRows)), dim3(256), 0, s, a, (const float2*)(ws + p.part),
                     (int)p.vtiles * p.WP, (double2*)(ws + p.sums), (int*)(ws + p.done));
  return hipGetLastError();
}

hipError_t vocab_bf16_bwd(const VocabArgs& a, void* wsp, hipStream_t s) {
  const Bf16Plan p = bf16_plan(a, true);
  char* ws = (char*)wsp;
  int *at = (int*)(ws + p.at), *place = (int*)(ws + p.place), *n = (int*)(ws + p.n);
  float* scale = (float*)(ws + p.scale);
  RowCoef* rows = (RowCoef*)(ws + p.rows);
  uint16_t* dz = (uint16_t*)(ws + p.dz);
  const float2* weight = (float2*)(ws + p.weight);
  if (a.teacher) {
    hipLaunchKernelGGL(vocab_flag_kernel, dim3((unsigned)per(a.M, 4)), dim3(256), 0, s, a, (uint8_t*)(ws + p.flag),
                       (float2*)(ws + p.weight));
    TRY(hipGetLastError());
  }
  hipLaunchKernelGGL(vocab_index_kernel, dim3(1), dim3(1024), 0, s, a, (const uint8_t*)(ws + p.flag), at, place, n, scale, rows);
  TRY(hipGetLastError());
  TRY(gather((const uint16_t*)a.x, a.ldx, at, n, a.M, a.K, (uint16_t*)(ws + p.x), p.Kp, s));
  const bool copy = odd_rows(a.W.w_bf16, a.K, a.K);
  const int64_t copied = std::max<int64_t>(256, (1 << 25) / p.Kp / 256 * 256);
  const int64_t piece = copy ? std::min(copied, p.piece) : p.piece;
  for (int64_t v0 = 0; v0 < a.V; v0 += piece) {
    const int64_t nv = std::min(piece, a.V - v0);
    const uint16_t* w = a.W.w_bf16 + v0 * a.K;
    if (copy) {
      TRY(gather(w, a.K, nullptr, nullptr, nv, a.K, (uint16_t*)(ws + p.w), p.Kp, s));
      w = (uint16_t*)(ws + p.w);
    }
    switch (p.logits.shape) {
      case BIG: TRY(grads<Big>(a, p, ws, w, nv, s)); break;
      case MID: TRY(grads<Mid>(a, p, ws, w, nv, s)); break;
      default: TRY(grads<FewQ>(a, p, ws, w, nv, s)); break;
    }
    if (a.teacher)
      hipLaunchKernelGGL(vocab_entry_kernel, dim3((unsigned)per(a.M, 4)), dim3(256), 0, s, a, at, n, rows, weight, v0, nv, dz, p.ldz);
    else
      hipLaunchKernelGGL(vocab_label_kernel, dim3((unsigned)per(a.M, 256)), dim3(256), 0, s, a, at, n, rows, v0, nv, dz, p.ldz);
    TRY(hipGetLastError());
    if (a.dx) {
      switch (p.dx.shape) {
        case BIG: TRY(data_grad<Big>(a, p, ws, w, nv, v0 == 0, s)); break;
        case MID: TRY(data_grad<Mid>(a, p, ws, w, nv, v0 == 0, s)); break;
        default: TRY(data_grad<FewP>(a, p, ws, w, nv, v0 == 0, s)); break;
      }
    }
    if (!a.fused && !a.dw) continue;
    HeadGrad g{};
    g.scale = scale;
    g.K = a.K;
    g.gbf = a.gbf;
    g.accumulate = a.accumulate;
    if (a.fused) {
      g.W = a.W;
      const int64_t o = v0 * a.K;
      g.W.w += o, g.W.m = a.W.m ? a.W.m + o : nullptr, g.W.v = a.W.v ? a.W.v + o : nullptr, g.W.w_bf16 += o;
      g.gW = a.gW ? a.gW + o : nullptr;
      g.opt = a.opt;
    } else {
      g.dw = a.gbf ? (void*)((uint16_t*)a.dw + v0 * a.K) : (void*)((float*)a.dw + v0 * a.K);
    }
    TRY(p.dw.shape == BIG ? head_grad<Big>(a, p, ws, g, nv, s) : head_grad<Mid>(a, p, ws, g, nv, s));
  }
  if (!a.dx) return hipSuccess;
  const bool vec = a.K % 4 == 0 && a.ldx % 4 == 0 && ((uintptr_t)a.dx) % (a.gbf ? 8 : 16) == 0;
  const float* part = (const float*)(ws + p.pdx);
  if (vec)
    hipLaunchKernelGGL(vocab_dx_kernel<4>, dim3(grid_of(a.M * a.K / 4)), dim3(256), 0, s, part, p.dx.S, a.M, p.Kp, place, scale,
                       a.K, a.dx, a.ldx, a.gbf ? 1 : 0);
  else
    hipLaunchKernelGGL(vocab_dx_kernel<1>, dim3(grid_of(a.M * a.K)), dim3(256), 0, s, part, p.dx.S, a.M, p.Kp, place, scale, a.K,
                       a.dx, a.ldx, a.gbf ? 1 : 0);
  return hipGetLastError();
}

}  // namespace opfuse
