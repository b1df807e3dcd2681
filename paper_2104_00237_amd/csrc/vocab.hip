// Vocabulary losses of few fp32 rows: softmax cross-entropy of an output head and distillation from a
// teacher's top logits, forward and backward, in pieces of the vocabulary: the logits of a piece are the
// only ones that ever exist.
//
// Per piece: its logits (the library's linear forward), then the rows' statistics (forward), or
// their gradient in place and from it dX and dW, or the update of the piece's W (backward): dX reads a
// piece's W before the update writes it, and no other piece reads it.  dX is summed over the pieces in
// order, so results are deterministic.

#include <algorithm>
#include <cstring>

#include "vocab.h"

namespace opfuse {

namespace {

// ------------------------------------------------------------ rows of a piece
// Rows are worked on in chunks of kChunk logits, 16 a thread in registers: few rows alone would not fill
// the chip (two rows of 22049: 40 us of 53 with a workgroup a row).
constexpr int kChunk = 4096;

struct Chunk {
  float v[16];
  // logits [from, n) of a row; what lies past n is `fill`
  __device__ __forceinline__ void load(const float* s, int from, int n, float fill) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = from + (u * 256 + (int)threadIdx.x) * 4;
      const float4 x = i < n ? ld4(s + i) : make_float4(fill, fill, fill, fill);   // (rows are padded to 4)
      v[4 * u] = x.x, v[4 * u + 1] = i + 1 < n ? x.y : fill, v[4 * u + 2] = i + 2 < n ? x.z : fill,
          v[4 * u + 3] = i + 3 < n ? x.w : fill;
    }
  }
};

// Statistics (a maximum of the logits, and the sum of exp((z - maximum) / T)) of a chunk of one row of
// the piece [v0, v0 + n), and the logits of the row's entries in it.
__global__ __launch_bounds__(256) void vocab_stats_kernel(VocabArgs a, const float* __restrict__ z, int64_t ldz, int64_t v0, int n,
                                                          float2* part, int* done) {
  __shared__ float red[2][4];
  const int64_t row = blockIdx.x;
  const int t = threadIdx.x, from = blockIdx.y * kChunk;
  const float* s = z + row * ldz;
  if (v0 == 0 && from == 0 && row == 0 && t == 0) *done = 0;
  Chunk c;
  c.load(s, from, n, -INFINITY);
  float m = -INFINITY;
#pragma unroll
  for (int u = 0; u < 16; ++u) {
    // (what lies past the end stays -infinity: a cap would make it a logit)
    if (c.v[u] != -INFINITY || from + (u / 4 * 256 + t) * 4 + u % 4 < n) c.v[u] = vocab_cap_exact(c.v[u], a.cap);
    m = fmaxf(m, c.v[u]);
  }
  m = wave_max(m);
  if ((t & 63) == 0) red[0][t >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const float shift = stat_shift(m);
  float sum = 0.f;
#pragma unroll
  for (int u = 0; u < 16; ++u) sum = __fadd_rn(sum, expf(__fdiv_rn(c.v[u] - shift, a.T)));
  sum = wave_sum(sum);
  if ((t & 63) == 0) red[1][t >> 6] = sum;
  __syncthreads();
  if (t == 0) part[(int64_t)blockIdx.y * a.M + row] = make_float2(m, (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]));
  const int end = min(n, from + kChunk);
  for (int j = t; j < a.k; j += 256) {
    const int64_t i = row * a.k + j, id = a.ids[i];
    if (id >= v0 + from && id < v0 + end) a.zt[i] = vocab_cap_exact(s[id - v0], a.cap);
    else if (v0 == 0 && from == 0 && (id < 0 || id >= a.V)) a.zt[i] = 0.f;
  }
}

// ------------------------------------------------------------------- backward
// A workgroup a row: what scales its gradient (g T for its targets; g T (1 + 2 c lse) for its
// probabilities; without given gradients g is 1 here, and 1 / (rows that count) where it is used), and its
// X for the products: zeros for a row that gets no gradient, so that nothing it holds (a NaN times
// its zero gradient, too) reaches dW.
__global__ __launch_bounds__(256) void vocab_prepare_kernel(VocabArgs a, float2* coef, float* counts, float* x) {
  __shared__ int on;
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  if (t < 64) {
    const RowTarget r = row_target(a, row, t);
    if (t == 0) {
      const bool live = r.counts && !r.bad;
      const float g = live ? (a.dloss ? a.dloss[row] : 1.f) * a.T : 0.f;
      coef[row] = make_float2(g, live ? __fmul_rn(g, __fmaf_rn(2.f * a.z_loss, a.lse[row], 1.f)) : 0.f);
      counts[row] = r.counts ? 1.f : 0.f;
      counts[a.M + row] = live ? 1.f : 0.f;
      on = live;
    }
  }
  __syncthreads();
  const float* src = (const float*)a.x + row * a.ldx;
  for (int64_t c = t; c < a.K; c += 256) x[row * a.K + c] = on ? src[c] : 0.f;
}

// How many rows count (whole numbers: exact in any order), in one workgroup: with more than kCountHere of them the
// gradient's workgroups, one for each row, no longer add them up themselves, which is quadratic in the rows.
// Added up there / here, whole backward in us, width 64: 1500 rows over 1000 45.1 / 45.8, 2048 53.1 / 52.8, 4096 over 500
// 57.5 / 53.9, 16384 over 100 131 / 74, 262144 over 4 11700 / 527.
constexpr int64_t kCountHere = 2048;
__global__ __launch_bounds__(1024) void vocab_count_kernel(int64_t M, const float* counts, float* total) {
  __shared__ int waves[16];
  const int t = threadIdx.x;
  int n = 0;
  constexpr int U = 8;
  for (int64_t i = t; i < M; i += 1024 * U) {
#pragma unroll
    for (int u = 0; u < U; ++u) n += i + u * 1024 < M && counts[i + u * 1024] != 0.f;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d);
  if ((t & 63) == 0) waves[t >> 6] = n;
  __syncthreads();
  if (t) return;
  for (int i = 1; i < 16; ++i) n += waves[i];
  *total = (float)n;
}

// dX of rows that get no gradient: zeros, where the products' zeros times an infinite or NaN W are NaN.
__global__ __launch_bounds__(64) void vocab_clear_kernel(VocabArgs a, const float* live) {
  const int64_t row = blockIdx.x;
  if (live[row] != 0.f) return;
  for (int64_t i = threadIdx.x; i < a.K; i += 64) ((float*)a.dx)[row * a.ldx + i] = 0.f;
}

// The gradient of a chunk of a row's logits, in place of them.  An entry's place is written by its first
// entry with the weights of all that name it; a label's logit is read before the row is overwritten.
__global__ __launch_bounds__(256) void vocab_grad_kernel(VocabArgs a, float* __restrict__ z, int64_t ldz, int64_t v0, int n,
                                                         const float2* coef, const float* counts, const float* total) {
  constexpr int EACH = kTopMax / 256;
  __shared__ float red[4];
  __shared__ __attribute__((aligned(16))) int places[kTopMax];   // of the entries in this chunk, or -1
  const int64_t row = blockIdx.x;
  const int t = threadIdx.x, from = blockIdx.y * kChunk, end = min(n, from + kChunk);
  float* s = z + row * ldz;
  const float2 c = coef[row];
  if (c.x == 0.f && c.y == 0.f) {
    for (int v = from + t; v < end; v += 256) s[v] = 0.f;
    return;
  }
  float g = 1.f;
  if (a.dloss == nullptr && total) {
    g = 1.f / fmaxf(*total, 1.f);
  } else if (a.dloss == nullptr) {
    float count = 0.f;
    for (int64_t i = t; i < a.M; i += 256) count += counts[i];
    count = wave_sum(count);
    if ((t & 63) == 0) red[t >> 6] = count;
    __syncthreads();
    g = 1.f / fmaxf(red[0] + red[1] + red[2] + red[3], 1.f);
  }
  const float lse = a.lse[row], ct = __fmul_rn(c.x, g), cp = __fmul_rn(c.y, g);
  auto grad = [&](float logit) {
    float slope;
    const float z = vocab_cap_exact(logit, a.cap, &slope);
    return place_grad(a.T, z, slope, lse, cp, 0.f, 0.f);
  };
  auto entry = [&](float z, float q) { return entry_grad(a.T, a.cap, z, lse, cp, ct, q); };
  const int64_t at = row * a.k;
  int where[EACH];
  float d[EACH];
  if (a.teacher == nullptr) {
    where[0] = -1;
    if (t == 0) {
      const int64_t id = a.ids[row] - v0;
      if (id >= from && id < end) where[0] = (int)id, d[0] = entry(entry_logit(vocab_cap_exact(s[id], a.cap), a.zt[row]), 1.f);
    }
#pragma unroll
    for (int u = 1; u < EACH; ++u) where[u] = -1;
  } else {
    const RowTarget r = row_target(a, row, t & 63);
    const int k4 = (a.k + 3) & ~3;
    for (int j = t; j < k4; j += 256) {
      const int64_t id = j < a.k ? a.ids[at + j] - v0 : -1;
      places[j] = id >= from && id < end ? (int)id : -1;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int j = t + u * 256;
      where[u] = j < a.k ? places[j] : -1;
      if (where[u] < 0) continue;
      // (entries that name one place twice are rare: four compares an LDS read, weights only where one matches)
      float q = r.weight(teacher_logit(a, at + j));
      bool first = true;
      for (int i = 0; i < k4; i += 4) {
        const int4 p = *reinterpret_cast<const int4*>(&places[i]);
        const int x[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (x[e] != where[u] || i + e == j) continue;
          first &= i + e > j;
          q = __fadd_rn(q, r.weight(teacher_logit(a, at + i + e)));
        }
      }
      if (first) d[u] = entry(a.zt[at + j], q);
      else where[u] = -1;
    }
  }
  Chunk k;
  k.load(s, from, n, 0.f);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int i = from + (u * 256 + t) * 4;
    if (i < n) st4(s + i, make_float4(grad(k.v[4 * u]), grad(k.v[4 * u + 1]), grad(k.v[4 * u + 2]), grad(k.v[4 * u + 3])));
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < EACH; ++u)
    if (where[u] >= 0) s[where[u]] = d[u];
}

// ---------------------------------------------------------------------- pieces
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Vocabulary entries of a piece: fp32 logits of up to 256 MB (the last-level cache), at least 256
// entries (64 where there are very many rows), and W's piece below the 2 GiB that the products address.
int64_t piece_of(const VocabArgs& a) {
  const int64_t most = std::max<int64_t>({1, std::min<int64_t>((1LL << 30) / (a.K * 4), (1LL << 26) / a.M)});
  const int64_t n = (a.V + most - 1) / most;
  return std::min(a.V, up((a.V + n - 1) / n, 64));
}

struct Plan {
  int64_t piece, ldz, chunks;   // chunks: of a piece
  size_t z, part, sums, done, counts, rows, coef, x, gemm, total;   // offsets; total: bytes
};

Plan plan_of(const VocabArgs& a, bool bwd) {
  Plan p{};
  p.piece = piece_of(a);
  p.ldz = up(p.piece, 4);
  p.chunks = (p.piece + kChunk - 1) / kChunk;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  p.z = take((size_t)a.M * p.ldz * 4);
  size_t g = 0;
  for (int64_t n : {p.piece, a.V % p.piece ? a.V % p.piece : p.piece}) {
    g = std::max(g, gemm_workspace_bytes(EPI_FWD, (int)a.M, (int)n, (int)a.K));
    if (bwd)
      g = std::max({g, gemm_workspace_bytes(EPI_DGRAD, (int)a.M, (int)a.K, (int)n),
                    gemm_workspace_bytes(EPI_WGRAD, (int)n, (int)a.K, (int)a.M)});
  }
  p.gemm = take(g);
  if (bwd) {
    p.counts = take((size_t)a.M * 8);   // rows that count, and those with a gradient
    p.rows = take(4);   // how many count
    p.coef = take((size_t)a.M * 8);
    p.x = take((size_t)a.M * a.K * 4);
  } else {
    p.part = take((size_t)((a.V + p.piece - 1) / p.piece * p.chunks) * a.M * 8);
    p.sums = take(vocab_join_bytes(a));
    p.done = take(4);
  }
  p.total = at;
  return p;
}

EpiArgs no_epi() {
  EpiArgs e;
  memset(&e, 0, sizeof(e));
  return e;
}

of_param piece_param(const of_param& W, int64_t off, int64_t n) {
  of_param p = W;
  if (p.w) p.w += off;
  if (p.m) p.m += off;
  if (p.v) p.v += off;
  if (p.w_bf16) p.w_bf16 += off;
  p.numel = n;
  return p;
}

struct Pieces {
  const VocabArgs& a;
  Plan p;
  char* ws;
  hipStream_t s;
  float* z() const { return (float*)(ws + p.z); }
  hipError_t product(int kind, const GemmProblem& pr, const EpiArgs& ea) const {
    return gemm_launch(kind, pr, ea, ws + p.gemm, s);
  }
  dim3 rows(int64_t n) const { return dim3((unsigned)a.M, (unsigned)((n + kChunk - 1) / kChunk)); }
  const float* w(int64_t v0) const { return a.W.w + v0 * a.K; }
  hipError_t logits(const float* x, int64_t ldx, int64_t v0, int64_t n) const {
    const GemmProblem pr{x, ldx, 1, w(v0), a.K, 1, (int)a.M, (int)n, (int)a.K};
    EpiArgs ea = no_epi();
    ea.out = z(), ea.ldo = p.ldz, ea.ldz = p.ldz, ea.ldr = p.ldz;
    return product(EPI_FWD, pr, ea);
  }
};

#define TRY(x)                                    \
  do {                                            \
    const hipError_t e_ = (x);                    \
    if (e_ != hipSuccess) return e_;              \
  } while (0)

}  // namespace

size_t vocab_ws_bytes(const VocabArgs& a, bool bwd) {
  return vocab_tiles_ok(a, bwd) ? vocab_tiles_ws_bytes(a, bwd) : plan_of(a, bwd).total;
}

hipError_t vocab_fwd_launch(const VocabArgs& a, void* ws, hipStream_t s) {
  if (vocab_tiles_ok(a, false)) return vocab_tiles_fwd(a, ws, s);
  const Pieces g{a, plan_of(a, false), (char*)ws, s};
  float2* part = (float2*)(g.ws + g.p.part);
  int* done = (int*)(g.ws + g.p.done);
  int64_t parts = 0;
  for (int64_t v0 = 0; v0 < a.V; v0 += g.p.piece) {
    const int64_t n = std::min(g.p.piece, a.V - v0);
    TRY(g.logits((const float*)a.x, a.ldx, v0, n));
    const dim3 grid = g.rows(n);
    hipLaunchKernelGGL(vocab_stats_kernel, grid, dim3(256), 0, s, a, g.z(), g.p.ldz, v0, (int)n, part + parts * a.M, done);
    TRY(hipGetLastError());
    parts += grid.y;
  }
  return vocab_join_launch(a, part, (int)parts, g.ws + g.p.sums, done, s);
}

hipError_t vocab_bwd_launch(const VocabArgs& a, void* ws, hipStream_t s) {
  if (vocab_tiles_ok(a, true)) return vocab_tiles_bwd(a, ws, s);
  const Pieces g{a, plan_of(a, true), (char*)ws, s};
  const Plan& p = g.p;
  float2* coef = (float2*)(g.ws + p.coef);
  float *counts = (float*)(g.ws + p.counts), *x = (float*)(g.ws + p.x);
  hipLaunchKernelGGL(vocab_prepare_kernel, dim3((unsigned)a.M), dim3(256), 0, s, a, coef, counts, x);
  TRY(hipGetLastError());
  float* total = a.dloss == nullptr && a.M > kCountHere ? (float*)(g.ws + p.rows) : nullptr;
  if (total) {
    hipLaunchKernelGGL(vocab_count_kernel, dim3(1), dim3(1024), 0, s, a.M, counts, total);
    TRY(hipGetLastError());
  }
  float* dx = (float*)a.dx;
  for (int64_t v0 = 0; v0 < a.V; v0 += p.piece) {
    const int64_t n = std::min(p.piece, a.V - v0);
    TRY(g.logits(x, a.K, v0, n));
    hipLaunchKernelGGL(vocab_grad_kernel, g.rows(n), dim3(256), 0, s, a, g.z(), p.ldz, v0, (int)n, coef, counts, total);
    TRY(hipGetLastError());
    if (a.dx) {
      const GemmProblem pr{g.z(), p.ldz, 1, g.w(v0), 1, a.K, (int)a.M, (int)a.K, (int)n};
      EpiArgs ea = no_epi();
      ea.out = dx, ea.ldo = ea.ldp = ea.ldr = a.ldx;
      ea.res = v0 ? dx : nullptr;
      TRY(g.product(EPI_DGRAD, pr, ea));
    }
    const GemmProblem pr{g.z(), 1, p.ldz, x, 1, a.K, (int)n, (int)a.K, (int)a.M};
    EpiArgs ea = no_epi();
    ea.ldo = a.K;
    if (a.fused) {
      ea.W = piece_param(a.W, v0 * a.K, n * a.K);
      ea.gW = a.gW ? a.gW + v0 * a.K : nullptr;
      ea.opt = a.opt;
      TRY(g.product(EPI_WGRAD_BF, pr, ea));
    } else if (a.dw) {
      ea.out = (float*)a.dw + v0 * a.K;
      ea.accumulate = a.accumulate;
      TRY(g.product(EPI_WGRAD, pr, ea));
    }
  }
  if (a.dx) hipLaunchKernelGGL(vocab_clear_kernel, dim3((unsigned)a.M), dim3(64), 0, s, a, counts + a.M);
  return hipGetLastError();
}

}  // namespace opfuse
