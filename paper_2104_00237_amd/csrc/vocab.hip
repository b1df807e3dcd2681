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
// A workgroup's statistics of one row, joined in thread order.
__device__ Stat block_stat(Stat v, Stat* sh) {
  const int t = threadIdx.x;
  sh[t] = v;
  __syncthreads();
  for (int d = 128; d > 0; d >>= 1) {
    if (t < d) sh[t] = stat_join(sh[t], sh[t + d]);
    __syncthreads();
  }
  return sh[0];
}

// The piece [v0, v0 + n) of every row: its statistics join the row's, and the logits of the row's
// entries in it are kept.
__global__ __launch_bounds__(256) void vocab_stats_kernel(VocabArgs a, const float* __restrict__ z, int64_t ldz,
                                                          int64_t v0, int n, Stat* stat) {
  __shared__ Stat sh[256];
  const int64_t row = blockIdx.x;
  const float* s = z + row * ldz;
  float m = -INFINITY;
  for (int v = threadIdx.x; v < n; v += 256) m = fmaxf(m, __fdiv_rn(vocab_cap(s[v], a.cap, a.rcap), a.T));
  const float shift = stat_shift(m);
  float sum = 0.f;
  for (int v = threadIdx.x; v < n; v += 256)
    sum = __fadd_rn(sum, expf(__fdiv_rn(vocab_cap(s[v], a.cap, a.rcap), a.T) - shift));
  const Stat mine = block_stat(Stat{m, sum}, sh);
  if (threadIdx.x == 0) stat[row] = v0 == 0 ? mine : stat_join(stat[row], mine);
  for (int j = threadIdx.x; j < a.k; j += 256) {
    const int64_t i = row * a.k + j, id = a.ids[i];
    if (id >= v0 && id < v0 + n) a.zt[i] = vocab_cap(s[id - v0], a.cap, a.rcap);
    else if (v0 == 0 && (id < 0 || id >= a.V)) a.zt[i] = 0.f;
  }
}

// A wavefront per row: lse and loss from the statistics; counts[row] for the mean.
__global__ __launch_bounds__(256) void vocab_loss_kernel(VocabArgs a, const Stat* stat, float* counts) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.M) return;
  const Stat s = stat[row];
  const float lse = __fadd_rn(s.m, logf(s.s));
  bool c;
  const float loss = row_loss(a, row, lse, lane, &c);
  if (lane == 0) {
    a.lse[row] = lse;
    a.loss[row] = loss;
    counts[row] = c ? 1.f : 0.f;
  }
}

// Sum of the rows' losses over the number that count, in float64 and one order.
__global__ __launch_bounds__(1024) void vocab_mean_kernel(const float* loss, const float* counts, int64_t M, float* mean) {
  __shared__ double sh[2][1024];
  const int t = threadIdx.x;
  double l = 0.0, c = 0.0;
  for (int64_t i = t; i < M; i += 1024) l += (double)loss[i], c += (double)counts[i];
  sh[0][t] = l, sh[1][t] = c;
  __syncthreads();
  for (int d = 512; d > 0; d >>= 1) {
    if (t < d) sh[0][t] += sh[0][t + d], sh[1][t] += sh[1][t + d];
    __syncthreads();
  }
  if (t == 0) *mean = (float)(sh[0][0] / fmax(sh[1][0], 1.0));
}

// ------------------------------------------------------------------- backward
// What scales a row's gradient: g T for its targets; g T (1 + 2 c lse) for its probabilities.
// Without given gradients g is 1 / (rows that count), which vocab_scale_kernel finds from counts.
__global__ __launch_bounds__(256) void vocab_coef_kernel(VocabArgs a, float2* coef, float* counts) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.M) return;
  const RowTarget r = row_target(a, row, lane);
  if (lane) return;
  // (a row that does not count has no gradient, whatever its g)
  const float g = r.counts && !r.bad ? (a.dloss ? a.dloss[row] : 1.f) * a.T : 0.f;
  coef[row] = make_float2(g, r.counts && !r.bad ? __fmul_rn(g, __fmaf_rn(2.f * a.z_loss, a.lse[row], 1.f)) : 0.f);
  counts[row] = r.counts ? 1.f : 0.f;
}

__global__ __launch_bounds__(1024) void vocab_scale_kernel(const float* counts, int64_t M, float* scale) {
  __shared__ double sh[1024];
  const int t = threadIdx.x;
  double c = 0.0;
  for (int64_t i = t; i < M; i += 1024) c += (double)counts[i];
  sh[t] = c;
  __syncthreads();
  for (int d = 512; d > 0; d >>= 1) {
    if (t < d) sh[t] += sh[t + d];
    __syncthreads();
  }
  if (t == 0) *scale = (float)(1.0 / fmax(sh[0], 1.0));
}

// The gradient of a row's logits, in place of them.  An entry's place is written by its first entry
// with the weights of all that name it; its logit is taken before the row is overwritten.
__global__ __launch_bounds__(256) void vocab_grad_kernel(VocabArgs a, float* __restrict__ z, int64_t ldz, int64_t v0, int n,
                                                         const float2* coef, const float* scale) {
  constexpr int EACH = kTopMax / 256;
  const int64_t row = blockIdx.x;
  float* s = z + row * ldz;
  const float2 c = coef[row];
  if (c.x == 0.f && c.y == 0.f) {
    for (int v = threadIdx.x; v < n; v += 256) s[v] = 0.f;
    return;
  }
  const float g = scale ? *scale : 1.f, lse = a.lse[row];
  const float ct = __fmul_rn(c.x, g), cp = __fmul_rn(c.y, g);
  auto grad = [&](float logit, float q) {
    const float zc = vocab_cap(logit, a.cap, a.rcap);
    const float p = expf(__fdiv_rn(zc, a.T) - lse);
    float d = __fmaf_rn(cp, p, -__fmul_rn(ct, q));
    if (a.cap > 0.f) {
      const float r = __fmul_rn(zc, a.rcap);
      d = __fmul_rn(d, __fmaf_rn(-r, r, 1.f));
    }
    return d;
  };
  const RowTarget r = row_target(a, row, threadIdx.x & 63);
  const int64_t at = row * a.k;
  int where[EACH];
  float d[EACH];
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    where[u] = -1;
    const int j = threadIdx.x + u * 256;
    if (j >= a.k) continue;
    const int64_t id = a.ids[at + j];
    if (id < v0 || id >= v0 + n) continue;
    float q = a.teacher ? 0.f : 1.f;
    bool first = true;
    if (a.teacher) {
      for (int i = 0; i < a.k; ++i) {
        if (a.ids[at + i] != id) continue;
        if (i < j) first = false;
        q = __fadd_rn(q, r.weight(teacher_logit(a, at + i)));
      }
    }
    if (!first) continue;
    where[u] = (int)(id - v0);
    d[u] = grad(s[id - v0], q);
  }
  __syncthreads();
  for (int v = threadIdx.x; v < n; v += 256) s[v] = grad(s[v], 0.f);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < EACH; ++u)
    if (where[u] >= 0) s[where[u]] = d[u];
}

// X for the backward's products: rows that get no gradient are zeros there, so that nothing they hold
// (a NaN times their zero gradient, too) reaches dW.
__global__ __launch_bounds__(256) void vocab_rows_kernel(const float* x, int64_t ldx, const float2* coef, float* dst, int64_t M,
                                                         int64_t K) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * K; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / K;
    const float2 c = coef[r];
    dst[i] = c.x == 0.f && c.y == 0.f ? 0.f : x[r * ldx + (i - r * K)];
  }
}

int store_grid(int64_t n) { return (int)std::min<int64_t>(4096, std::max<int64_t>(1, (n + 255) / 256)); }

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
  int64_t piece, ldz;
  size_t z, stat, counts, coef, scale, x, gemm, total;   // offsets; total: bytes
};

Plan plan_of(const VocabArgs& a, bool bwd) {
  Plan p{};
  p.piece = piece_of(a);
  p.ldz = up(p.piece, 4);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  p.z = take((size_t)a.M * p.ldz * 4);
  p.stat = take((size_t)a.M * 8);
  p.coef = p.stat;
  p.counts = take((size_t)a.M * 4);
  p.scale = take(4);
  auto bytes = [&](int kind, int64_t P, int64_t Q, int64_t R) {
    return gemm_workspace_bytes(kind, (int)P, (int)Q, (int)R);
  };
  size_t g = 0;
  for (int64_t n : {p.piece, a.V % p.piece ? a.V % p.piece : p.piece}) {
    g = std::max(g, bytes(EPI_FWD, a.M, n, a.K));
    if (bwd) g = std::max({g, bytes(EPI_DGRAD, a.M, a.K, n), bytes(EPI_WGRAD, n, a.K, a.M)});
  }
  if (bwd) p.x = take((size_t)a.M * a.K * 4);
  p.gemm = take(g);
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
  return vocab_tiles_ok(a) ? vocab_tiles_ws_bytes(a, bwd) : plan_of(a, bwd).total;
}

hipError_t vocab_fwd_launch(const VocabArgs& a, void* ws, hipStream_t s) {
  if (vocab_tiles_ok(a)) return vocab_tiles_fwd(a, ws, s);
  const Pieces g{a, plan_of(a, false), (char*)ws, s};
  Stat* stat = (Stat*)(g.ws + g.p.stat);
  float* counts = (float*)(g.ws + g.p.counts);
  for (int64_t v0 = 0; v0 < a.V; v0 += g.p.piece) {
    const int64_t n = std::min(g.p.piece, a.V - v0);
    TRY(g.logits((const float*)a.x, a.ldx, v0, n));
    hipLaunchKernelGGL(vocab_stats_kernel, dim3((unsigned)a.M), dim3(256), 0, s, a, g.z(), g.p.ldz, v0, (int)n, stat);
    TRY(hipGetLastError());
  }
  hipLaunchKernelGGL(vocab_loss_kernel, dim3((unsigned)((a.M + 3) / 4)), dim3(256), 0, s, a, stat, counts);
  TRY(hipGetLastError());
  if (a.mean) hipLaunchKernelGGL(vocab_mean_kernel, dim3(1), dim3(1024), 0, s, a.loss, counts, a.M, a.mean);
  return hipGetLastError();
}

hipError_t vocab_bwd_launch(const VocabArgs& a, void* ws, hipStream_t s) {
  if (vocab_tiles_ok(a)) return vocab_tiles_bwd(a, ws, s);
  const Pieces g{a, plan_of(a, true), (char*)ws, s};
  const Plan& p = g.p;
  float2* coef = (float2*)(g.ws + p.coef);
  float* counts = (float*)(g.ws + p.counts);
  float* scale = a.dloss ? nullptr : (float*)(g.ws + p.scale);
  hipLaunchKernelGGL(vocab_coef_kernel, dim3((unsigned)((a.M + 3) / 4)), dim3(256), 0, s, a, coef, counts);
  TRY(hipGetLastError());
  if (scale) hipLaunchKernelGGL(vocab_scale_kernel, dim3(1), dim3(1024), 0, s, counts, a.M, scale);
  TRY(hipGetLastError());
  float* x = (float*)(g.ws + p.x);
  hipLaunchKernelGGL(vocab_rows_kernel, dim3(store_grid(a.M * a.K)), dim3(256), 0, s, (const float*)a.x, a.ldx, coef, x, a.M, a.K);
  TRY(hipGetLastError());
  float* dx = (float*)a.dx;
  for (int64_t v0 = 0; v0 < a.V; v0 += p.piece) {
    const int64_t n = std::min(p.piece, a.V - v0);
    TRY(g.logits(x, a.K, v0, n));
    hipLaunchKernelGGL(vocab_grad_kernel, dim3((unsigned)a.M), dim3(256), 0, s, a, g.z(), p.ldz, v0, (int)n, coef, scale);
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
  return hipSuccess;
}

}  // namespace opfuse
