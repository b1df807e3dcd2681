// Softmax attention, backward.  The probabilities are computed again from the forward's row
// statistics, P = exp(scale S - lse), so nothing of size queries x keys is stored:
//   delta_i = sum_d dO_id O_id                      (= sum_j P_ij dP_ij)
//   dP = dO V^T,  dS = P (dP - delta)
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K
// Three launches: delta; dK and dV with a wavefront's own keys in its columns and the queries
// streaming by; dQ with its own queries and the keys streaming.  Every sum has one owner and one
// order (the query heads of a key head are summed in its workgroup), so results are deterministic.

#include "attention.h"

namespace opfuse {

namespace {
constexpr int NW = 4;
constexpr int BM = 32 * NW;   // own rows of a workgroup
}  // namespace

// delta, and dO rounded to the products' operand type when it is stored in another (fp32 gradients
// of bf16 operands: dO as the products see it also enters delta).  A wavefront a row.
template <typename T, typename G>
__global__ __launch_bounds__(256) void attn_delta_kernel(AttnArgs a, T* copy) {
  const int lane = threadIdx.x & 63;
  int s;
  int64_t tile;
  find_tile(a.q_off, a.Tq, a.nseq, a.Hq, 4, blockIdx.x, s, tile);
  const SeqRows q = seq_rows(a.q_off, a.q_len, a.Tq, a.nseq, s);
  const int64_t r = tile * 4 + (threadIdx.x >> 6);
  if (tile < 0 || r >= (int64_t)q.len * a.Hq) return;
  const int64_t i = r / a.Hq, t = q.beg + i;
  const int h = (int)(r - i * a.Hq);
  const T* o = (const T*)a.o.p + t * a.o.ld + (int64_t)h * a.o.hs;
  const G* g = (const G*)a.dout.p + t * a.dout.ld + (int64_t)h * a.dout.hs;
  float x = 0.f;
  for (int d = lane; d < a.D; d += 64) {
    const T v = Mma<T>::from(Mma<G>::to(g[d]));
    if (copy) copy[((int64_t)t * a.Hq + h) * a.D + d] = v;
    x = __fmaf_rn(Mma<T>::to(v), Mma<T>::to(o[d]), x);
  }
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) x += __shfl_xor(x, k);
  if (lane == 0) a.delta[(int64_t)h * a.Tq + t] = x;
}

// dQ: own rows are queries (all heads of a key head's group), keys stream.
template <typename T, typename G, int DP, int BN, bool VEC>
__global__ __launch_bounds__(256) void attn_dq_kernel(AttnArgs a) {
  constexpr int ES = sizeof(T), SLOTS = DP * ES / 16, NS = SLOTS / 2, NB = DP / 32, NK = BN / 32;
  typedef typename Mma<T>::frag frag;
  __shared__ __attribute__((aligned(1024))) char sk[BN * SLOTS * 16], sv[BN * SLOTS * 16];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int64_t w = blockIdx.x;
  const int hk = (int)(w % a.Hkv);
  w /= a.Hkv;
  int s;
  int64_t tile;
  find_tile(a.q_off, a.Tq, a.nseq, a.G, BM, w, s, tile);
  const SeqRows q = seq_rows(a.q_off, a.q_len, a.Tq, a.nseq, s);
  const SeqRows kv = seq_rows(a.k_off, a.k_len, a.Tk, a.nseq, s);
  const int64_t R = (int64_t)q.len * a.G;
  const int64_t tiles = (R + BM - 1) / BM;
  if (tile < 0 || tile >= tiles) return;
  tile = tiles - 1 - tile;
  const int shift = kv.len - q.len;
  const int r0 = (int)(tile * BM), r1 = (int)min(R, (int64_t)r0 + BM);
  const int r = r0 + wave * 32 + (lane & 31);
  const bool has = r < R;
  const int i = fdiv(has ? r : r0, a.dG), h = hk * a.G + ((has ? r : r0) - i * a.G);
  int lo, hi, klo, khi, lo1, hi0;
  keys_of(a.causal, a.window, i, shift, kv.len, lo, hi);
  keys_of(a.causal, a.window, fdiv(r0, a.dG), shift, kv.len, klo, hi0);
  keys_of(a.causal, a.window, fdiv(r1 - 1, a.dG), shift, kv.len, lo1, khi);
  const int t0 = klo / BN, t1 = (khi + BN - 1) / BN;
  const unsigned span = has ? max(hi - lo, 0) : 0;

  frag fq[NS], fo[NS];
  load_own<T, NS, VEC>(fq, (const T*)a.q.p + (q.beg + i) * a.q.ld + (int64_t)h * a.q.hs, has, a.D, lane);
  load_own<T, NS, VEC>(fo, (const T*)a.dout.p + (q.beg + i) * a.dout.ld + (int64_t)h * a.dout.hs, has, a.D, lane);
  const int64_t stat = (int64_t)h * a.Tq + q.beg + i;
  // a row that saw no key (lse -inf) or does not exist has no probabilities: exp2(s - inf) = 0
  const float lse = a.lse[stat], lse2 = has && lse > -INFINITY ? lse * kLog2e : INFINITY;
  const float delta = a.delta[stat];
  acc16_t acc[NB];
  zero_acc(acc);

  for (int t = t0; t < t1; ++t) {
    const int j0 = t * BN;
    __syncthreads();
    load_tile<T, SLOTS, BN, 256, VEC>(sk, a.k, kv.beg + j0, hk, min(BN, kv.len - j0), a.D, tid);
    load_tile<T, SLOTS, BN, 256, VEC>(sv, a.v, kv.beg + j0, hk, min(BN, kv.len - j0), a.D, tid);
    __syncthreads();
    const bool part = j0 < lo1 || j0 + BN > hi0 || r1 - r0 < BM;
#pragma unroll
    for (int n = 0; n < NK; ++n) {
      acc16_t z[1], p[1];
      zero_acc(z);
      zero_acc(p);
#pragma unroll
      for (int u = 0; u < NS; ++u) z[0] = Mma<T>::mma(row_frag<T, SLOTS>(sk, n * 32, u, lane), fq[u], z[0]);
#pragma unroll
      for (int u = 0; u < NS; ++u) p[0] = Mma<T>::mma(row_frag<T, SLOTS>(sv, n * 32, u, lane), fo[u], p[0]);
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const int j = j0 + n * 32 + (k >> 2) * 8 + half * 4 + (k & 3);
        const float e = exp2_fast(__fmaf_rn(z[0][k], a.c, -lse2));
        z[0][k] = part && (unsigned)(j - lo) >= span ? 0.f : e * (p[0][k] - delta);
      }
#pragma unroll
      for (int u = 0; u < 32 / Mma<T>::TR; ++u) {
        const frag f = Mma<T>::pack(z[0], u);
#pragma unroll
        for (int b = 0; b < NB; ++b)
          acc[b] = Mma<T>::mma(Mma<T>::template tr<SLOTS>(sk, n * 32 + u * Mma<T>::TR, b * 32, lane), f, acc[b]);
      }
    }
  }
  if (!has) return;
  store_own((G*)a.dq.p + (q.beg + i) * a.dq.ld + (int64_t)h * a.dq.hs, acc, a.scale, a.D, a.ovec, lane);
}

// dK and dV: own rows are keys, the queries of the group's heads stream, one head after the other.
// DO: columns of dK and dV a workgroup computes (all of them, or a part chosen by its number).
template <typename T, typename G, int DP, int DO, int BQ, bool VEC>
__global__ __launch_bounds__(256) void attn_dkv_kernel(AttnArgs a) {
  constexpr int ES = sizeof(T), SLOTS = DP * ES / 16, NS = SLOTS / 2, NB = DO / 32, NQ = BQ / 32;
  typedef typename Mma<T>::frag frag;
  __shared__ __attribute__((aligned(1024))) char sq[BQ * SLOTS * 16], so[BQ * SLOTS * 16];
  __shared__ float sl[BQ], sd[BQ];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int64_t w = blockIdx.x;
  const int hk = (int)(w % a.Hkv);
  w /= a.Hkv;
  const int d0 = (int)(w % (DP / DO)) * DO;   // first column of dK and dV
  w /= DP / DO;
  if (d0 >= a.D) return;
  int s;
  int64_t tile;
  find_tile(a.k_off, a.Tk, a.nseq, 1, BM, w, s, tile);
  const SeqRows q = seq_rows(a.q_off, a.q_len, a.Tq, a.nseq, s);
  const SeqRows kv = seq_rows(a.k_off, a.k_len, a.Tk, a.nseq, s);
  if (tile < 0 || tile * BM >= kv.len) return;
  const int shift = kv.len - q.len;
  const int j0 = (int)(tile * BM), j1 = min(kv.len, j0 + BM);
  const int j = j0 + wave * 32 + (lane & 31);
  const bool has = j < kv.len;
  int lo, hi, qlo, qhi, lo1, hi0;
  queries_of(a.causal, a.window, has ? j : j0, shift, q.len, lo, hi);
  queries_of(a.causal, a.window, j0, shift, q.len, qlo, hi0);       // queries of the tile's keys: [qlo, qhi),
  queries_of(a.causal, a.window, j1 - 1, shift, q.len, lo1, qhi);   // of all of them: [lo1, hi0)
  const unsigned span = has ? max(hi - lo, 0) : 0;

  frag fk[NS], fv[NS];
  load_own<T, NS, VEC>(fk, (const T*)a.k.p + (kv.beg + (has ? j : j0)) * a.k.ld + (int64_t)hk * a.k.hs, has, a.D, lane);
  load_own<T, NS, VEC>(fv, (const T*)a.v.p + (kv.beg + (has ? j : j0)) * a.v.ld + (int64_t)hk * a.v.hs, has, a.D, lane);
  acc16_t ak[NB], av[NB];
  zero_acc(ak);
  zero_acc(av);

  for (int g = 0; g < a.G; ++g) {
    const int h = hk * a.G + g;
    for (int i0 = qlo; i0 < qhi; i0 += BQ) {
      const int n = min(BQ, q.len - i0);
      __syncthreads();
      load_tile<T, SLOTS, BQ, 256, VEC>(sq, a.q, q.beg + i0, h, n, a.D, tid);
      load_tile<T, SLOTS, BQ, 256, VEC>(so, a.dout, q.beg + i0, h, n, a.D, tid);
      if (tid < BQ) {
        const int64_t stat = (int64_t)h * a.Tq + q.beg + i0 + min(tid, n - 1);
        const float lse = a.lse[stat];
        sl[tid] = tid < n && lse > -INFINITY ? lse * kLog2e : INFINITY;
        sd[tid] = a.delta[stat];
      }
      __syncthreads();
      const bool part = i0 < lo1 || i0 + BQ > hi0 || j1 - j0 < BM;
#pragma unroll
      for (int m = 0; m < NQ; ++m) {
        acc16_t z[1], p[1];
        zero_acc(z);
        zero_acc(p);
#pragma unroll
        for (int u = 0; u < NS; ++u) z[0] = Mma<T>::mma(row_frag<T, SLOTS>(sq, m * 32, u, lane), fk[u], z[0]);
#pragma unroll
        for (int u = 0; u < NS; ++u) p[0] = Mma<T>::mma(row_frag<T, SLOTS>(so, m * 32, u, lane), fv[u], p[0]);
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4) {
          const int x = m * 32 + k4 * 8 + half * 4;
          const float4 ls = ld4(sl + x), de = ld4(sd + x);
          const float lsv[4] = {ls.x, ls.y, ls.z, ls.w}, dev[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int k = k4 * 4 + e;
            const float pr = exp2_fast(__fmaf_rn(z[0][k], a.c, -lsv[e]));
            const bool no = part && (unsigned)(i0 + x + e - lo) >= span;
            z[0][k] = no ? 0.f : pr;
            p[0][k] = no ? 0.f : pr * (p[0][k] - dev[e]);
          }
        }
#pragma unroll
        for (int u = 0; u < 32 / Mma<T>::TR; ++u) {
          const frag fp = Mma<T>::pack(z[0], u), fs = Mma<T>::pack(p[0], u);
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            av[b] = Mma<T>::mma(Mma<T>::template tr<SLOTS>(so, m * 32 + u * Mma<T>::TR, d0 + b * 32, lane), fp, av[b]);
            ak[b] = Mma<T>::mma(Mma<T>::template tr<SLOTS>(sq, m * 32 + u * Mma<T>::TR, d0 + b * 32, lane), fs, ak[b]);
          }
        }
      }
    }
  }
  if (!has) return;
  const int64_t row = kv.beg + j;
  store_own((G*)a.dk.p + row * a.dk.ld + (int64_t)hk * a.dk.hs + d0, ak, a.scale, a.D - d0, a.ovec, lane);
  store_own((G*)a.dv.p + row * a.dv.ld + (int64_t)hk * a.dv.hs + d0, av, 1.f, a.D - d0, a.ovec, lane);
}

namespace {
template <typename T, typename G, int DP, int DO, int BN, bool VEC>
hipError_t launch_vec(const AttnArgs& a, hipStream_t stream) {
  const int64_t nk = attn_tiles(a.Tk, a.nseq, a.k_off != nullptr, 1, BM) * (DP / DO) * a.Hkv;
  hipLaunchKernelGGL((attn_dkv_kernel<T, G, DP, DO, BN, VEC>), dim3((unsigned)nk), dim3(256), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t nq = attn_tiles(a.Tq, a.nseq, a.q_off != nullptr, a.G, BM) * a.Hkv;
  hipLaunchKernelGGL((attn_dq_kernel<T, G, DP, BN, VEC>), dim3((unsigned)nq), dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <typename T, typename G>
hipError_t launch(AttnArgs a, bool vec, void* ws, hipStream_t stream) {
  constexpr bool conv = sizeof(T) != sizeof(G);
  a.delta = (float*)ws;
  T* copy = conv ? (T*)(a.delta + (((int64_t)a.Hq * a.Tq + 3) & ~3ll)) : nullptr;
  const int64_t nd = attn_tiles(a.Tq, a.nseq, a.q_off != nullptr, a.Hq, 4);
  hipLaunchKernelGGL((attn_delta_kernel<T, G>), dim3((unsigned)nd), dim3(256), 0, stream, a, copy);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (conv) a.dout = HeadRows{copy, (int64_t)a.Hq * a.D, a.D};
  if (sizeof(T) == 2) {
    if (a.D <= 64) return vec ? launch_vec<T, G, 64, 64, 64, true>(a, stream) : launch_vec<T, G, 64, 64, 64, false>(a, stream);
    if (a.D <= 128) return vec ? launch_vec<T, G, 128, 128, 64, true>(a, stream) : launch_vec<T, G, 128, 128, 64, false>(a, stream);
    return vec ? launch_vec<T, G, 256, 128, 32, true>(a, stream) : launch_vec<T, G, 256, 128, 32, false>(a, stream);
  }
  if (a.D <= 64) return vec ? launch_vec<T, G, 64, 64, 32, true>(a, stream) : launch_vec<T, G, 64, 64, 32, false>(a, stream);
  if (a.D <= 128) return vec ? launch_vec<T, G, 128, 128, 32, true>(a, stream) : launch_vec<T, G, 128, 128, 32, false>(a, stream);
  return vec ? launch_vec<T, G, 256, 64, 32, true>(a, stream) : launch_vec<T, G, 256, 64, 32, false>(a, stream);
}
}  // namespace

size_t attn_bwd_ws_bytes(const AttnArgs& a, bool bf16, bool grad_bf16) {
  const size_t stats = (((size_t)a.Hq * a.Tq + 3) & ~(size_t)3) * 4;
  return stats + (bf16 != grad_bf16 ? (((size_t)a.Hq * a.Tq * a.D * 2 + 15) & ~(size_t)15) : 0);
}

hipError_t attn_bwd_launch(AttnArgs a, bool bf16, bool grad_bf16, bool vec, void* ws, hipStream_t stream) {
  if (!bf16) return launch<float, float>(a, vec, ws, stream);
  return grad_bf16 ? launch<uint16_t, uint16_t>(a, vec, ws, stream) : launch<uint16_t, float>(a, vec, ws, stream);
}

}  // namespace opfuse
