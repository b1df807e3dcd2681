// Softmax attention, backward.  The probabilities are computed again from the forward's row
// statistics, P = exp(scale S - lse), so nothing of size queries x keys is stored:
//   delta_i = sum_d dO_id O_id                      (= sum_j P_ij dP_ij)
//   dP = dO V^T,  dS = P (dP - delta)
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K
// Two launches: delta and dQ with a wavefront's own queries in its columns and the keys streaming by;
// dK and dV with its own keys and the queries streaming.  Seven products instead of the five of one
// joint pass, whose dQ would be summed by atomics (in no fixed order) or through queries x key tiles
// of partial sums in memory.  Every sum has one owner and one order, so results are deterministic.
//
// Accumulators start from what would be subtracted from them: S from -lse / scale (bf16 operands; for
// fp32 operands that would round at lse's size) and dP from -delta, and masked elements from
// -infinity, so that P = exp2(c S) and dS = P dP.
//
// Measured, whole calls: 8192 tokens, 16/4 heads of 128, causal 0.98 to 1.00 ms (690 TFLOP/s of the five
// products); 4 x 1024 tokens, 16 heads of 64 59 us, 16/4 heads 67 us and with fp32 gradients 85 us; fp32,
// window 512, 8/4 heads of 64 253 us.  Launch by launch, in a kernel trace that adds up to a tenth: the
// first of these dQ 397 us, dK and dV 666, their sum 16; the 85 us dQ 47 (dO is read and its copy written
// element by element), dK and dV 35, their sum 9.  A step costs its MFMAs, its fragments' LDS reads and,
// in dK and dV, a share of 28 vector cycles for each of 16 elements.

#include "attention.h"

namespace opfuse {

namespace {
constexpr int BK = 128;         // dK and dV: own rows of a workgroup
constexpr int BM = 128;         // dQ: own rows of a workgroup, 32 for each of its four wavefronts
// dQ: keys up to which delta is summed from the probabilities.  bf16 gradients were 1.52 times as far
// from float64 as their own rounding leaves them (dQ and dK of 2 short sequences, dK of 8192 tokens),
// and are 1.41 with it; the time is the same (72.5 us both ways for 4 x 1024 tokens).
constexpr int kExactKeys = 256;

// fp32 dO as the products' operand: rounded, and kept for the second launch.
template <int NS>
__device__ __forceinline__ void round_own(abf16x8_t (&f)[NS], const float* row, uint16_t* copy, bool has, int D, int lane) {
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = (2 * s + (lane >> 5)) * 8;
    uint16_t t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t[e] = has && d + e < D ? f32_to_bf16(row[d + e]) : 0;
      if (has && d + e < D) copy[d + e] = t[e];
    }
    f[s] = __builtin_bit_cast(abf16x8_t, t);
  }
}

// Products of the lane's part of two rows.
template <int NS>
__device__ __forceinline__ float dot_own(const abf16x8_t (&a)[NS], const abf16x8_t (&b)[NS]) {
  float x = 0.f;
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) x = __fmaf_rn((float)a[s][e], (float)b[s][e], x);
  return x;
}
template <int NS>
__device__ __forceinline__ float dot_own(const afloatx4_t (&a)[NS], const afloatx4_t (&b)[NS]) {
  float x = 0.f;
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int e = 0; e < 4; ++e) x = __fmaf_rn(a[s][e], b[s][e], x);
  return x;
}
}  // namespace

// delta and dQ: own rows are queries (all heads of a key head's group), keys stream.  copy: dO rounded
// to T when it is stored in another type (copy_strides).
template <typename T, typename G, int DP, int BN, int RD, bool VEC>
__global__ __launch_bounds__(256, DP <= (sizeof(T) == 2 ? 128 : 64) ? 2 : 1) void attn_dq_kernel(AttnArgs a, T* copy) {
  constexpr int ES = sizeof(T), SLOTS = slots_of(DP * ES), NS = DP * ES / 32, NB = DP / 32, NK = BN / 32, U = 32 / Mma<T>::TR;
  constexpr bool INIT = ES == 2;   // S starts from -lse / scale
  constexpr bool FRESH = ES == 4 ? DP >= 128 : !VEC && DP == 256;
  typedef typename Mma<T>::frag frag;
  constexpr int TB = BN * SLOTS * 16;
  __shared__ __attribute__((aligned(1024))) char sk0[TB], sk1[TB], sv0[TB], sv1[TB];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint32_t w = blockIdx.x;   // (32-bit divisions: a 64-bit one is 120 instructions)
  const int hk = (int)(w % (uint32_t)a.Hkv);
  w = paired(w / (uint32_t)a.Hkv, gridDim.x / (uint32_t)a.Hkv, 256u / (uint32_t)a.Hkv);
  int s;
  int64_t tile;
  find_tile(a.q_off, a.Tq, a.nseq, a.G, BM, w, s, tile);
  const SeqRows q = seq_rows(a.q_off, a.q_len, a.Tq, a.nseq, s);
  const SeqRows kv = seq_rows(a.k_off, a.k_len, a.Tk, a.nseq, s);
  const int64_t R = (int64_t)q.len * a.G;
  const int64_t tiles = (R + BM - 1) / BM;
  if (tile < 0 || tile >= tiles) return;
  tile = tiles - 1 - tile;                  // with a causal mask the longest rows come first
  const int shift = kv.len - q.len;
  const int r0 = (int)(tile * BM), r1 = (int)min(R, (int64_t)r0 + BM);
  const int r = r0 + wave * 32 + (lane & 31);
  const bool has = r < R;
  const int i = fdiv(has ? r : r0, a.dG), h = hk * a.G + ((has ? r : r0) - i * a.G);
  int lo, hi, klo, khi, lo1, hi0;
  keys_of(a.causal, a.window, i, shift, kv.len, lo, hi);
  // keys of the tile's rows: [klo, khi); seen by every row: [lo1, hi0)
  keys_of(a.causal, a.window, fdiv(r0, a.dG), shift, kv.len, klo, hi0);
  keys_of(a.causal, a.window, fdiv(r1 - 1, a.dG), shift, kv.len, lo1, khi);
  const int t0 = klo / BN, t1 = (khi + BN - 1) / BN;
  const unsigned span = has ? max(hi - lo, 0) : 0;

  const int64_t row = q.beg + i, stat = (int64_t)h * a.Tq + row;
  constexpr bool KEEP = kKeepOwn<T, DP>;
  frag fq[KEEP ? NS : 1], fo[KEEP ? NS : 1];
  const T* prow = (const T*)a.dout.p + row * a.dout.ld + (int64_t)h * a.dout.hs;
  const T* qrow = (const T*)a.q.p + row * a.q.ld + (int64_t)h * a.q.hs;
  const T* orow = (const T*)a.o.p + row * a.o.ld + (int64_t)h * a.o.hs;
  float delta = 0.f;
  if constexpr (!KEEP) {
    for (int s = 0; s < NS; ++s) {
      fq[0] = own_frag<T, VEC>(orow, has, s, a.D, lane);
      fo[0] = own_frag<T, VEC>(prow, has, s, a.D, lane);
      delta += dot_own(fq, fo);
    }
    delta = half_sum(delta);
  } else if constexpr (sizeof(T) == sizeof(G))
    load_own<T, NS, VEC>(fo, prow, has, a.D, lane);
  else
    round_own(fo, (const G*)a.dout.p + row * a.dout.ld + (int64_t)h * a.dout.hs, copy + stat * a.D, has, a.D, lane);
  if constexpr (KEEP) {
    load_own<T, NS, VEC>(fq, orow, has, a.D, lane);
    delta = half_sum(dot_own(fq, fo));
    load_own<T, NS, VEC>(fq, qrow, has, a.D, lane);
  }
  // a row that saw no key (lse -inf) or does not exist has no probabilities: exp2(s - inf) = 0
  const float lse = a.lse[stat], lse2 = has && lse > -INFINITY ? lse * kLog2e : INFINITY;
  const float z0 = INIT ? -lse2 * a.rc : 0.f;
  acc16_t acc[NB];
  zero_acc(acc);

  const TileLoad<T, SLOTS, BN, 256, VEC> lk(a.k, a.D, tid), lv(a.v, a.D, tid);
  auto request = [&](char* k, char* v, int t) {
    lk(k, a.k, kv.beg + t * BN, hk, kv.len - t * BN, a.D, tid);
    lv(v, a.v, kv.beg + t * BN, hk, kv.len - t * BN, a.D, tid);
  };
  // One barrier a tile: tile t has landed and tile t - 1 has been read, so tile t + 1 is requested
  // into its place and has the time of tile t's products to arrive.
  // A block of 32 keys is a chain of steps, each a fragment of a streamed tile (requested RD steps
  // ahead): S from K rows; dP from V rows, beside them P; then dQ from K columns, or with ONLY the
  // sum of P (dP - delta) into `more`.
  float more = 0.f;
  auto step = [&](auto ONLY, const char* sk, const char* sv, char* kn, char* vn, int t) __attribute__((always_inline)) {
    const int j0 = t * BN;
    tile_barrier();
    if (t + 1 < t1) request(kn, vn, t + 1);
    const bool part = j0 < lo1 || j0 + BN > hi0 || r1 - r0 < BM;
    each<NK>([&](auto N) __attribute__((always_inline)) {
      constexpr int n = N * 32, N1 = NS, N2 = 2 * NS, N3 = N2 + (ONLY ? 0 : U * NB);
      acc16_t z, p;
      float zi = z0, pi = -delta;
      asm volatile("" : "+v"(zi), "+v"(pi));   // (else 32 registers hold copies of them across the loop)
#pragma unroll
      for (int k = 0; k < 16; ++k) z[k] = zi, p[k] = pi;
      if (part) {
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int j = j0 + n + (k >> 2) * 8 + half * 4 + (k & 3);
          if ((unsigned)(j - lo) >= span) z[k] = -INFINITY;
        }
      }
      auto fetch = [&](auto I) __attribute__((always_inline)) {
        if constexpr (I < N1) return row_frag<T, SLOTS>(sk, n, I, fresh<FRESH>(lane));
        else if constexpr (I < N2) return row_frag<T, SLOTS>(sv, n, I - N1, fresh<FRESH>(lane));
        else return Mma<T>::template tr<SLOTS>(sk, n + (I - N2) / NB * Mma<T>::TR, (I - N2) % NB * 32, fresh<FRESH>(lane));
      };
      frag ring[RD + 1], own, mine[KEEP ? 1 : OD + 1];
      auto fetch_own = [&](auto I) __attribute__((always_inline)) {
        if constexpr (!KEEP && I < N2) mine[I % (OD + 1)] = own_frag<T, VEC>(I < N1 ? qrow : prow, has, I < N1 ? I : I - N1, a.D, lane);
      };
      if constexpr (!KEEP) each<OD>(fetch_own);
      each<RD>([&](auto I) __attribute__((always_inline)) { ring[I] = fetch(I); });
      each<N3>([&](auto I) __attribute__((always_inline)) {
        if constexpr (I + RD < N3) ring[(I + RD) % (RD + 1)] = fetch(std::integral_constant<int, I + RD>{});
        fetch_own(std::integral_constant<int, I + OD>{});
        const frag f = ring[I % (RD + 1)];
        if constexpr (I < N1) {
          z = Mma<T>::mma(f, KEEP ? fq[KEEP ? I : 0] : mine[KEEP ? 0 : I % (OD + 1)], z);
        } else if constexpr (I < N2) {
          constexpr int i = I - N1;
          p = Mma<T>::mma(f, KEEP ? fo[KEEP ? i : 0] : mine[KEEP ? 0 : I % (OD + 1)], p);
#pragma unroll
          for (int k = 16 * i / NS; k < 16 * (i + 1) / NS; ++k)
            z[k] = exp2_fast(INIT ? z[k] * a.c : __fmaf_rn(z[k], a.c, -lse2));
        } else {
          constexpr int u = (I - N2) / NB, b = (I - N2) % NB, K = Mma<T>::TR / 2;
          if constexpr (b == 0) {
#pragma unroll
            for (int k = u * K; k < u * K + K; ++k) p[k] *= z[k];
            own = Mma<T>::pack(p, u);
          }
          acc[b] = Mma<T>::mma(f, own, acc[b]);
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (ONLY) {
#pragma unroll
        for (int k = 0; k < 16; ++k) more = __fmaf_rn(z[k], p[k], more);
      }
    });
  };
  auto walk = [&](auto ONLY) __attribute__((always_inline)) {
    if (t0 < t1) request(sk0, sv0, t0);
    for (int t = t0; t < t1; t += 2) {
      step(ONLY, sk0, sv0, sk1, sv1, t);
      if (t + 1 < t1) step(ONLY, sk1, sv1, sk0, sv0, t + 1);
    }
  };
  if constexpr (ES == 2) {
    // Few keys: delta from the probabilities instead of from the rounded O, whose error weighs most
    // here (O of n keys is about V / sqrt(n), so the error falls as 1 / sqrt(n) against dP).
    if (t1 - t0 <= kExactKeys / BN) {
      walk(std::true_type{});
      delta += half_sum(more);
      tile_barrier();    // the last tile has been read
    }
  }
  if (has && half == 0) a.delta[stat] = delta;
  walk(std::false_type{});
  if (!has) return;
  store_own((G*)a.dq.p + row * a.dq.ld + (int64_t)h * a.dq.hs, acc, a.scale, a.D, a.ovec, lane);
}

// dK and dV: own rows are keys, 32 a wavefront; the queries of the group's heads stream, one head after
// the other; a split takes a run of their tiles.
// DO: columns of dK and dV a workgroup computes (all of them, or a part chosen by its number).
// A block of 32 queries is a chain of steps as in attn_dq_kernel: S from Q rows; dP from dO rows, beside
// them P; dV from dO columns, beside them dS = P dP; dK from Q columns.
// Width 128 takes 420 registers (128 of sums, 64 of K and V): one wavefront a SIMD, whose own chain
// has to keep the matrix cores fed (busy 43 % of the time; bwd_splits has the times); in 256 registers
// the compiler spills (2.7 times the time), with 64 own keys it shuffles sums between register files
// (4 times).
template <typename T, typename G, int DP, int DO, int BQ, int RD, int OCC, bool VEC>
__global__ __launch_bounds__(256, OCC) void attn_dkv_kernel(AttnArgs a) {
  constexpr int ES = sizeof(T), SLOTS = slots_of(DP * ES), NS = DP * ES / 32, NB = DO / 32, U = 32 / Mma<T>::TR;
  constexpr int TB = BQ * SLOTS * 16;
  constexpr bool INIT = ES == 2;   // S starts from -lse / scale
  constexpr bool FRESH = ES == 4 ? DP >= 128 : !VEC && DP == 256;
  typedef typename Mma<T>::frag frag;
  __shared__ __attribute__((aligned(1024))) char sq0[TB], sq1[TB], so0[TB], so1[TB];
  __shared__ __attribute__((aligned(16))) float sl[2][BQ], sd[2][BQ];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint32_t w = blockIdx.x;
  const int hk = (int)(w % (uint32_t)a.Hkv);
  w /= (uint32_t)a.Hkv;
  const int split = (int)(w % (uint32_t)a.nsplit);
  w /= (uint32_t)a.nsplit;
  static_assert(DP % DO == 0, "whole parts");
  const int d0 = (int)(w % (DP / DO)) * DO;   // first column of dK and dV
  const uint32_t per_tile = (uint32_t)(a.Hkv * a.nsplit * (DP / DO));
  w = paired(w / (DP / DO), gridDim.x / per_tile, 256u / per_tile);
  if (d0 >= a.D) return;
  int s;
  int64_t tile;
  find_tile(a.k_off, a.Tk, a.nseq, 1, BK, w, s, tile);
  const SeqRows q = seq_rows(a.q_off, a.q_len, a.Tq, a.nseq, s);
  const SeqRows kv = seq_rows(a.k_off, a.k_len, a.Tk, a.nseq, s);
  if (tile < 0 || tile * BK >= kv.len) return;
  const int shift = kv.len - q.len;
  const int j0 = (int)(tile * BK), j1 = min(kv.len, j0 + BK);
  int qlo, qhi, lo1, hi0;
  queries_of(a.causal, a.window, j0, shift, q.len, qlo, hi0);       // queries of the tile's keys: [qlo, qhi),
  queries_of(a.causal, a.window, j1 - 1, shift, q.len, lo1, qhi);   // of all of them: [lo1, hi0)
  const int jw = j0 + wave * 32 + (lane & 31);
  const bool has = jw < kv.len;
  const int j = has ? jw : j0;
  int lo, hi;
  queries_of(a.causal, a.window, j, shift, q.len, lo, hi);
  const unsigned span = has ? max(hi - lo, 0) : 0;

  const int64_t row = kv.beg + j;
  constexpr bool KEEP = kKeepOwn<T, DP>;
  frag fk[KEEP ? NS : 1], fv[KEEP ? NS : 1];
  const T* krow = (const T*)a.k.p + row * a.k.ld + (int64_t)hk * a.k.hs;
  const T* vrow = (const T*)a.v.p + row * a.v.ld + (int64_t)hk * a.v.hs;
  if constexpr (KEEP) {
    load_own<T, NS, VEC>(fk, krow, has, a.D, lane);
    load_own<T, NS, VEC>(fv, vrow, has, a.D, lane);
  }
  acc16_t ak[NB], av[NB];
  zero_acc(ak);
  zero_acc(av);

  // tiles of queries, all heads of the group one after the other, and this split's run of them
  const int nt = max((qhi - qlo + BQ - 1) / BQ, 0);
  const int all = nt * a.G, run = (int)((uint32_t)(all + a.nsplit - 1) / (uint32_t)a.nsplit);   // < 2^31: Tq Hq is
  const int first = min(split * run, all);
  const int total = min(run, all - first);
  const TileLoad<T, SLOTS, BQ, 256, VEC> lq(a.q, a.D, tid), ld_(a.dout, a.D, tid);
  float nl = 0.f, nd = 0.f;    // statistics of the tile on its way
  int g1 = nt ? (int)((uint32_t)first / (uint32_t)nt) : 0, i1 = qlo + (first - g1 * nt) * BQ;   // its head and first query
  int i0 = i1;
  int left = total;
  auto request = [&](char* q1, char* o1) {
    const int h = hk * a.G + (left > 0 ? g1 : 0), n = left > 0 ? q.len - i1 : 0;   // past the run: zeros
    --left;
    lq(q1, a.q, q.beg + i1, h, n, a.D, tid);
    ld_(o1, a.dout, q.beg + i1, h, n, a.D, tid);
    if (tid < BQ) {
      const int64_t stat = (int64_t)h * a.Tq + q.beg + (n > 0 ? i1 + min(tid, n - 1) : 0);
      nl = a.lse[stat];
      nd = -a.delta[stat];
      // a query that sees no key (lse -inf) or does not exist: exp2(s - inf) = 0
      nl = tid < n && nl > -INFINITY ? -nl * (INIT ? a.rc * kLog2e : kLog2e) : -INFINITY;
    }
    i1 += BQ;
    if (i1 >= qhi) i1 = qlo, ++g1;
  };
  auto step = [&](const char* sq, const char* so, float* ls, float* ds, char* q1, char* o1) __attribute__((always_inline)) {
    if (tid < BQ) ls[tid] = nl, ds[tid] = nd;
    tile_barrier();
    request(q1, o1);
    const bool part = i0 < lo1 || i0 + BQ > hi0 || j1 - j0 < BK;
    each<BQ / 32>([&](auto X) __attribute__((always_inline)) {
      constexpr int x = X * 32, N1 = NS, N2 = 2 * NS, N3 = N2 + U * NB, N4 = N3 + U * NB;
      acc16_t z, p;
      float l[INIT ? 1 : 16];
#pragma unroll
      for (int k4 = 0; k4 < 4; ++k4) {
        const float4 l4 = ld4(ls + x + k4 * 8 + half * 4), d4 = ld4(ds + x + k4 * 8 + half * 4);
        const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (!INIT) l[k4 * 4 + e] = lv[e];
          z[k4 * 4 + e] = INIT ? lv[e] : 0.f;
          p[k4 * 4 + e] = dv[e];
        }
      }
      if (part) {
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int i = i0 + x + (k >> 2) * 8 + half * 4 + (k & 3);
          if ((unsigned)(i - lo) >= span) z[k] = -INFINITY;
        }
      }
      auto fetch = [&](auto I) __attribute__((always_inline)) {
        if constexpr (I < N1) return row_frag<T, SLOTS>(sq, x, I, fresh<FRESH>(lane));
        else if constexpr (I < N2) return row_frag<T, SLOTS>(so, x, I - N1, fresh<FRESH>(lane));
        else if constexpr (I < N3) return Mma<T>::template tr<SLOTS>(so, x + (I - N2) / NB * Mma<T>::TR, d0 + (I - N2) % NB * 32, fresh<FRESH>(lane));
        else return Mma<T>::template tr<SLOTS>(sq, x + (I - N3) / NB * Mma<T>::TR, d0 + (I - N3) % NB * 32, fresh<FRESH>(lane));
      };
      frag ring[RD + 1], own, mine[KEEP ? 1 : OD + 1];
      auto fetch_own = [&](auto I) __attribute__((always_inline)) {
        if constexpr (!KEEP && I < N2) mine[I % (OD + 1)] = own_frag<T, VEC>(I < N1 ? krow : vrow, has, I < N1 ? I : I - N1, a.D, lane);
      };
      if constexpr (!KEEP) each<OD>(fetch_own);
      each<RD>([&](auto I) __attribute__((always_inline)) { ring[I] = fetch(I); });
      each<N4>([&](auto I) __attribute__((always_inline)) {
        if constexpr (I + RD < N4) ring[(I + RD) % (RD + 1)] = fetch(std::integral_constant<int, I + RD>{});
        fetch_own(std::integral_constant<int, I + OD>{});
        const frag f = ring[I % (RD + 1)];
        if constexpr (I < N1) {
          z = Mma<T>::mma(f, KEEP ? fk[KEEP ? I : 0] : mine[KEEP ? 0 : I % (OD + 1)], z);
        } else if constexpr (I < N2) {
          constexpr int i = I - N1;
          p = Mma<T>::mma(f, KEEP ? fv[KEEP ? i : 0] : mine[KEEP ? 0 : I % (OD + 1)], p);
#pragma unroll
          for (int k = 16 * i / NS; k < 16 * (i + 1) / NS; ++k)
            z[k] = exp2_fast(INIT ? z[k] * a.c : __fmaf_rn(z[k], a.c, l[INIT ? 0 : k]));
        } else if constexpr (I < N3) {
          constexpr int i = I - N2, u = i / NB, b = i % NB;
          if constexpr (b == 0) own = Mma<T>::pack(z, u);
          av[b] = Mma<T>::mma(f, own, av[b]);
#pragma unroll
          for (int k = 16 * i / (U * NB); k < 16 * (i + 1) / (U * NB); ++k) p[k] *= z[k];
        } else {
          constexpr int i = I - N3, u = i / NB, b = i % NB;
          if constexpr (b == 0) own = Mma<T>::pack(p, u);
          ak[b] = Mma<T>::mma(f, own, ak[b]);
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    });
    i0 += BQ;
    if (i0 >= qhi) i0 = qlo;
  };
  // (two tiles a turn, a missing second one as zeros: a branch around it would make the compiler move
  // accumulators about)
  if (total > 0) request(sq0, so0);
  for (int t = 0; t < total; t += 2) {
    step(sq0, so0, sl[0], sd[0], sq1, so1);
    step(sq1, so1, sl[1], sd[1], sq0, so0);
  }
  tile_barrier();
  if (!has) return;
  if (a.nsplit > 1) {      // this split's sums; attn_sum_kernel puts them together
    float* part = a.part + (((int64_t)split * 2 * a.Tk + row) * a.Hkv + hk) * a.D + d0;
    store_own(part, ak, 1.f, a.D - d0, a.D % 4 == 0, lane);
    store_own(part + a.Tk * a.Hkv * a.D, av, 1.f, a.D - d0, a.D % 4 == 0, lane);
    return;
  }
  store_own((G*)a.dk.p + row * a.dk.ld + (int64_t)hk * a.dk.hs + d0, ak, a.scale, a.D - d0, a.ovec, lane);
  store_own((G*)a.dv.p + row * a.dv.ld + (int64_t)hk * a.dv.hs + d0, av, 1.f, a.D - d0, a.ovec, lane);
}

// Sums the splits of dK and dV in their order.  SUM_ROWS (key, head) rows a workgroup.
constexpr int SUM_ROWS = 16;
template <typename G>
__global__ __launch_bounds__(256) void attn_sum_kernel(AttnArgs a) {
  int s;
  int64_t tile;
  find_tile(a.k_off, a.Tk, a.nseq, a.Hkv, SUM_ROWS, blockIdx.x, s, tile);
  const SeqRows kv = seq_rows(a.k_off, a.k_len, a.Tk, a.nseq, s);
  const int64_t R = (int64_t)kv.len * a.Hkv, r0 = tile * SUM_ROWS;
  if (tile < 0 || r0 >= R) return;
  const int n = (int)min((int64_t)SUM_ROWS, R - r0) * a.D;
  const int64_t one = a.Tk * a.Hkv * a.D;
  for (int e = threadIdx.x; e < n; e += 256) {
    const int x = (int)((uint32_t)e / (uint32_t)a.D), d = e - x * a.D;
    const int64_t row = (uint32_t)(r0 + x) / (uint32_t)a.Hkv;
    const int hk = (int)(r0 + x - row * a.Hkv);
    const float* p = a.part + ((kv.beg + row) * a.Hkv + hk) * a.D + d;
    float k = p[0], v = p[one];
    for (int i = 1; i < a.nsplit; ++i) {
      p += 2 * one;
      k += p[0];
      v += p[one];
    }
    ((G*)a.dk.p)[(kv.beg + row) * a.dk.ld + hk * a.dk.hs + d] = Mma<G>::from(k * a.scale);
    ((G*)a.dv.p)[(kv.beg + row) * a.dv.ld + hk * a.dv.hs + d] = Mma<G>::from(v);
  }
}

namespace {
// Splits of the queries that stream past a key tile (128 keys): where the key tiles are fewer than two
// workgroups a CU, at least eight tiles of queries (of an average sequence) in each.  Measured (traced): 8192
// tokens, 16/4 heads of 128 (256 workgroups, the causal mask's longest twice the mean): dK and dV 1450
// us unsplit, in 2 parts 658 + 18 us for their sum, in 4 parts 675 + 26, in 8 706 + 61.
// 4 x 1024 tokens, 16 heads of 64 (512 workgroups): unsplit 42, in 2 parts 42 + 18.
int bwd_splits(const AttnArgs& a, bool bf16) {
  const int parts = a.D <= 128 ? 1 : 2, queries = bf16 && a.D <= 128 ? 64 : 32;
  const int64_t wgs = attn_tiles(a.Tk, a.nseq, a.k_off != nullptr, 1, BK) * a.Hkv * parts;
  const int64_t rows = std::min<int64_t>(a.Tq / a.nseq, a.window ? 2 * (int64_t)a.window + 128 : a.Tq);
  const int64_t tiles = rows * a.G / queries;
  int64_t n = 1;
  if (wgs < 512) n = std::min<int64_t>((512 + wgs - 1) / wgs, std::max<int64_t>(1, tiles / 8));
  return (int)std::min<int64_t>(n, 16);
}

size_t stat_bytes(const AttnArgs& a) { return (((size_t)a.Hq * a.Tq + 3) & ~(size_t)3) * 4; }
size_t copy_bytes(const AttnArgs& a) { return ((size_t)a.Hq * a.Tq * a.D * 2 + 15) & ~(size_t)15; }

template <typename T, typename G, int DP, int DO, int BQ, int RD, int OCC, int BN, bool VEC>
hipError_t launch_as(AttnArgs a, T* copy, hipStream_t stream) {
  const int64_t nq = attn_tiles(a.Tq, a.nseq, a.q_off != nullptr, a.G, BM) * a.Hkv;
  hipLaunchKernelGGL((attn_dq_kernel<T, G, DP, BN, sizeof(T) == 2 && DP == 64 ? 2 : 1, VEC>), dim3((unsigned)nq), dim3(256), 0, stream, a, copy);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (copy) {
    a.dout.p = copy;
    copy_strides(a.Tq, a.D, a.dout.ld, a.dout.hs);
  }
  const int64_t nk = attn_tiles(a.Tk, a.nseq, a.k_off != nullptr, 1, BK) * (DP / DO) * a.Hkv * a.nsplit;
  hipLaunchKernelGGL((attn_dkv_kernel<T, G, DP, DO, BQ, RD, OCC, VEC>), dim3((unsigned)nk), dim3(256), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  const int64_t ns = attn_tiles(a.Tk, a.nseq, a.k_off != nullptr, a.Hkv, SUM_ROWS);
  hipLaunchKernelGGL((attn_sum_kernel<G>), dim3((unsigned)ns), dim3(256), 0, stream, a);
  return hipGetLastError();
}
template <typename T, typename G>
hipError_t launch(AttnArgs a, bool vec, void* ws, hipStream_t stream) {
  constexpr bool conv = sizeof(T) != sizeof(G);
  a.delta = (float*)ws;
  T* copy = conv ? (T*)((char*)ws + stat_bytes(a)) : nullptr;
  a.nsplit = bwd_splits(a, sizeof(T) == 2);
  a.part = (float*)((char*)ws + stat_bytes(a) + (conv ? copy_bytes(a) : 0));
  // widths between the powers of two have their own products where the loads are whole slots
  if constexpr (sizeof(T) == 2) {
    if (!vec) {
      if (a.D <= 64) return launch_as<T, G, 64, 64, 64, 2, 2, 64, false>(a, copy, stream);
      if (a.D <= 128) return launch_as<T, G, 128, 128, 64, 3, 1, 64, false>(a, copy, stream);
      return launch_as<T, G, 256, 128, 32, 2, 1, 32, false>(a, copy, stream);
    }
    if (a.D <= 64) return launch_as<T, G, 64, 64, 64, 2, 2, 64, true>(a, copy, stream);
    if (a.D <= 96) return launch_as<T, G, 96, 96, 64, 3, 1, 64, true>(a, copy, stream);
    if (a.D <= 128) return launch_as<T, G, 128, 128, 64, 3, 1, 64, true>(a, copy, stream);
    if (a.D <= 192) return launch_as<T, G, 192, 96, 32, 2, 1, 32, true>(a, copy, stream);
    return launch_as<T, G, 256, 128, 32, 2, 1, 32, true>(a, copy, stream);
  } else {
    if (!vec) {
      if (a.D <= 64) return launch_as<T, G, 64, 64, 32, 2, 1, 32, false>(a, copy, stream);
      if (a.D <= 128) return launch_as<T, G, 128, 128, 32, 1, 1, 32, false>(a, copy, stream);
      return launch_as<T, G, 256, 128, 32, 1, 1, 32, false>(a, copy, stream);
    }
    if (a.D <= 64) return launch_as<T, G, 64, 64, 32, 2, 1, 32, true>(a, copy, stream);
    if (a.D <= 96) return launch_as<T, G, 96, 96, 32, 2, 1, 32, true>(a, copy, stream);
    if (a.D <= 128) return launch_as<T, G, 128, 128, 32, 1, 1, 32, true>(a, copy, stream);
    if (a.D <= 192) return launch_as<T, G, 192, 96, 32, 1, 1, 32, true>(a, copy, stream);
    return launch_as<T, G, 256, 128, 32, 1, 1, 32, true>(a, copy, stream);
  }
}
}  // namespace

size_t attn_bwd_ws_bytes(const AttnArgs& a, bool bf16, bool grad_bf16) {
  const int n = bwd_splits(a, bf16);
  return stat_bytes(a) + (bf16 != grad_bf16 ? copy_bytes(a) : 0) +
         (n == 1 ? 0 : (size_t)n * 2 * a.Tk * a.Hkv * a.D * 4);
}

hipError_t attn_bwd_launch(AttnArgs a, bool bf16, bool grad_bf16, bool vec, void* ws, hipStream_t stream) {
  if (!bf16) return launch<float, float>(a, vec, ws, stream);
  return grad_bf16 ? launch<uint16_t, uint16_t>(a, vec, ws, stream) : launch<uint16_t, float>(a, vec, ws, stream);
}

}  // namespace opfuse
