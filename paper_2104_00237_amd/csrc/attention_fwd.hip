// Softmax attention, forward: O = softmax(scale Q K^T + mask) V and lse = log sum exp, one pass over
// the keys with a running maximum and sum (the probabilities never reach memory).
//
// Bound by instruction issue.  Of 32 rows and 64 keys at width 64 a wavefront has 16 MFMAs (512 cycles)
// and, where nothing is masked, about 200 vector instructions, 32 of them exponentials at a quarter of
// the rate (1200 cycles); at width 128 the MFMAs take 1024.  Counted over whole kernels, MFMAs, masks,
// entry and exit included: 189 a tile for 16384 tokens of width 128, 257 for 4 x 1024 of width 64, where
// a wavefront has nine tiles on average.  Two wavefronts a SIMD fill each other's gaps; LDS delivers a
// fragment of a tile to every wavefront for one MFMA (half its rate at width 128).
// Measured, whole calls (a kernel trace adds up to a tenth): 16384 tokens, 16/4 heads of 128, causal
// 1.03 to 1.06 ms, 1.05 PFLOP/s (a library product of 16384^3: 1.33), MFMAs busy 58 % of the time; 4 x 1024
// tokens, 16 heads of 64, causal 22 us; fp32, 16 ragged sequences, 12 heads of 80: 123 us, 65 TFLOP/s
// (a library product of 8192^3: 154).

#include "attention.h"

namespace opfuse {

namespace {
constexpr int BM = 128;   // rows of a workgroup: (query, head of the group) pairs, 32 for each of its four wavefronts
}  // namespace

// Rows r of a key head's group: query r / G, head r % G, so that the query heads that share a key
// head share its tiles.  BN: keys of a tile.
template <typename T, int DP, int BN, bool VEC>
__global__ __launch_bounds__(256, DP <= (sizeof(T) == 2 ? 128 : 96) ? 2 : 1) void attn_fwd_kernel(AttnArgs a) {
  constexpr int ES = sizeof(T), SLOTS = slots_of(DP * ES), NS = DP * ES / 32, NB = DP / 32, NK = BN / 32;
  constexpr bool FRESH = ES == 4 ? DP == 256 || (!VEC && DP == 128) : !VEC && DP == 256;
  typedef typename Mma<T>::frag frag;
  constexpr int TB = BN * SLOTS * 16;
  __shared__ __attribute__((aligned(1024))) char sk0[TB], sk1[TB], sv0[TB], sv1[TB];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint32_t w = blockIdx.x;   // (32-bit divisions: a 64-bit one is 120 instructions)
  const int hk = (int)(w % (uint32_t)a.Hkv);
  w /= (uint32_t)a.Hkv;
  const int split = (int)(w % (uint32_t)a.nsplit);
  const uint32_t per_tile = (uint32_t)(a.Hkv * a.nsplit);
  w = paired(w / (uint32_t)a.nsplit, gridDim.x / per_tile, 256u / per_tile);
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
  klo = klo / BN;                           // in tiles from here on
  const int nt = max((khi + BN - 1) / BN - klo, 0);
  const int per = (int)((uint32_t)(nt + a.nsplit - 1) / (uint32_t)a.nsplit);
  const int t0 = klo + min(split * per, nt), t1 = klo + min(split * per + per, nt);
  const unsigned span = has ? max(hi - lo, 0) : 0;

  frag fq[NS];
  load_own<T, NS, VEC>(fq, (const T*)a.q.p + (q.beg + i) * a.q.ld + (int64_t)h * a.q.hs, has, a.D, lane);
  acc16_t acc[NB];
  zero_acc(acc);
  float m = -INFINITY, ms = 0.f, l = 0.f;
  constexpr float GROW = 8.f;

  const TileLoad<T, SLOTS, BN, 256, VEC> lk(a.k, a.D, tid), lv(a.v, a.D, tid);
  auto request = [&](char* k, char* v, int t) {
    lk(k, a.k, kv.beg + t * BN, hk, kv.len - t * BN, a.D, tid);
    lv(v, a.v, kv.beg + t * BN, hk, kv.len - t * BN, a.D, tid);
  };
  // One barrier a tile: tile t has landed and tile t - 1 has been read, so tile t + 1 is requested
  // into its place and has the time of tile t's products to arrive.
  auto step = [&](const char* sk, const char* sv, char* kn, char* vn, int t) {
    const int j0 = t * BN;
    tile_barrier();
    if (t + 1 < t1) request(kn, vn, t + 1);
    acc16_t z[NK];
    zero_acc(z);
#pragma unroll
    for (int n = 0; n < NK; ++n)
#pragma unroll
      for (int u = 0; u < NS; ++u) z[n] = Mma<T>::mma(row_frag<T, SLOTS>(sk, n * 32, u, fresh<FRESH>(lane)), fq[u], z[n]);
    if (j0 < lo1 || j0 + BN > hi0 || r1 - r0 < BM) {   // some row does not see some key
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int j = j0 + n * 32 + (k >> 2) * 8 + half * 4 + (k & 3);
          if ((unsigned)(j - lo) >= span) z[n][k] = -INFINITY;
        }
    }
    float top = z[0][0];
#pragma unroll
    for (int n = 0; n < NK; ++n)
#pragma unroll
      for (int k = n == 0; k < 16; ++k) top = maxi(top, z[n][k]);
    top = with_half(top, maxi) * a.c;
    // m is raised only where the maximum has grown by more than 2^GROW: P up to 2^GROW is as exact, and
    // most tiles then have no sums to scale
    if (__any(top > m + GROW)) {
      const float mn = maxi(m, top);
      ms = mn == -INFINITY ? 0.f : mn;      // no key so far: exp2(-inf - 0) = 0
      const float f = exp2_fast(m - ms);
      m = mn;
      l *= f;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[b][k] *= f;
    }
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NK; ++n)
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        z[n][k] = exp2_fast(__fmaf_rn(z[n][k], a.c, -ms));
        sum[k & 3] += z[n][k];
      }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
    for (int n = 0; n < NK; ++n)
#pragma unroll
      for (int u = 0; u < 32 / Mma<T>::TR; ++u) {
        const frag p = Mma<T>::pack(z[n], u);
#pragma unroll
        for (int b = 0; b < NB; ++b)
          acc[b] = Mma<T>::mma(Mma<T>::template tr<SLOTS>(sv, n * 32 + u * Mma<T>::TR, b * 32, fresh<FRESH>(lane)), p, acc[b]);
      }
  };
  if (t0 < t1) request(sk0, sv0, t0);
  for (int t = t0; t < t1; t += 2) {
    step(sk0, sv0, sk1, sv1, t);
    if (t + 1 < t1) step(sk1, sv1, sk0, sv0, t + 1);
  }
  l = half_sum(l);
  if (!has) return;
  const int64_t stat = (int64_t)h * a.Tq + q.beg + i;
  if (a.nsplit > 1) {      // this split's sums; attn_join_kernel puts them together
    const int64_t rows = (int64_t)a.Hq * a.Tq;
    float* part = a.part + (split * rows + stat) * a.D;
    store_own(part, acc, 1.f, a.D, a.D % 4 == 0, lane);
    if (half == 0) {
      float* st = a.part + a.nsplit * rows * a.D + (split * rows + stat) * 2;
      st[0] = m;
      st[1] = l;
    }
    return;
  }
  store_own((T*)a.o.p + (q.beg + i) * a.o.ld + (int64_t)h * a.o.hs, acc, l == 0.f ? 0.f : 1.f / l, a.D, a.ovec, lane);
  if (a.lse && half == 0) a.lse[stat] = l == 0.f ? -INFINITY : __fmaf_rn(m, kLn2, logf(l));
}

// Joins the splits of a row: O = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  A wavefront a row: its
// lanes hold the splits' statistics (at most 64), then columns; the splits' loads do not wait for
// each other (8 sequences of one token, 16 splits: 17 -> 7.5 us).
template <typename T>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  const int lane = threadIdx.x & 63;
  int s;
  int64_t tile;
  find_tile(a.q_off, a.Tq, a.nseq, a.Hq, 4, blockIdx.x, s, tile);
  const SeqRows q = seq_rows(a.q_off, a.q_len, a.Tq, a.nseq, s);
  const int64_t r = tile * 4 + (threadIdx.x >> 6);
  if (tile < 0 || r >= (int64_t)q.len * a.Hq) return;
  const int64_t i = (uint32_t)r / (uint32_t)a.Hq;
  const int h = (int)(r - i * a.Hq);
  const int64_t rows = (int64_t)a.Hq * a.Tq, stat = h * a.Tq + q.beg + i;
  const float* st = a.part + a.nsplit * rows * a.D + stat * 2;
  const float mine = lane < a.nsplit ? st[lane * rows * 2] : -INFINITY;
  const float sum = lane < a.nsplit ? st[lane * rows * 2 + 1] : 0.f;
  float m = mine;
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) m = maxi(m, __shfl_xor(m, k));
  const float f = exp2_fast(mine - (m == -INFINITY ? 0.f : m));   // a split that saw no key: 0
  float l = f * sum;
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) l += __shfl_xor(l, k);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* o = (T*)a.o.p + (q.beg + i) * a.o.ld + (int64_t)h * a.o.hs;
  const float* p = a.part + stat * a.D;
  const int64_t next = rows * a.D;
  for (int d0 = 0; d0 < a.D; d0 += 64) {
    const int d = min(d0 + lane, a.D - 1);
    float x = 0.f;
    for (int k0 = 0; k0 < a.nsplit; k0 += 8) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = p[min(k0 + k, a.nsplit - 1) * next + d];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k0 + k < a.nsplit) x = __fmaf_rn(__shfl(f, k0 + k), v[k], x);
    }
    if (d0 + lane < a.D) o[d] = Mma<T>::from(x * inv);
  }
  if (a.lse && lane == 0) a.lse[stat] = l == 0.f ? -INFINITY : __fmaf_rn(m, kLn2, logf(l));
}

namespace {
// Splits of the keys: where the rows give less than a workgroup a CU, enough parts to fill the chip
// twice, at least 512 keys (of an average sequence) in each and only from 2048 on: joining costs about
// 7 us, the time of 8 tiles of 64 keys.  Measured: 8 sequences of one token, up to 8192 keys, 16/4 heads
// (32 workgroups): 28 us in 16 parts, 34 in 32; 1024 queries of 16 heads: 25 us in 4 parts, 21 unsplit.
// The rule sees the slots, not a window: then the window's tiles alone are shared out, and some parts
// may have none.  8 sequences of one token in slots of 8192, causal window of 64 / 512 / 1024 / 2000 keys: 14
// / 14 / 14 / 16 us in 16 parts, 8 / 18 / 29 / 51 us unsplit.
int splits(const AttnArgs& a) {
  const int64_t wgs = attn_tiles(a.Tq, a.nseq, a.q_off != nullptr, a.G, BM) * a.Hkv;
  const int64_t keys = a.Tk / a.nseq;
  int64_t n = 1;
  if (wgs < 256 && keys >= 2048) n = std::min<int64_t>((512 + wgs - 1) / wgs, keys / 512);
  return (int)std::min<int64_t>(n, 64);
}

template <typename T, int DP, int BN, bool VEC>
hipError_t launch(const AttnArgs& a, hipStream_t stream) {
  const int64_t n = attn_tiles(a.Tq, a.nseq, a.q_off != nullptr, a.G, BM) * a.Hkv * a.nsplit;
  hipLaunchKernelGGL((attn_fwd_kernel<T, DP, BN, VEC>), dim3((unsigned)n), dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  const int64_t nj = attn_tiles(a.Tq, a.nseq, a.q_off != nullptr, a.Hq, 4);
  hipLaunchKernelGGL((attn_join_kernel<T>), dim3((unsigned)nj), dim3(256), 0, stream, a);
  return hipGetLastError();
}
}  // namespace

size_t attn_fwd_ws_bytes(const AttnArgs& a) {
  const int n = splits(a);
  return n == 1 ? 0 : (size_t)n * a.Hq * a.Tq * (a.D + 2) * 4;
}

hipError_t attn_fwd_launch(AttnArgs a, bool bf16, bool vec, void* ws, hipStream_t stream) {
  a.nsplit = splits(a);
  a.part = (float*)ws;
  // widths between the powers of two have their own products where the loads are whole slots
  if (bf16) {
    if (!vec) {
      if (a.D <= 64) return launch<uint16_t, 64, 64, false>(a, stream);
      if (a.D <= 128) return launch<uint16_t, 128, 64, false>(a, stream);
      return launch<uint16_t, 256, 64, false>(a, stream);
    }
    if (a.D <= 64) return launch<uint16_t, 64, 64, true>(a, stream);
    if (a.D <= 96) return launch<uint16_t, 96, 64, true>(a, stream);
    if (a.D <= 128) return launch<uint16_t, 128, 64, true>(a, stream);
    if (a.D <= 192) return launch<uint16_t, 192, 64, true>(a, stream);
    return launch<uint16_t, 256, 64, true>(a, stream);
  }
  if (!vec) {
    if (a.D <= 64) return launch<float, 64, 32, false>(a, stream);
    if (a.D <= 128) return launch<float, 128, 32, false>(a, stream);
    return launch<float, 256, 32, false>(a, stream);
  }
  if (a.D <= 64) return launch<float, 64, 32, true>(a, stream);
  if (a.D <= 96) return launch<float, 96, 32, true>(a, stream);
  if (a.D <= 128) return launch<float, 128, 32, true>(a, stream);
  if (a.D <= 192) return launch<float, 192, 32, true>(a, stream);
  return launch<float, 256, 32, true>(a, stream);
}

}  // namespace opfuse
