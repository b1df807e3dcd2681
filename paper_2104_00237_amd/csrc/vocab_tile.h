// Products of bf16 operands in tiles, for the vocabulary losses: C[p, q] = sum_r A(p, r) B(q, r) on
// v_mfma_f32_32x32x16_bf16, with what becomes of a finished tile left to an epilogue.
//
// A workgroup's wavefronts (WP x WQ of them) hold IP x IQ blocks of 32x32 each.  Operands go from
// memory straight to LDS, in stages of BK reduction elements, a ring of four of them:
//   step 0 .. n-2 of stage c   MFMAs of step k, LDS reads of step k + 1, the rest of stage c + 3 requested
//   barrier                    stage c has been read, stage c + 1 has landed; two stages stay in flight
//   step n-1                   MFMAs, reads of stage c + 1's step 0, the first loads of stage c + 4
// Loads are spread over all MFMAs: sixteen at once take a CU's load path twice the time of the MFMAs
// beside them, and the wavefront, which issues in order, waits.
//
// Operands are rows with the reduction index contiguous (RC: [x][r]) or the output index ([r][x]).  RC
// stages lie in LDS as rows [x][BK], 16-byte slots swizzled so that 16 consecutive rows' reads cover all
// banks; the others as rows [r][BX] with 64-byte blocks swizzled by r % 4, read with ds_read_b64_tr_b16.
// A load to LDS writes lane i at base + 16 i, so the swizzle is applied to the address each lane loads.
// Rows are whole 16-byte pieces at 16-byte boundaries; r past R and x past the operand read as zeros.
//
// fp32 operands (PL = 3) come as three bf16 planes each, x = high + middle + low with every part the
// nearest bf16 to what the ones before leave (the splitting of Henry, Tang and Heinecke, Leveraging the
// bfloat16 Artificial Intelligence Datatype For Higher-Precision Computations, ARITH 2019).  Parts shrink
// by 2^-9, so three hold all 24 bits, and of the nine partial products the three below 2^-26 of the
// whole are left out: six are summed in one accumulator.
#pragma once

#include <type_traits>
#include <utility>

#include "vocab.h"

namespace opfuse {

typedef __bf16 vbf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 vbf16x2_t __attribute__((ext_vector_type(2)));
typedef float vfloat2_t __attribute__((ext_vector_type(2)));
typedef short vshort4_t __attribute__((ext_vector_type(4)));
typedef short vshort8_t __attribute__((ext_vector_type(8)));
typedef float vacc_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ uint32_t pack2(float a, float b) {   // round to nearest even
  const vfloat2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, vbf16x2_t));
}

template <int... T, class F>
__device__ __forceinline__ void each(std::integer_sequence<int, T...>, F&& f) {
  (f(std::integral_constant<int, T>{}), ...);
}

template <int IP_, int IQ_, int WP_, int WQ_, int BK_, int OCC_>
struct TileShape {
  static constexpr int IP = IP_, IQ = IQ_, WP = WP_, WQ = WQ_, BK = BK_, OCC = OCC_;
  static constexpr int NW = WP * WQ, NT = NW * 64;
  static constexpr int BP = WP * IP * 32, BQ = WQ * IQ * 32;
  static constexpr int ABYTES = BP * BK * 2, BBYTES = BQ * BK * 2;
  static constexpr int NA = ABYTES / 1024 / NW, NB = BBYTES / 1024 / NW, NL = NA + NB;   // loads of a wavefront
  static constexpr int NK = BK / 16;                                                     // steps of a stage
  static_assert(NA * NW * 1024 == ABYTES && NB * NW * 1024 == BBYTES, "whole loads for every wavefront");
  static_assert(BK == 32 || BK == 64, "stages");
};

// Loads of one operand's stages by one wavefront: N instructions of 1 KB.
template <bool RC, int BX, int BK, int N>
struct StageLoad {
  uint32_t off[N];
  int r[N];
  __device__ __forceinline__ StageLoad(int64_t ld, int nx, int lane, int wave) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int blk = wave * N + i;
      int x;
      if constexpr (RC) {
        constexpr int S = BK / 8, PER = 64 / S, SH = BK == 64 ? 1 : 2;   // slots of a row, rows of a load
        x = blk * PER + lane / S;
        r[i] = ((lane % S) ^ ((x >> SH) & (S - 1))) * 8;
        off[i] = x < nx ? (uint32_t)((x * ld + r[i]) * 2) : kOOB;
      } else {
        constexpr int L = BX / 8;                                        // lanes of a row
        r[i] = blk * (64 / L) + lane / L;
        x = (((lane % L) >> 2) ^ (r[i] & 3)) * 32 + (lane & 3) * 8;
        off[i] = x < nx ? (uint32_t)((r[i] * ld + x) * 2) : kOOB;
      }
    }
  }
};

// One load of 1 KB to LDS.
__device__ __forceinline__ void load_lds(const rsrc_t& rs, char* lds, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)lds, 16, off, 0, 0, 0);
}

template <bool RC, int BX, int BK>
__device__ __forceinline__ vbf16x8_t stage_frag(const char* lds, int x0, int k, int lane) {
  if constexpr (RC) {
    constexpr int S = BK / 8, SH = BK == 64 ? 1 : 2;
    const int x = x0 + (lane & 31);
    return *reinterpret_cast<const vbf16x8_t*>(lds + x * (BK * 2) + (((2 * k + (lane >> 5)) ^ ((x >> SH) & (S - 1))) * 16));
  } else {
    const int r = k * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2);
    const int x = x0 + (lane & 16) + (lane & 3) * 4;
    const char* a = lds + r * (BX * 2) + ((x * 2) ^ ((r & 3) << 6));
    typedef __attribute__((address_space(3))) vshort4_t* lp;
    const vshort4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)a);
    const vshort4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(a + 4 * BX * 2));
    return __builtin_bit_cast(vbf16x8_t, (vshort8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
}

// One product.  P, Q, R may be larger than the product: rows (device memory, NULL: none) is the true
// size of the dimension that the epilogue names.
struct TileProblem {
  const uint16_t *A, *B;
  int64_t lda, ldb;
  int P, Q, R;
  const int* rows;
  int gp, gq, S;        // tiles, and parts of the reduction
  int64_t pa, pb;       // PL = 3: elements from one plane to the next
};
enum TileRows { ROWS_NONE = 0, ROWS_P = 1, ROWS_Q = 2, ROWS_R = 3 };

// What a workgroup of a product works on.
struct TilePlace {
  int p0, q0, np, nq;       // its corner, and rows and columns from there to the product's end
  int split, rbeg, rend;
};

// Tile of workgroup b: the XCDs take runs of tiles, and a run walks strips of 8 tile rows column by
// column, so that the tiles an XCD has at one time share their operands in its L2.
template <class T>
__device__ __forceinline__ bool tile_place(const TileProblem& pr, int rows_dim, TilePlace* t) {
  constexpr int G = 8;
  const int tiles = pr.gp * pr.gq;
  int l = xcd_run((int)blockIdx.x, tiles * pr.S);
  t->split = l / tiles;
  l -= t->split * tiles;
  const int strip = l / (G * pr.gq), in = l - strip * G * pr.gq, h = min(G, pr.gp - strip * G);
  const int tq = in / h, tp = strip * G + in - tq * h;
  const int n = rows_dim ? __builtin_amdgcn_readfirstlane(*pr.rows) : 0;
  const int P = rows_dim == ROWS_P ? n : pr.P, Q = rows_dim == ROWS_Q ? n : pr.Q, R = rows_dim == ROWS_R ? n : pr.R;
  t->p0 = tp * T::BP, t->q0 = tq * T::BQ;
  t->np = P - t->p0, t->nq = Q - t->q0;
  const int per = ((R + pr.S - 1) / pr.S + T::BK - 1) / T::BK * T::BK;
  t->rbeg = min(R, t->split * per), t->rend = min(R, t->rbeg + per);
  return t->np > 0 && t->nq > 0;
}

// The main loop.  e(place, acc, lds, lane, wave, wp, wq): the finished tile; lds: the ring, free.
template <class T, int PL, bool A_RC, bool B_RC, class Epi>
__global__ __launch_bounds__(T::NT, T::OCC) void tile_kernel(TileProblem pr, Epi e) {
  constexpr int IP = T::IP, IQ = T::IQ, NK = T::NK, NL = T::NL, STAGE = T::ABYTES + T::BBYTES;
  __shared__ __attribute__((aligned(1024))) char s0[STAGE], s1[STAGE], s2[STAGE], s3[STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wp = wave % T::WP, wq = wave / T::WP;
  TilePlace t;
  if (!tile_place<T>(pr, Epi::ROWS, &t)) return;
  const int nst = (t.rend - t.rbeg + T::BK - 1) / T::BK;
  const StageLoad<A_RC, T::BP, T::BK, T::NA> la(pr.lda, t.np, lane, wave);
  const StageLoad<B_RC, T::BQ, T::BK, T::NB> lb(pr.ldb, t.nq, lane, wave);
  const char* A = (const char*)(pr.A + (A_RC ? t.p0 * pr.lda + t.rbeg : t.rbeg * pr.lda + t.p0));
  const char* B = (const char*)(pr.B + (B_RC ? t.q0 * pr.ldb + t.rbeg : t.rbeg * pr.ldb + t.q0));
  const int64_t da = (A_RC ? 1 : pr.lda) * T::BK * 2, db = (B_RC ? 1 : pr.ldb) * T::BK * 2;

  vacc_t acc[IP][IQ];
#pragma unroll
  for (int i = 0; i < IP; ++i)
#pragma unroll
    for (int j = 0; j < IQ; ++j)
#pragma unroll
      for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.f;
  struct Frags {
    vbf16x8_t a[IP], b[IQ];
  };
  Frags f[2];

  // loads [from, to) of stage c.  Planes: a stage for each of the products high high, high middle, high
  // low, middle high, middle middle, low high of the same reduction elements
  auto request = [&](char* s, int c, int from, int to) __attribute__((always_inline)) {
    const int k = PL == 1 ? c : c / 6, pi = PL == 1 ? 0 : (c - k * 6) * 4;
    const int nr = k < nst ? t.rend - t.rbeg - k * T::BK : 0;   // 0 past the end: zeros
    const int64_t at = k < nst ? k : 0;
    const char *a = A + at * da, *b = B + at * db;
    if constexpr (PL == 3) a += (0x211000 >> pi & 3) * pr.pa * 2, b += (0x010210 >> pi & 3) * pr.pb * 2;
    const rsrc_t ra = make_rsrc(a), rb = make_rsrc(b);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      if (i < from || i >= to) continue;
      if (i < T::NA) {
        load_lds(ra, s + (wave * T::NA + i) * 1024, la.r[i % T::NA] < nr ? la.off[i % T::NA] : kOOB);
      } else {
        const int u = (i - T::NA) % T::NB;
        load_lds(rb, s + T::ABYTES + (wave * T::NB + u) * 1024, lb.r[u] < nr ? lb.off[u] : kOOB);
      }
    }
  };
  auto read = [&](Frags& d, const char* s, int k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < IP; ++i) d.a[i] = stage_frag<A_RC, T::BP, T::BK>(s, (wp * IP + i) * 32, k, lane);
#pragma unroll
    for (int j = 0; j < IQ; ++j) d.b[j] = stage_frag<B_RC, T::BQ, T::BK>(s + T::ABYTES, (wq * IQ + j) * 32, k, lane);
  };
  auto mfma = [&](const Frags& d) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < IP; ++i)
#pragma unroll
      for (int j = 0; j < IQ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(d.a[i], d.b[j], acc[i][j], 0, 0, 0);
  };
  // MFMAs with a share of the LDS reads and of the loads behind each
  constexpr int READS = (A_RC ? 1 : 2) * IP + (B_RC ? 1 : 2) * IQ, MF = IP * IQ;
  auto sched = [&](auto N) __attribute__((always_inline)) {
    constexpr int n = decltype(N)::value;
#pragma unroll
    for (int g = 0; g < MF; ++g) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
      for (int u = 0; u < READS; ++u)
        if (u * MF / READS / 2 == g) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
      for (int u = 0; u < n; ++u)
        if (u * MF / n + MF / n / 2 == g) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // loads that step k of a stage asks for (of stage c + 3; the last step: the first of stage c + 4)
  constexpr int L1 = (NL + NK - 1) / NK;

  // Stage c is in s, stage c + 1 lands in sn, stage c + 3 is asked for in s3n.
  auto stage = [&](char* s, char* sn, char* s3n, int c) __attribute__((always_inline)) {
    each(std::make_integer_sequence<int, NK - 1>{}, [&](auto K_) {
      constexpr int k = decltype(K_)::value;
      read(f[(k + 1) & 1], s, k + 1);
      request(s3n, c + 3, L1 + k * (NL - L1) / (NK - 1), L1 + (k + 1) * (NL - L1) / (NK - 1));
      mfma(f[k & 1]);
      sched(std::integral_constant<int, L1 + (k + 1) * (NL - L1) / (NK - 1) - (L1 + k * (NL - L1) / (NK - 1))>{});
    });
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * NL) : "memory");
    __builtin_amdgcn_sched_barrier(0);
    read(f[0], sn, 0);
    request(s, c + 4, 0, L1);
    mfma(f[(NK - 1) & 1]);
    sched(std::integral_constant<int, L1>{});
  };

  request(s0, 0, 0, NL);
  request(s1, 1, 0, NL);
  request(s2, 2, 0, NL);
  request(s3, 3, 0, L1);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * NL + L1) : "memory");
  __builtin_amdgcn_sched_barrier(0);
  read(f[0], s0, 0);
  __builtin_amdgcn_sched_barrier(0);
  // (stages past the end are zeros: a branch around them makes the compiler move accumulators
  // between register files)
  for (int c = 0; c < (PL == 1 ? nst : 6 * nst); c += 4) {
    stage(s0, s1, s3, c);
    stage(s1, s2, s0, c + 1);
    stage(s2, s3, s1, c + 2);
    stage(s3, s0, s2, c + 3);
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  char* const ring[4] = {s0, s1, s2, s3};
  e(t, acc, ring, lane, wave, wp, wq);
}

}  // namespace opfuse
