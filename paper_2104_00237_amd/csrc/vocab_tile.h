// Products of bf16 operands in tiles, for the vocabulary losses: C[p, q] = sum_r A(p, r) B(q, r) on
// v_mfma_f32_32x32x16_bf16, with what becomes of a finished tile left to an epilogue.
//
// A workgroup's wavefronts (WP x WQ of them) hold IP x IQ blocks of 32x32 each.  Operands go from
// memory straight to LDS, in stages of BK reduction elements, a ring of NS of them:
//   step 0 .. n-2 of stage c   MFMAs of step k, LDS reads of step k + 1, the rest of stage c + NS - 1 requested
//   barrier                    stage c has been read, stage c + 1 has landed; NS - 2 stages stay in flight
//   step n-1                   MFMAs, reads of stage c + 1's step 0, the first loads of stage c + NS
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
// whole are left out: six are summed in one accumulator.  An infinite x is (0, 0, x): its low part meets the
// other operand's high part alone.
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

template <int IP_, int IQ_, int WP_, int WQ_, int BK_, int NS_, int OCC_>
struct TileShape {
  static constexpr int IP = IP_, IQ = IQ_, WP = WP_, WQ = WQ_, BK = BK_, NS = NS_, OCC = OCC_;
  static constexpr int NW = WP * WQ, NT = NW * 64;
  static constexpr int BP = WP * IP * 32, BQ = WQ * IQ * 32;
  static constexpr int ABYTES = BP * BK * 2, BBYTES = BQ * BK * 2;
  static constexpr int NA = ABYTES / 1024 / NW, NB = BBYTES / 1024 / NW, NL = NA + NB;   // loads of a wavefront
  static constexpr int NK = BK / 16;                                                     // steps of a stage
  static_assert(NA * NW * 1024 == ABYTES && NB * NW * 1024 == BBYTES, "whole loads for every wavefront");
  static_assert(BK == 32 || BK == 64, "stages");
  static_assert(NS == 3 || NS == 4, "stages of the ring");
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

// A workgroup's tile: what its main loop works on.
template <class T, int PL, bool A_RC, bool B_RC, class Epi>
struct TileLoop {
  static constexpr int IP = T::IP, IQ = T::IQ, NK = T::NK, MF = IP * IQ;
  static constexpr int READA = (A_RC ? 1 : 2) * IP, READB = (B_RC ? 1 : 2) * IQ;   // LDS reads of a step
  const TileProblem& pr;
  const TilePlace& t;
  const int lane, wave, wp, wq, nst;
  const StageLoad<A_RC, T::BP, T::BK, T::NA> la;
  const StageLoad<B_RC, T::BQ, T::BK, T::NB> lb;
  const char *A, *B;
  const int64_t da, db;
  vacc_t (&acc)[IP][IQ];

  __device__ __forceinline__ TileLoop(const TileProblem& pr_, const TilePlace& t_, vacc_t (&acc_)[IP][IQ], int lane_, int wave_)
      : pr(pr_), t(t_), lane(lane_), wave(wave_), wp(wave_ % T::WP), wq(wave_ / T::WP),
        nst((t_.rend - t_.rbeg + T::BK - 1) / T::BK), la(pr_.lda, t_.np, lane_, wave_), lb(pr_.ldb, t_.nq, lane_, wave_),
        A((const char*)(pr_.A + (A_RC ? t_.p0 * pr_.lda + t_.rbeg : t_.rbeg * pr_.lda + t_.p0))),
        B((const char*)(pr_.B + (B_RC ? t_.q0 * pr_.ldb + t_.rbeg : t_.rbeg * pr_.ldb + t_.q0))),
        da((A_RC ? 1 : pr_.lda) * T::BK * 2), db((B_RC ? 1 : pr_.ldb) * T::BK * 2), acc(acc_) {
#pragma unroll
    for (int i = 0; i < IP; ++i)
#pragma unroll
      for (int j = 0; j < IQ; ++j)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.f;
  }
  // Reduction elements of stage c inside the operands (0 past the end: zeros), and where it starts.
  __device__ __forceinline__ int inside(int c) const { return c < nst ? t.rend - t.rbeg - c * T::BK : 0; }
  __device__ __forceinline__ int64_t start(int c) const { return c < nst ? c : 0; }
  // Loads [FROM, TO) of this wavefront of A's stage c, plane p.
  template <int FROM, int TO>
  __device__ __forceinline__ void load_a(char* s, int c, int p) const {
    const int nr = inside(c);
    const rsrc_t r = make_rsrc(A + start(c) * da + p * pr.pa * 2);
#pragma unroll
    for (int i = FROM; i < TO; ++i) load_lds(r, s + (wave * T::NA + i) * 1024, la.r[i] < nr ? la.off[i] : kOOB);
  }
  template <int FROM, int TO>
  __device__ __forceinline__ void load_b(char* s, int c, int p) const {
    const int nr = inside(c);
    const rsrc_t r = make_rsrc(B + start(c) * db + p * pr.pb * 2);
#pragma unroll
    for (int i = FROM; i < TO; ++i) load_lds(r, s + (wave * T::NB + i) * 1024, lb.r[i] < nr ? lb.off[i] : kOOB);
  }
  __device__ __forceinline__ void read_a(vbf16x8_t (&f)[IP], const char* s, int k) const {
#pragma unroll
    for (int i = 0; i < IP; ++i) f[i] = stage_frag<A_RC, T::BP, T::BK>(s, (wp * IP + i) * 32, k, lane);
  }
  __device__ __forceinline__ void read_b(vbf16x8_t (&f)[IQ], const char* s, int k) const {
#pragma unroll
    for (int j = 0; j < IQ; ++j) f[j] = stage_frag<B_RC, T::BQ, T::BK>(s, (wq * IQ + j) * 32, k, lane);
  }
  __device__ __forceinline__ void mfma(const vbf16x8_t (&a)[IP], const vbf16x8_t (&b)[IQ]) const {
#pragma unroll
    for (int i = 0; i < IP; ++i)
#pragma unroll
      for (int j = 0; j < IQ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
  }
  // A step's MFMAs with a share of its LDS reads and of its loads behind each.
  template <int READS, int LOADS>
  __device__ __forceinline__ static void sched() {
#pragma unroll
    for (int g = 0; g < MF; ++g) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
      for (int u = 0; u < READS; ++u)
        if (u * MF / READS / 2 == g) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
      for (int u = 0; u < LOADS; ++u)
        if (u * MF / LOADS + MF / LOADS / 2 == g) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // All LDS reads of this wavefront done and all but its LEFT latest loads landed; then everyone's.
  template <int LEFT>
  __device__ __forceinline__ static void sync() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
};

// LDS arrays by their addresses.  (Opaque to the compiler, which otherwise makes a constant table of
// them, where LDS addresses cannot stand.)
typedef __attribute__((address_space(3))) char lds_char;
struct Ring {
  uint32_t at[8];
};
__device__ __forceinline__ uint32_t lds_address(char* p) {
  uint32_t a = (uint32_t)(uintptr_t)(lds_char*)p;
  asm volatile("" : "+s"(a));
  return a;
}

// The main loop.  e(place, acc, ring, lane, wave, wp, wq): the finished tile; ring: LDS, free, in arrays
// of kRingBytes.
template <class T, int PL>
constexpr int kRingBytes = PL == 1 ? T::ABYTES + T::BBYTES : T::ABYTES < T::BBYTES ? T::ABYTES : T::BBYTES;
template <class T, int PL>
constexpr int kRingArrays = PL == 1 ? T::NS : 8;

template <class T, bool A_RC, bool B_RC, class Epi>
__device__ __forceinline__ void tile_body1(const TileProblem& pr, const TilePlace& t, const Epi& e, int lane, int wave) {
  constexpr int IP = T::IP, IQ = T::IQ, NK = T::NK, NA = T::NA, NL = T::NL, NS = T::NS, STAGE = T::ABYTES + T::BBYTES;
  using Loop = TileLoop<T, 1, A_RC, B_RC, Epi>;
  __shared__ __attribute__((aligned(1024))) char s0[STAGE], s1[STAGE], s2[STAGE], s3[NS == 4 ? STAGE : 16];
  vacc_t acc[IP][IQ];
  const Loop l(pr, t, acc, lane, wave);
  vbf16x8_t a[2][IP], b[2][IQ];

  // loads [FROM, TO) of stage c, A's first
  auto request = [&](char* s, int c, auto From, auto To) __attribute__((always_inline)) {
    constexpr int from = decltype(From)::value, to = decltype(To)::value;
    if constexpr (from < NA) l.template load_a<from, (to < NA ? to : NA)>(s, c, 0);
    if constexpr (to > NA) l.template load_b<(from > NA ? from - NA : 0), to - NA>(s + T::ABYTES, c, 0);
  };
  auto read = [&](int f, const char* s, int k) __attribute__((always_inline)) {
    l.read_a(a[f], s, k);
    l.read_b(b[f], s + T::ABYTES, k);
  };
  // loads that the last step of a stage asks for, the first of stage c + NS
  constexpr int L1 = (NL + NK - 1) / NK;
  using First = std::integral_constant<int, L1>;
  using Zero = std::integral_constant<int, 0>;
  using All = std::integral_constant<int, NL>;
  // Stage c is in s, stage c + 1 lands in sn, the rest of stage c + NS - 1 is asked for in sl.
  auto stage = [&](char* s, char* sn, char* sl, int c) __attribute__((always_inline)) {
    each(std::make_integer_sequence<int, NK - 1>{}, [&](auto K_) __attribute__((always_inline)) {
      constexpr int k = decltype(K_)::value;
      constexpr int from = L1 + k * (NL - L1) / (NK - 1), to = L1 + (k + 1) * (NL - L1) / (NK - 1);
      read((k + 1) & 1, s, k + 1);
      request(sl, c + NS - 1, std::integral_constant<int, from>{}, std::integral_constant<int, to>{});
      l.mfma(a[k & 1], b[k & 1]);
      Loop::template sched<Loop::READA + Loop::READB, to - from>();
    });
    Loop::template sync<(NS - 2) * NL>();
    read(0, sn, 0);
    request(s, c + NS, Zero{}, First{});
    l.mfma(a[(NK - 1) & 1], b[(NK - 1) & 1]);
    Loop::template sched<Loop::READA + Loop::READB, L1>();
  };

  request(s0, 0, Zero{}, All{});
  request(s1, 1, Zero{}, All{});
  if constexpr (NS == 4) {
    request(s2, 2, Zero{}, All{});
    request(s3, 3, Zero{}, First{});
  } else {
    request(s2, 2, Zero{}, First{});
  }
  Loop::template sync<(NS - 2) * NL + L1>();
  read(0, s0, 0);
  __builtin_amdgcn_sched_barrier(0);
  // (stages past the end are zeros: a branch around them makes the compiler move accumulators
  // between register files)
  for (int c = 0; c < l.nst; c += NS) {
    if constexpr (NS == 4) {
      stage(s0, s1, s3, c);
      stage(s1, s2, s0, c + 1);
      stage(s2, s3, s1, c + 2);
      stage(s3, s0, s2, c + 3);
    } else {
      stage(s0, s1, s2, c);
      stage(s1, s2, s0, c + 1);
      stage(s2, s0, s1, c + 2);
    }
  }
  Loop::template sync<0>();
  const Ring ring{{lds_address(s0), lds_address(s1), lds_address(s2), NS == 4 ? lds_address(s3) : 0u, 0u, 0u, 0u, 0u}};
  e(t, acc, ring, lane, wave, l.wp, l.wq);
}

// Three planes: six products of a stage's 32 reduction elements in six phases of two steps, each plane
// loaded to LDS once,
//   phase      0            1            2            3              4               5
//   product    high high    high middle  high low     middle high    middle middle   low high
//   loads      A low        B high'      A high'      B middle'      B low'          A middle'   (': next stage)
// A's fragments stay in registers while their plane is in use.  A slot is asked for once its last reader
// is behind a barrier, three phases before its first; B's high and middle planes have two slots each.
template <class T, bool A_RC, bool B_RC, class Epi>
__device__ __forceinline__ void tile_body3(const TileProblem& pr, const TilePlace& t, const Epi& e, int lane, int wave) {
  constexpr int IP = T::IP, IQ = T::IQ, NA = T::NA, NB = T::NB, A1 = (NA + 1) / 2, B1 = (NB + 1) / 2;
  static_assert(T::NK == 2, "stages of 32");
  using Loop = TileLoop<T, 3, A_RC, B_RC, Epi>;
  __shared__ __attribute__((aligned(1024))) char ah[T::ABYTES], am[T::ABYTES], al[T::ABYTES];
  __shared__ __attribute__((aligned(1024))) char bh0[T::BBYTES], bh1[T::BBYTES], bm0[T::BBYTES], bm1[T::BBYTES], bl[T::BBYTES];
  vacc_t acc[IP][IQ];
  const Loop l(pr, t, acc, lane, wave);
  vbf16x8_t a[2][IP], b[2][IQ];

  // Stage c in ah, am, al, bh, bm, bl; the next one's in bhn, bmn and the others.
  auto stage = [&](char* bh, char* bhn, char* bm, char* bmn, int c) __attribute__((always_inline)) {
    each(std::make_integer_sequence<int, 12>{}, [&](auto S_) __attribute__((always_inline)) {
      constexpr int s = decltype(S_)::value, f = s / 2, k = s % 2, s1 = (s + 1) % 12, f1 = s1 / 2;
      // loads landed by the barriers of phases 5 (B high', A high'), 0 (B middle), 1 (B low), 2 (A middle) and 4 (A
      // low): all but those of the two phases before
      constexpr int left[6] = {NB + NA, NA + NA, NA + NB, NB + NA, NA + NB, NB + NB};
      if constexpr (k == 1) Loop::template sync<left[f]>();
      constexpr bool next_a = s1 < 2 || s1 == 6 || s1 == 7 || s1 >= 10;
      if constexpr (next_a) l.read_a(a[s1 % 2], f1 < 3 ? ah : f1 < 5 ? am : al, s1 % 2);
      l.read_b(b[s1 % 2], f1 == 2 ? bl : f1 == 1 || f1 == 4 ? bm : s == 11 ? bhn : bh, s1 % 2);
      // a phase's loads: the first behind its barrier, the rest in the next step
      constexpr int g = k == 1 ? f : (f + 5) % 6;   // whose
      constexpr bool first = k == 1, of_a = g == 0 || g == 2 || g == 5;
      if constexpr (g == 0) l.template load_a<first ? 0 : A1, first ? A1 : NA>(al, c, 2);
      if constexpr (g == 1) l.template load_b<first ? 0 : B1, first ? B1 : NB>(bhn, c + 1, 0);
      if constexpr (g == 2) l.template load_a<first ? 0 : A1, first ? A1 : NA>(ah, c + 1, 0);
      if constexpr (g == 3) l.template load_b<first ? 0 : B1, first ? B1 : NB>(bmn, c + 1, 1);
      if constexpr (g == 4) l.template load_b<first ? 0 : B1, first ? B1 : NB>(bl, c + 1, 2);
      if constexpr (g == 5) l.template load_a<first ? 0 : A1, first ? A1 : NA>(am, first ? c + 1 : c, 1);
      l.mfma(a[k], b[k]);
      Loop::template sched<(next_a ? Loop::READA : 0) + Loop::READB, of_a ? (first ? A1 : NA - A1) : (first ? B1 : NB - B1)>();
    });
  };

  l.template load_b<0, NB>(bh0, 0, 0);
  l.template load_a<0, NA>(ah, 0, 0);
  l.template load_b<0, NB>(bm0, 0, 1);
  l.template load_b<0, NB>(bl, 0, 2);
  l.template load_a<0, A1>(am, 0, 1);
  Loop::template sync<NB + NB + A1>();
  l.read_a(a[0], ah, 0);
  l.read_b(b[0], bh0, 0);
  __builtin_amdgcn_sched_barrier(0);
  for (int c = 0; c < l.nst; c += 2) {
    stage(bh0, bh1, bm0, bm1, c);
    stage(bh1, bh0, bm1, bm0, c + 1);
  }
  Loop::template sync<0>();
  const Ring ring{{lds_address(ah), lds_address(am), lds_address(al), lds_address(bh0), lds_address(bh1), lds_address(bm0),
                   lds_address(bm1), lds_address(bl)}};
  e(t, acc, ring, lane, wave, l.wp, l.wq);
}

template <class T, int PL, bool A_RC, bool B_RC, class Epi>
__global__ __launch_bounds__(T::NT, T::OCC) void tile_kernel(TileProblem pr, Epi e) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  TilePlace t;
  if (!tile_place<T>(pr, Epi::ROWS, &t)) return;
  if constexpr (PL == 1) tile_body1<T, A_RC, B_RC>(pr, t, e, lane, wave);
  else tile_body3<T, A_RC, B_RC>(pr, t, e, lane, wave);
}

// Part i of the ring, BYTES each, of at least COUNT.
template <class T, int PL, int BYTES, int COUNT>
__device__ __forceinline__ char* ring_part(const Ring& ring, int i) {
  constexpr int EACH = kRingBytes<T, PL> / BYTES;
  static_assert(EACH * kRingArrays<T, PL> >= COUNT, "parts of the ring");
  uint32_t a = ring.at[0];
  if constexpr (COUNT > EACH) {
#pragma unroll
    for (int r = 1; r < kRingArrays<T, PL>; ++r) a = i / EACH == r ? ring.at[r] : a;
  }
  return (char*)(lds_char*)(uintptr_t)(a + (uint32_t)(i % EACH) * BYTES);
}

}  // namespace opfuse
