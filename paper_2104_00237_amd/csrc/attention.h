// Device helpers shared by the attention kernels: which rows a workgroup works on, LDS tiles and
// their fragments, loads and stores of head rows.
//
// All products run on 32x32 MFMA tiles whose *columns* (lane % 32) are the rows a wavefront owns
// (queries in the forward and for dQ, keys for dK and dV) and whose rows (registers) are the rows
// that stream by.  A register k of lane half h = lane / 32 holds streamed row 8 (k/4) + 4 h + k % 4:
//   - row statistics of an owned row are sums over one lane's registers and its other half's;
//   - exp(S) is already the B operand of the next product, whose contraction runs over the streamed
//     rows: the order of a contraction is free, so the A operand (the streamed tile, transposed) is
//     read in the registers' order and the probabilities never go through LDS.
#pragma once

#include <type_traits>
#include <utility>

#include "attention_seq.h"
#include "gemm_common.h"

namespace opfuse {

typedef __bf16 abf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 abf16x2_t __attribute__((ext_vector_type(2)));
typedef float afloat2_t __attribute__((ext_vector_type(2)));
typedef float afloatx4_t __attribute__((ext_vector_type(4)));
typedef float acc16_t __attribute__((ext_vector_type(16)));
typedef short ashort4_t __attribute__((ext_vector_type(4)));
typedef short ashort8_t __attribute__((ext_vector_type(8)));
typedef uint32_t au32x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// ------------------------------------------------------------------- tiles
// A tile in LDS: rows of 16-byte slots (a power of two of them), slot s of row x at slot
// s ^ swz(x).  Rows are read as fragments (16 bytes of 32 rows at one slot: 16 consecutive rows take
// all 64 banks) and transposed (four consecutive rows of one 64-byte block, again all banks), so the
// two low bits of x go to the block bits of the slot and the next two below them.
// 16-byte slots of a row of `bytes` (a power of two, at least 8).
constexpr int slots_of(int bytes) {
  int s = 8;
  while (s * 16 < bytes) s *= 2;
  return s;
}
template <int SLOTS>
__device__ __forceinline__ int swz(int x) {
  if constexpr (SLOTS == 8) return (((x >> 1) & 1) << 2) | ((x >> 2) & 3);   // two rows take the banks
  return ((x & 3) << 2) | ((x >> 2) & 3);
}

template <typename T>
struct Mma;

template <>
struct Mma<uint16_t> {   // bf16 operands, v_mfma_f32_32x32x16_bf16
  static constexpr int E = 8;     // elements of a 16-byte slot
  static constexpr int TR = 16;   // streamed rows of one transposed fragment
  typedef abf16x8_t frag;
  static __device__ __forceinline__ acc16_t mma(frag a, frag b, acc16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ frag zero() { return __builtin_bit_cast(frag, au32x4_t{0, 0, 0, 0}); }
  // probabilities u: registers 8u .. 8u + 7, rounded to nearest even (an MFMA operand)
  static __device__ __forceinline__ frag pack(const acc16_t& s, int u) {
    au32x4_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const afloat2_t v = {s[8 * u + 2 * i], s[8 * u + 2 * i + 1]};
      r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, abf16x2_t));
    }
    return __builtin_bit_cast(frag, r);
  }
  // rows r0 .. r0 + 15 of columns x0 .. x0 + 31, transposed: lane: column x0 + lane % 32, rows
  // 4 h + j and 8 + 4 h + j
  template <int SLOTS>
  static __device__ __forceinline__ frag tr(const char* t, int r0, int x0, int lane) {
    const int r = r0 + (lane >> 5) * 4 + ((lane & 15) >> 2);
    const int x = x0 + (lane & 16) + (lane & 3) * 4;
    typedef __attribute__((address_space(3))) ashort4_t* lp;
    const char* a = t + r * (SLOTS * 16) + (((x >> 3) ^ swz<SLOTS>(r)) << 4) + (x & 4) * 2;
    const char* b = t + (r + 8) * (SLOTS * 16) + (((x >> 3) ^ swz<SLOTS>(r + 8)) << 4) + (x & 4) * 2;
    const ashort4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)a);
    const ashort4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)b);
    return __builtin_bit_cast(frag, (ashort8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  static __device__ __forceinline__ uint16_t from(float f) { return f32_to_bf16(f); }
  static __device__ __forceinline__ float to(uint16_t u) { return __uint_as_float((uint32_t)u << 16); }
};

template <>
struct Mma<float> {   // fp32 operands, v_mfma_f32_32x32x2_f32: four of them make one fragment's step
  static constexpr int E = 4;
  static constexpr int TR = 8;
  typedef afloatx4_t frag;
  static __device__ __forceinline__ acc16_t mma(frag a, frag b, acc16_t c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ frag zero() { return frag{0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ frag pack(const acc16_t& s, int u) {
    return frag{s[4 * u], s[4 * u + 1], s[4 * u + 2], s[4 * u + 3]};
  }
  template <int SLOTS>
  static __device__ __forceinline__ frag tr(const char* t, int r0, int x0, int lane) {
    const int x = x0 + (lane & 31);
    frag f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = r0 + (lane >> 5) * 4 + j;
      f[j] = *reinterpret_cast<const float*>(t + r * (SLOTS * 16) + (((x >> 2) ^ swz<SLOTS>(r)) << 4) + (x & 3) * 4);
    }
    return f;
  }
  static __device__ __forceinline__ float from(float f) { return f; }
  static __device__ __forceinline__ float to(float f) { return f; }
};

// 16 bytes of row x0 + lane % 32 for contraction step s (slot 2 s + h)
template <typename T, int SLOTS>
__device__ __forceinline__ typename Mma<T>::frag row_frag(const char* t, int x0, int s, int lane) {
  const int x = x0 + (lane & 31);
  return *reinterpret_cast<const typename Mma<T>::frag*>(t + x * (SLOTS * 16) + (((2 * s + (lane >> 5)) ^ swz<SLOTS>(x)) << 4));
}

// 16 bytes a lane from memory to LDS, lane i to `lds` + 16 i.  (A function of its own, no template: in
// the host pass the builtin has no 16-byte form, and a template that calls it is given up silently,
// with the kernels that use it.)
__device__ __forceinline__ void load_lds16(rsrc_t rs, char* lds, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)lds, 16, off, 0, 0, 0);
}

// Loads of a tile's rows: rows row0 .. row0 + n - 1 (n <= ROWS) of one head; the rest of the tile is
// zero, and so are columns from D on.  NT threads.
// VEC (pointer and strides are multiples of 16 bytes and D of a slot): memory to LDS, 16 bytes a lane
// and no registers.  A wavefront's load writes 1 KB in lane order, so the swizzle is applied to the
// address a lane loads from; the offsets are the same for every tile.  Else element by element.
template <typename T, int SLOTS, int ROWS, int NT, bool VEC>
struct TileLoad {
  static constexpr int E = Mma<T>::E, ES = sizeof(T), PER = ROWS * SLOTS / NT;
  static_assert(PER * NT == ROWS * SLOTS, "whole slots per thread");
  // the swizzle repeats every 16 rows: load i is load i % OFFS, some whole 16 rows further
  static constexpr int OFFS = PER < 16 * SLOTS / NT ? PER : 16 * SLOTS / NT > 0 ? 16 * SLOTS / NT : 1;
  static constexpr int FURTHER = OFFS * NT / SLOTS;   // rows
  uint32_t off[OFFS];
  uint32_t step;

  __device__ __forceinline__ TileLoad(const HeadRows& x, int D, int tid) {
    step = (uint32_t)(x.ld * FURTHER * ES);
#pragma unroll
    for (int i = 0; i < OFFS; ++i) {
      const int id = tid + i * NT, r = id / SLOTS, s = (id % SLOTS) ^ swz<SLOTS>(r);
      off[i] = s * E < D ? (uint32_t)(r * x.ld * ES) + s * 16 : kOOB;
    }
  }
  __device__ __forceinline__ void operator()(char* tile, const HeadRows& x, int64_t row0, int head, int n, int D, int tid) const {
    n = min(n, ROWS);   // none: an empty buffer, all zeros
    // (rows from n on lie beyond the buffer's end: ld >= D.  The end is checked against the vector
    // offset, so the whole offset is in it.)
    const rsrc_t rs = make_rsrc((const T*)x.p + row0 * x.ld + head * x.hs, n > 0 ? (int)(((n - 1) * x.ld + D) * ES) : 0);
    if constexpr (VEC) {
      const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
      for (int i = 0; i < PER; ++i)
        load_lds16(rs, tile + (wave * 64 + i * NT) * 16, off[i % OFFS] + (i / OFFS) * step);
    } else {
      au32x4_t v[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int id = tid + i * NT, r = id / SLOTS, d = ((id % SLOTS) ^ swz<SLOTS>(r)) * E;
        const uint32_t at = off[i % OFFS] + (i / OFFS) * step;
        if constexpr (ES == 4) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            v[i][e] = __builtin_amdgcn_raw_buffer_load_b32(rs, d + e < D ? at + 4 * e : kOOB, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            const uint32_t lo = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, d + e < D ? at + 2 * e : kOOB, 0, 0);
            const uint32_t hi = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, d + e + 1 < D ? at + 2 * e + 2 : kOOB, 0, 0);
            v[i][e / 2] = lo | hi << 16;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) *reinterpret_cast<au32x4_t*>(tile + (tid + i * NT) * 16) = v[i];
    }
  }
};

// This wavefront's loads to LDS and LDS accesses are done, then everyone's.
__device__ __forceinline__ void tile_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// The lane's own row as B fragments: 16 bytes at slot 2 s + h for step s.
template <typename T, bool VEC>
__device__ __forceinline__ typename Mma<T>::frag own_frag(const T* row, bool has, int s, int D, int lane) {
  constexpr int E = Mma<T>::E;
  const int d = (2 * s + (lane >> 5)) * E;
  typename Mma<T>::frag f = Mma<T>::zero();
  if constexpr (VEC) {
    if (has && d < D) f = *reinterpret_cast<const typename Mma<T>::frag*>(row + d);
  } else {
    T t[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      t[e] = 0;
      if (has && d + e < D) t[e] = row[d + e];
    }
    f = __builtin_bit_cast(typename Mma<T>::frag, t);
  }
  return f;
}
template <typename T, int NS, bool VEC>
__device__ __forceinline__ void load_own(typename Mma<T>::frag (&f)[NS], const T* row, bool has, int D, int lane) {
#pragma unroll
  for (int s = 0; s < NS; ++s) f[s] = own_frag<T, VEC>(row, has, s, D, lane);
}
// Own rows stay in registers, but for wide fp32 rows, which do not fit beside the sums: those are
// loaded again (from the caches) OD steps before each use, whose four MFMAs take 256 cycles.
template <typename T, int DP>
constexpr bool kKeepOwn = sizeof(T) == 2 || DP <= 128;
constexpr int OD = 4;

// A lane number, with FRESH one that the compiler knows nothing of: a fragment's LDS addresses are then
// computed where it is read instead of held in registers by the dozen.  For the kernels that spill
// most otherwise (forward, fp32, width 256: 903 -> 409 us; backward 4275 -> 2006); elsewhere it
// costs (forward, fp32, width 128: 163 -> 207 us; bf16, 256: 67 -> 95).  Registers that spill all the same:
// forward 17 (bf16, 256), 36 (fp32, 192), 11 (bf16, 128, not VEC); dQ 50 (bf16, 256) and 355 with fp32
// gradients (733 and 829 us traced: 4096 tokens, 16/4 heads), not VEC 24 (fp32, 256), 26 and 134 (bf16, 256), 61 (bf16, 128).
template <bool FRESH>
__device__ __forceinline__ int fresh(int lane) {
  if constexpr (FRESH) asm volatile("" : "+v"(lane));
  return lane;
}

// Accumulators [d, own row] times f, stored to the lane's row.
template <typename T, int NB>
__device__ __forceinline__ void store_own(T* row, const acc16_t (&acc)[NB], float f, int D, bool vec, int lane) {
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = b * 32 + g * 8 + (lane >> 5) * 4;
      float4 v = make_float4(acc[b][4 * g] * f, acc[b][4 * g + 1] * f, acc[b][4 * g + 2] * f, acc[b][4 * g + 3] * f);
      if (vec && d + 3 < D) {
        if constexpr (sizeof(T) == 4) st4((float*)row + d, v);
        else st_bf16x4((uint16_t*)row + d, v);
      } else {
        const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (d + j < D) row[d + j] = Mma<T>::from(e[j]);
      }
    }
}

// f(0) .. f(N - 1) with constants: registers are indexed statically.
template <int... I, class F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F&& f) {
  each_of(std::make_integer_sequence<int, N>{}, f);
}

template <int N>
__device__ __forceinline__ void zero_acc(acc16_t (&a)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int k = 0; k < 16; ++k) a[i][k] = 0.f;
}

// f of a lane's value and the other half's of the same column.
template <class F>
__device__ __forceinline__ float with_half(float x, F&& f) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  return with_half(x, [](float a, float b) { return a + b; });
}

// v_maximum3_f32: a NaN stays (fmaxf would drop it, and takes an instruction more for each operand
// to make it canonical first)
__device__ __forceinline__ float maxi(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace opfuse
