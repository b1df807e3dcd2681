// Rotary positions: pairs of a head's elements turned by an angle that grows with the row's position.
// Forward and backward are the same kernel; the backward turns the other way.
//
// Bound by memory: every element is read once and written once.  The angles of a row are the same
// for all its heads: a workgroup takes a few rows, puts their cosines and sines into LDS (position
// times frequency in float64, reduced to a part of a turn: a float32 angle at position 1e6 is off
// by 0.03; what the functions' float32 argument leaves out is added to their values), and then streams
// the heads with 16-byte accesses.
// Measured: 4096 rows, 32 heads of 64 in packed bf16 rows 8.6 us (3.9 TB/s with the launch; a large copy
// reaches 4.8); 16384 rows, 24 heads of 128 in fp32, half of each turned: 75 us (5.3 TB/s, part of it
// from the last-level cache).

#include <algorithm>

#include "common.h"

namespace opfuse {

constexpr int ROT_LDS = 2048;   // cosine / sine pairs of a workgroup

__device__ __forceinline__ float2 rotate(float u, float v, float2 cs) {
  return make_float2(__fsub_rn(__fmul_rn(u, cs.x), __fmul_rn(v, cs.y)),
                     __fmaf_rn(u, cs.y, __fmul_rn(v, cs.x)));
}

template <typename T>
struct Vec16;
template <>
struct Vec16<float> {
  static constexpr int N = 4;
  float v[4];
  __device__ __forceinline__ void load(const float* p) {
    const float4 x = ld4(p);
    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
  }
  __device__ __forceinline__ void store(float* p) const { st4(p, make_float4(v[0], v[1], v[2], v[3])); }
};
template <>
struct Vec16<uint16_t> {
  static constexpr int N = 8;
  float v[8];
  __device__ __forceinline__ void load(const uint16_t* p) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void store(uint16_t* p) const {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bf16(v[2 * i]) | (uint32_t)f32_to_bf16(v[2 * i + 1]) << 16;
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

__device__ __forceinline__ float ldf(const float* p) { return *p; }
__device__ __forceinline__ float ldf(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void stf(float* p, float v) { *p = v; }
__device__ __forceinline__ void stf(uint16_t* p, float v) { *p = f32_to_bf16(v); }

template <typename T, bool VEC, bool INTER>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  constexpr int V = VEC ? Vec16<T>::N : 1;
  __shared__ float2 cs[ROT_LDS];
  const int half = a.rot / 2;
  const int64_t t0 = (int64_t)blockIdx.x * a.rows;
  const int rows = (int)min((int64_t)a.rows, a.T - t0);
  for (int i = threadIdx.x; i < rows * half; i += 256) {
    const int r = i / half, k = i - r * half;
    const int64_t t = t0 + r;
    const double pos = a.pos ? (double)a.pos[t] : (double)(a.pos0 + t % a.seq_len);
    const double turns = pos * a.w[k];
    // half turns in [-1, 1], and what their rounding to fp32 leaves (at most pi 2^-25 = 1.6 half steps of 1,
    // as much as everything else in an element): to first order, its square is below 1e-14
    const double x = 2.0 * (turns - rint(turns));
    const float near = (float)x, rest = (float)(x - near) * 3.14159265f;
    float s, c;
    sincospif(near, &s, &c);
    // sign: +-mscale
    cs[i] = make_float2(__fmaf_rn(-s, rest, c) * a.mscale, __fmaf_rn(c, rest, s) * a.sign);
  }
  __syncthreads();
  // items of a head: turned pieces (V pairs in the half layout, V elements of neighbouring pairs,
  // or one pair), then pieces that pass through (none in place)
  const int turned = VEC ? (INTER ? a.rot / V : half / V) : half;
  const int per = turned + (a.copy ? (a.D - a.rot) / V : 0);
  const int n = rows * a.H * per;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int q = i / per, u = i - q * per, r = q / a.H, h = q - r * a.H;
    const T* x = (const T*)a.x + (t0 + r) * a.ldx + (int64_t)h * a.hsx;
    T* y = (T*)a.y + (t0 + r) * a.ldy + (int64_t)h * a.hsy;
    const float2* f = cs + r * half;
    if (u >= turned) {
      const int d = a.rot + (u - turned) * V;
      if constexpr (VEC) {
        *reinterpret_cast<uint4*>(y + d) = *reinterpret_cast<const uint4*>(x + d);
      } else {
        y[d] = x[d];
      }
    } else if constexpr (!VEC) {
      const int p = INTER ? 2 * u : u, p2 = INTER ? 2 * u + 1 : u + half;
      const float2 z = rotate(ldf(x + p), ldf(x + p2), f[u]);
      stf(y + p, z.x);
      stf(y + p2, z.y);
    } else if constexpr (INTER) {
      Vec16<T> v;
      v.load(x + u * V);
#pragma unroll
      for (int k = 0; k < V; k += 2) {
        const float2 z = rotate(v.v[k], v.v[k + 1], f[(u * V + k) / 2]);
        v.v[k] = z.x, v.v[k + 1] = z.y;
      }
      v.store(y + u * V);
    } else {
      Vec16<T> v, w;
      v.load(x + u * V);
      w.load(x + half + u * V);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float2 z = rotate(v.v[k], w.v[k], f[u * V + k]);
        v.v[k] = z.x, w.v[k] = z.y;
      }
      v.store(y + u * V);
      w.store(y + half + u * V);
    }
  }
}

bool rotary_rows(RotaryArgs& a, bool bf16) {
  const int V = bf16 ? 8 : 4, es = bf16 ? 2 : 4;
  auto lines = [&](const void* p, int64_t ld, int64_t hs) {
    return aligned16(p) && ld * es % 16 == 0 && hs * es % 16 == 0;
  };
  const bool vec = a.D % V == 0 && (a.interleaved ? a.rot : a.rot / 2) % V == 0 && lines(a.x, a.ldx, a.hsx) &&
                   lines(a.y, a.ldy, a.hsy);
  const int per = a.H * ((vec ? (a.interleaved ? a.rot : a.rot / 2) / V : a.rot / 2) + (a.D - a.rot) / (vec ? V : 1));
  a.rows = (int)std::max<int64_t>(1, std::min<int64_t>({8, ROT_LDS / (a.rot / 2), 1024 / std::max(per, 1)}));
  return vec;
}

hipError_t rotary_launch(const RotaryArgs& a, bool bf16, bool vec, hipStream_t stream) {
  const dim3 grid((unsigned)((a.T + a.rows - 1) / a.rows));
  auto go = [&](auto* kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
  if (bf16) {
    if (vec) go(a.interleaved ? rotary_kernel<uint16_t, true, true> : rotary_kernel<uint16_t, true, false>);
    else go(a.interleaved ? rotary_kernel<uint16_t, false, true> : rotary_kernel<uint16_t, false, false>);
  } else {
    if (vec) go(a.interleaved ? rotary_kernel<float, true, true> : rotary_kernel<float, true, false>);
    else go(a.interleaved ? rotary_kernel<float, false, true> : rotary_kernel<float, false, false>);
  }
  return hipGetLastError();
}

}  // namespace opfuse
