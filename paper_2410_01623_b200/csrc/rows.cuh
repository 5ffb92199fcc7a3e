// Pieces of a row as fp32 registers, by 16-byte accesses on 16-byte boundaries, wherever the row begins.
#pragma once
#include "common.cuh"

namespace fira {
namespace rows {

template <typename T>
constexpr int PER16 = 16 / (int)sizeof(T);      // elements of a 16-byte access

// The elements of 16 bytes.
template <typename T>
__device__ __forceinline__ void unpack(const uint4& u, float* v) {
  const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (sizeof(T) == 4) {
      v[k] = __uint_as_float(w[k]);
    } else {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  }
}
// Two fp32 operations in one instruction, each rounded like the single one.
__device__ __forceinline__ unsigned long long bits2(float2 v) { return *reinterpret_cast<const unsigned long long*>(&v); }
__device__ __forceinline__ float2 from_bits2(unsigned long long b) { return *reinterpret_cast<const float2*>(&b); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)));
  return from_bits2(d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)));
  return from_bits2(d);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
  return from_bits2(d);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// The elements of 16 bytes in pairs, and back (rounded).
template <typename T>
__device__ __forceinline__ void unpack(const uint4& u, float2 (&v)[PER16<T> / 2]) { unpack<T>(u, &v[0].x); }
template <typename T>
__device__ __forceinline__ uint4 pack(const float2 (&v)[PER16<T> / 2]) {
  unsigned w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (sizeof(T) == 4) {
      w[k] = __float_as_uint(k & 1 ? v[k / 2].y : v[k / 2].x);
    } else {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[k].x, v[k].y);
      w[k] = *reinterpret_cast<const unsigned*>(&h);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T, int N>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[N]) {
  static_assert(N % PER16<T> == 0, "whole 16-byte accesses");
#pragma unroll
  for (int i = 0; i < N / PER16<T>; ++i) unpack<T>(reinterpret_cast<const uint4*>(p)[i], v + i * PER16<T>);
}
template <typename T, int N>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N * (int)sizeof(T) / 16; ++i) {
    unsigned w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4) {
        w[k] = __float_as_uint(v[4 * i + k]);
      } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[8 * i + 2 * k], v[8 * i + 2 * k + 1]);
        w[k] = *reinterpret_cast<const unsigned*>(&h);
      }
    }
    reinterpret_cast<uint4*>(p)[i] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// The 16 bytes that begin `skip` bytes behind the start of a, the last ones from b (0 <= skip < 16, the same in all lanes or not).
__device__ __forceinline__ uint4 funnel16(const uint4& a, const uint4& b, int skip) {
  unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (skip & 8) {
#pragma unroll
    for (int k = 0; k < 6; ++k) w[k] = w[k + 2];
  }
  if (skip & 4) {
#pragma unroll
    for (int k = 0; k < 5; ++k) w[k] = w[k + 1];
  }
  const int bits = (skip & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}
// 16 bytes to `p`, which lies on a 16-byte boundary: those of its elements whose column, the first one being `col`, is in lo .. hi-1.
template <typename T>
__device__ __forceinline__ void store_between(T* p, const uint4& u, int col, int lo, int hi) {
  constexpr int N = PER16<T>;
  if (col >= lo && col + N <= hi) {
    *reinterpret_cast<uint4*>(p) = u;
  } else {
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (col + e >= lo && col + e < hi) {
        if constexpr (sizeof(T) == 4) reinterpret_cast<unsigned*>(p)[e] = w[e];
        else reinterpret_cast<unsigned short*>(p)[e] = (unsigned short)(w[e / 2] >> (e & 1) * 16);
      }
  }
}

// Whether rows of `width` elements that are `ld` apart from p on can be read in 16-byte accesses of whole pieces.
inline bool aligned16(const void* p, long long ld, long long width, size_t size) {
  return ((uintptr_t)p & 15) == 0 && (ld * (long long)size) % 16 == 0 && (width * (long long)size) % 16 == 0;
}

}  // namespace rows
}  // namespace fira
