// Pieces of a row as fp32 registers: 16-byte accesses where rows start on 16-byte boundaries and their width is a
// multiple of the piece, single elements otherwise.
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

// Whether rows of `width` elements that are `ld` apart from p on can be read in 16-byte accesses of whole pieces.
inline bool aligned16(const void* p, long long ld, long long width, size_t size) {
  return ((uintptr_t)p & 15) == 0 && (ld * (long long)size) % 16 == 0 && (width * (long long)size) % 16 == 0;
}

}  // namespace rows
}  // namespace fira
