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
// Two fp32 additions in one instruction.
__device__ __forceinline__ void add2(float& a, float& b, float x, float y) {
  asm("{ .reg .b64 p, q;\n\t"
      "mov.b64 p, {%0, %1};\n\t"
      "mov.b64 q, {%2, %3};\n\t"
      "add.rn.f32x2 p, p, q;\n\t"
      "mov.b64 {%0, %1}, p; }" : "+f"(a), "+f"(b) : "f"(x), "f"(y));
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
