// Rows to microscaled 4-bit floating point: a thread's 16 elements, a block's scale, eight numbers to a word.  (The formats and the
// definition stand at the head of e2m1.cu.)
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace luqdev {

constexpr int kChunk = 16;                 // elements of a thread
constexpr int kScaleTile = 512;

// The words of a thread's 16 elements, zeros beyond the row's end.  Where they do not lie in whole aligned pieces of 16 bytes they
// are put together from the pieces that hold an element of theirs.
template <typename T> constexpr int kWords = kChunk * static_cast<int>(sizeof(T)) / 4;
template <typename T>
__device__ __forceinline__ void load_chunk16(const T* row, int c0, int cols, bool vec, uint32_t (&w)[kWords<T>]) {
  constexpr int W = kWords<T>;
  if (vec && c0 + kChunk <= cols) {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const uint4 u = reinterpret_cast<const uint4*>(row + c0)[i];
      w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
    }
    return;
  }
  if (c0 >= cols) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0u;
    return;
  }
  const uintptr_t at = reinterpret_cast<uintptr_t>(row + c0), end = reinterpret_cast<uintptr_t>(row + min(c0 + kChunk, cols));
  const uintptr_t low = at & ~static_cast<uintptr_t>(15);
  const int shift = static_cast<int>(at & 15u);
  uint32_t v[W + 4];
#pragma unroll
  for (int i = 0; i <= W / 4; ++i) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (low + 16 * i < end) u = *reinterpret_cast<const uint4*>(low + 16 * i);
    v[4 * i] = u.x; v[4 * i + 1] = u.y; v[4 * i + 2] = u.z; v[4 * i + 3] = u.w;
  }
  if (shift & 8) {
#pragma unroll
    for (int i = 0; i < W + 2; ++i) v[i] = v[i + 2];
  }
  if (shift & 4) {
#pragma unroll
    for (int i = 0; i < W + 1; ++i) v[i] = v[i + 1];
  }
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = sizeof(T) == 4 ? v[i] : __funnelshift_r(v[i], v[i + 1], 8 * (shift & 2));
  if (c0 + kChunk > cols) {
#pragma unroll
    for (int i = 0; i < kChunk; ++i)
      if (c0 + i >= cols) {
        if constexpr (sizeof(T) == 4) w[i] = 0u;
        else w[i / 2] &= i & 1 ? 0x0000FFFFu : 0xFFFF0000u;
      }
  }
}
// the largest pattern of |x|, as a binary32 one: of numbers the largest, Inf above every number, NaN above Inf
template <typename T>
__device__ __forceinline__ uint32_t top_of(const uint32_t (&w)[kWords<T>]) {
  uint32_t t = 0;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < kWords<T>; ++i) t = max(t, w[i] & 0x7FFFFFFFu);
    return t;
  } else {
#pragma unroll
    for (int i = 0; i < kWords<T>; ++i) asm("max.u16x2 %0, %0, %1;" : "+r"(t) : "r"(w[i] & 0x7FFF7FFFu));
    return max(t << 16, t & 0xFFFF0000u);
  }
}
template <typename T>
__device__ __forceinline__ float2 pair_of(const uint32_t (&w)[kWords<T>], int i) {
  if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
  else return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
// eight numbers from pairs `first` .. `first` + 3, the first in the lowest four bits
template <typename T>
__device__ __forceinline__ uint32_t pack8(const uint32_t (&w)[kWords<T>], int first, float f) {
  float2 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __fmul2_rn(pair_of<T>(w, first + i), make_float2(f, f));
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0].x), "f"(v[0].y), "f"(v[1].x), "f"(v[1].y), "f"(v[2].x), "f"(v[2].y), "f"(v[3].x), "f"(v[3].y));
  return r;
}
// the e4m3 number nearest to v >= 0 (at most 448), and its value
__device__ __forceinline__ uint32_t to_e4m3(float v, float& value) {
  uint16_t b;
  uint32_t h;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(0.0f), "f"(v));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(b));
  asm("{\n\t.reg .f16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.f32.f16 %0, lo;\n\t}" : "=f"(value) : "r"(h));
  return b & 0xFFu;
}

// What a row's elements are made of: the row's scale and six times it (blocks of 16), and whether it has numbers at all
struct RowScale {
  float g, six;
  bool dead;             // Inf or NaN, or nothing to scale by: zero codes
};
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  RowScale s;
  s.dead = top >= 0x7F800000u || top < 0x0D800000u;                 // 2^-100
  s.g = s.dead ? (top >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : 0.0f) : __fdiv_rn(__uint_as_float(top), 2688.0f);
  s.six = __fmul_rn(s.g, 6.0f);
  return s;
}
// a block's scale byte and the factor of its elements
template <int BLOCK>
__device__ __forceinline__ uint32_t block_scale(uint32_t top, const RowScale& row, float& factor) {
  if constexpr (BLOCK == 16) {
    factor = 0.0f;
    if (row.dead) return 0u;
    float s;
    const uint32_t byte = to_e4m3(__fdiv_rn(__uint_as_float(top), row.six), s);
    if (s > 0.0f) factor = __frcp_rn(__fmul_rn(s, row.g));
    return byte;
  } else {
    if (top >= 0x7F800000u) { factor = 0.0f; return 255u; }
    const uint32_t byte = max(static_cast<int>(top >> 23) - 2, 0);
    factor = __uint_as_float((254u - byte) << 23);
    return byte;
  }
}

// A chunk in registers -> its codes and scale byte
template <typename T, int BLOCK>
__device__ __forceinline__ void quantize_chunk(const uint32_t (&w)[kWords<T>], uint32_t top, const RowScale& row, uint2& codes, uint32_t& byte) {
  float f;
  byte = block_scale<BLOCK>(top, row, f);
  // (a factor of zero would leave NaN where there is Inf)
  codes = f > 0.0f ? make_uint2(pack8<T>(w, 0, f), pack8<T>(w, 4, f)) : make_uint2(0u, 0u);
}

}  // namespace luqdev
