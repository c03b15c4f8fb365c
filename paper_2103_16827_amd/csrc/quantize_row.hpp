// The arithmetic of the quantiser with a scale per row: S = max|x| / 127 over finite x, codes Int(x / S).
#pragma once
#include "floats.hpp"

namespace qasr {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef unsigned short v2us __attribute__((ext_vector_type(2)));

template <typename T>
constexpr int kPer = 16 / (int)sizeof(T);              // elements per 16 bytes

// Magnitudes as unsigned numbers in the type's own bits: what is kInf or above is no finite number.
template <typename T>
constexpr uint32_t kInf = sizeof(T) == 4 ? 0x7f800000u : __is_same(T, bf16) ? 0x7f80u : 0x7c00u;
template <typename T>
__device__ __forceinline__ uint32_t bits_of(T v) {
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(uint32_t, v);
  else return __builtin_bit_cast(uint16_t, v);
}
template <typename T>
__device__ __forceinline__ float magnitude(uint32_t bits) {
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, bits);
  else return to_float(__builtin_bit_cast(T, (uint16_t)bits));
}
template <typename T>
__device__ __forceinline__ uint32_t sign_off(uint32_t word) { return word & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu); }
template <typename T>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {        // of a word's numbers
  if constexpr (sizeof(T) == 4) return a > b ? a : b;
  else return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2us, a), __builtin_bit_cast(v2us, b)));
}
template <typename T>
__device__ __forceinline__ uint32_t largest_of(uint32_t word) {
  if constexpr (sizeof(T) == 4) return word;
  else return (word & 0xffffu) > word >> 16 ? word & 0xffffu : word >> 16;
}
template <typename T>
__device__ __forceinline__ float element(const v4u& v, int e) {
  const uint32_t word = v[sizeof(T) == 4 ? e : e >> 1];
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, word);
  else return to_float(__builtin_bit_cast(T, (uint16_t)(e & 1 ? word >> 16 : word)));
}

__device__ __forceinline__ float scale_of(float a) { return a > 0.0f ? fmaxf(__fdiv_rn(a, 127.0f), 0x1p-126f) : 1.0f; }
// (the conversion saturates, and makes 0 of a NaN: what is clipped here is what the definition clips before it rounds)
__device__ __forceinline__ int32_t code_of(float v, float S) {
  int32_t q;
  asm("v_cvt_i32_f32 %0, %1" : "=v"(q) : "v"(rintf(__fdiv_rn(v, S))));
  return min(127, max(-127, q));
}

// four codes in a word
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d, float S) {
  return __builtin_amdgcn_perm((uint32_t)code_of(b, S), (uint32_t)code_of(a, S), 0x0c0c0400u) |
         __builtin_amdgcn_perm((uint32_t)code_of(d, S), (uint32_t)code_of(c, S), 0x04000c0cu);
}

}  // namespace qasr
