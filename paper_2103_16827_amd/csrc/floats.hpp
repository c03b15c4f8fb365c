// Float element types of the language-model operators' tensors, as the ABI numbers them (QASR_F32, _F16, _BF16).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qasr {

struct bf16 { uint16_t bits; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(_Float16 v) { return (float)v; }
__device__ __forceinline__ float to_float(bf16 v) { return __builtin_bit_cast(float, (uint32_t)v.bits << 16); }

// to nearest, ties to even
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ _Float16 from_float<_Float16>(float v) { return (_Float16)v; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float v) { return bf16{__builtin_bit_cast(uint16_t, (__bf16)v)}; }

// calls f(T()) with the type that `type` names
template <typename F>
inline auto with_type(int type, F f) {
  if (type == 0) return f(float());
  if (type == 1) return f(_Float16());
  return f(bf16());
}

}  // namespace qasr
