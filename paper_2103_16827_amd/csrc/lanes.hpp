// Reductions over the 64 lanes of a wave.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace qasr {

// Reductions over the lanes, by moves among them that are part of the operation (a shuffle through LDS costs a round trip each):
// within rows of 16, then across them.  The result is in every lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lane_move(uint32_t keep, uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)keep, (int)v, CTRL, ROWS, 0xf, false);
}
// every lane's v with those of the lanes before it
template <typename V, typename Op>
__device__ __forceinline__ V wave_scan(V v, V none, Op op) {
  auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
    constexpr int C = decltype(ctrl)::value, R = decltype(rows)::value;
    if constexpr (sizeof(V) == 8) {
      const uint64_t n = __builtin_bit_cast(uint64_t, none), b = __builtin_bit_cast(uint64_t, v);
      const uint64_t o = (uint64_t)lane_move<C, R>((uint32_t)(n >> 32), (uint32_t)(b >> 32)) << 32 | lane_move<C, R>((uint32_t)n, (uint32_t)b);
      v = op(v, __builtin_bit_cast(V, o));
    } else {
      v = op(v, __builtin_bit_cast(V, lane_move<C, R>(__builtin_bit_cast(uint32_t, none), __builtin_bit_cast(uint32_t, v))));
    }
  };
  using std::integral_constant;
  step(integral_constant<int, 0x111>(), integral_constant<int, 0xf>());      // from the lanes 1, 2, 4, 8 before it in its row of 16
  step(integral_constant<int, 0x112>(), integral_constant<int, 0xf>());
  step(integral_constant<int, 0x114>(), integral_constant<int, 0xf>());
  step(integral_constant<int, 0x118>(), integral_constant<int, 0xf>());
  step(integral_constant<int, 0x142>(), integral_constant<int, 0xa>());      // the last of a row to the row after it (rows 1 and 3)
  step(integral_constant<int, 0x143>(), integral_constant<int, 0xc>());      // the last of the second row to the third and fourth
  return v;
}
template <typename V, typename Op>
__device__ __forceinline__ V wave_reduce(V v, V none, Op op) {
  v = wave_scan(v, none, op);
  if constexpr (sizeof(V) == 8) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(V, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), 63) << 32 |
                                     (uint32_t)__builtin_amdgcn_readlane((int)b, 63));
  } else {
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
  }
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_reduce(v, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_reduce(v, 0.0f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  return wave_reduce(v, (uint64_t)0, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint32_t wave_min(uint32_t v) {
  return wave_reduce(v, ~0u, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}

}  // namespace qasr
