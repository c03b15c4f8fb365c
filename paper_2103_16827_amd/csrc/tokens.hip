// The quantiser with a scale per row (Eq. 1 with the row's own clipping range): one workgroup a row, a pass for the largest
// finite magnitude and a pass that rounds (the row is in the caches by then).
#include "floats.hpp"
#include "kernels.hpp"
#include "launch_shape.hpp"

namespace qasr {
namespace {

__device__ __forceinline__ int32_t code_of(float v, float S) {
  const float t = __fdiv_rn(v, S);
  return t != t ? 0 : (int32_t)rintf(fminf(127.0f, fmaxf(-127.0f, t)));
}

__device__ __forceinline__ float scale_of(float a) { return a > 0.0f ? fmaxf(__fdiv_rn(a, 127.0f), 0x1p-126f) : 1.0f; }

template <typename T>
__global__ __launch_bounds__(256) void quantize_tokens_kernel(const T* __restrict__ x, int64_t M, int K, int64_t xs,
                                                              int8_t* __restrict__ q, int64_t qs, float* __restrict__ scale) {
  __shared__ float part[4];
  const int64_t m = ((int64_t)blockIdx.y << kGridShift) + blockIdx.x;
  if (m >= M) return;
  const T* row = x + m * xs;
  float a = 0.0f;
  for (int k = threadIdx.x; k < K; k += 256) {
    const float v = fabsf(to_float(row[k]));
    a = v < __builtin_inff() ? fmaxf(a, v) : a;
  }
  for (int d = 32; d > 0; d >>= 1) a = fmaxf(a, __shfl_xor(a, d));
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = a;
  __syncthreads();
  const float S = scale_of(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
  if (threadIdx.x == 0) scale[m] = S;
  for (int k = threadIdx.x; k < K; k += 256) q[m * qs + k] = (int8_t)code_of(to_float(row[k]), S);
}

}  // namespace

hipError_t launch_quantize_tokens(const void* x, int x_type, int64_t M, int K, int64_t x_stride, int8_t* q, int64_t q_stride,
                                  float* scale, hipStream_t st) {
  const GridShape g = grid_shape(M);
  return with_type(x_type, [&](auto t) {
    using T = decltype(t);
    return launch_kernel(quantize_tokens_kernel<T>, dim3(g.x, g.y), dim3(256), 0, st, (const T*)x, M, K, x_stride, q, q_stride, scale);
  });
}

}  // namespace qasr
