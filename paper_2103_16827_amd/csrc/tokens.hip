// The quantiser with a scale per row (Eq. 1 with the row's own clipping range): S = max|x| / 127 over finite x, codes Int(x / S).
//
// A row belongs to one workgroup, or to one wave where it is short, which reads it once into registers: the largest magnitude
// (as unsigned numbers, whose order is that of floats: two 16-bit ones at a time), then a correctly rounded division, a
// rounding and a conversion per element.  What bounds it is memory (3 to 5 bytes an element); the division's eleven
// instructions stay below that.  Rows longer than the registers are read twice.
#include "floats.hpp"
#include "kernels.hpp"
#include "lanes.hpp"
#include "launch_shape.hpp"

namespace qasr {
namespace {

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

// W waves a row, R loads of 16 bytes a lane from a 16-byte boundary on; what is before and behind them, an element for
// each of the first threads.  W == 1: four rows a workgroup, a wave each.
template <typename T, int W, int R>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void quantize_tokens_kernel(const T* __restrict__ x, int64_t M, int K, int64_t xs,
                                                                                int8_t* __restrict__ q, int64_t qs, float* __restrict__ scale) {
  constexpr int N = kPer<T>, kRows = W == 1 ? 4 : 1;
  __shared__ uint32_t part[2][W];
  const int tid = W == 1 ? threadIdx.x & 63 : threadIdx.x, lane = tid & 63;
  const int64_t m = (((int64_t)blockIdx.y << kGridShift) + blockIdx.x) * kRows + (W == 1 ? threadIdx.x >> 6 : 0);
  if (m >= M) return;                                  // (W == 1: no barriers below)
  const T* row = x + m * xs;
  const int head = min(K, (int)(-(uintptr_t)row & 15) / (int)sizeof(T));
  const int loads = (K - head) / N, rest = tid < head ? tid : loads * N + tid;
  const v4u* aligned = reinterpret_cast<const v4u*>(row + head);
  v4u raw[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    raw[i] = (v4u){0, 0, 0, 0};
    if (i * 64 * W + tid < loads) raw[i] = aligned[i * 64 * W + tid];
  }
  T last = from_float<T>(0.0f);
  if (rest < K) last = row[rest];

  // the row's largest number; finite: of those that are
  auto largest = [&](int turn, auto&& all) __attribute__((always_inline)) {
    uint32_t a = wave_max(all());
    if constexpr (W > 1) {
      if (lane == 0) part[turn][tid >> 6] = a;
      __syncthreads();
      a = wave_max(part[turn][lane % W]);
    }
    return a;
  };
  uint32_t a = largest(0, [&]() __attribute__((always_inline)) {
    uint32_t word = sign_off<T>(bits_of(last));
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) word = larger<T>(word, sign_off<T>(raw[i][k]));
    return largest_of<T>(word);
  });
  if (a >= kInf<T>)                                    // an infinity or a NaN somewhere (uniform)
    a = largest(1, [&]() __attribute__((always_inline)) {
      auto finite = [](uint32_t v) { return v < kInf<T> ? v : 0u; };
      uint32_t most = finite(sign_off<T>(bits_of(last)));
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t word = sign_off<T>(raw[i][k]);
          if constexpr (sizeof(T) == 4) most = max(most, finite(word));
          else most = max(most, max(finite(word & 0xffffu), finite(word >> 16)));
        }
      return most;
    });
  const float S = scale_of(magnitude<T>(a));
  if (tid == 0) scale[m] = S;
  int8_t* to = q + m * qs;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i * 64 * W + tid < loads) {
      struct __attribute__((packed)) { uint32_t word[N / 4]; } out;
#pragma unroll
      for (int w = 0; w < N / 4; ++w) {
        int32_t c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) c[k] = code_of(element<T>(raw[i], 4 * w + k), S);
        out.word[w] = __builtin_amdgcn_perm((uint32_t)c[1], (uint32_t)c[0], 0x0c0c0400u) | __builtin_amdgcn_perm((uint32_t)c[3], (uint32_t)c[2], 0x04000c0cu);
      }
      *reinterpret_cast<decltype(out)*>(to + head + (i * 64 * W + tid) * N) = out;
    }
  if (rest < K) to[rest] = (int8_t)code_of(to_float(last), S);
}

// rows of any length, read twice
template <typename T>
__global__ __launch_bounds__(1024) void quantize_long_kernel(const T* __restrict__ x, int64_t M, int K, int64_t xs, int8_t* __restrict__ q,
                                                             int64_t qs, float* __restrict__ scale) {
  __shared__ uint32_t part[16];
  const int64_t m = ((int64_t)blockIdx.y << kGridShift) + blockIdx.x;
  if (m >= M) return;
  const T* row = x + m * xs;
  uint32_t a = 0;
  for (int k = threadIdx.x; k < K; k += 1024) {
    const uint32_t v = sign_off<T>(bits_of(row[k]));
    a = v < kInf<T> && v > a ? v : a;
  }
  a = wave_max(a);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = a;
  __syncthreads();
  const float S = scale_of(magnitude<T>(wave_max(part[threadIdx.x % 16])));
  if (threadIdx.x == 0) scale[m] = S;
  for (int k = threadIdx.x; k < K; k += 1024) q[m * qs + k] = (int8_t)code_of(to_float(row[k]), S);
}

}  // namespace

hipError_t launch_quantize_tokens(const void* x, int x_type, int64_t M, int K, int64_t x_stride, int8_t* q, int64_t q_stride,
                                  float* scale, hipStream_t st) {
  return with_type(x_type, [&](auto t) {
    using T = decltype(t);
    const int loads = K / kPer<T>;
    auto launch = [&](auto kernel, int threads, int rows) {
      const GridShape g = grid_shape((M + rows - 1) / rows);
      return launch_kernel(kernel, dim3(g.x, g.y), dim3(threads), 0, st, (const T*)x, M, K, x_stride, q, q_stride, scale);
    };
    // A wave for a short row where there are enough of them for the chip, else the lanes that a load each of the row needs.
    if (loads <= 64) return launch(quantize_tokens_kernel<T, 1, 1>, 256, 4);
    if (loads <= 256 && M >= 2048) return launch(quantize_tokens_kernel<T, 1, 4>, 256, 4);
    if (loads <= 256) return launch(quantize_tokens_kernel<T, 4, 1>, 256, 1);
    if (loads <= 1024 && M >= 512) return launch(quantize_tokens_kernel<T, 4, 4>, 256, 1);
    if (loads <= 1024) return launch(quantize_tokens_kernel<T, 16, 1>, 1024, 1);
    if (loads <= 4096) return launch(quantize_tokens_kernel<T, 16, 4>, 1024, 1);
    return launch(quantize_long_kernel<T>, 1024, 1);
  });
}

}  // namespace qasr
