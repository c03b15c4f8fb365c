// The quantiser with a scale per row (Eq. 1 with the row's own clipping range): S = max|x| / 127 over finite x, codes Int(x / S).
//
// A row belongs to one workgroup, or to one wave where it is short, which reads it once into registers: the largest magnitude
// (as unsigned numbers, whose order is that of floats: two 16-bit ones at a time), then a correctly rounded division, a
// rounding and a conversion per element.  What bounds it is memory (3 to 5 bytes an element); the division's eleven
// instructions stay below that.  Rows longer than the registers are read twice.
// 8192 x 8192: bf16 41.5 us (4.8 TB/s), float32 60.6 (5.5); 16384 x 512 bf16 7.8; one token of 4096 2.4, most of it the launch.
// Codes stored past the caches would save 2 to 15 % here, and cost the layer that reads them next more (2000 x 2048 into 512
// channels: 22.9 us for both against 21.1).
#include "floats.hpp"
#include "kernels.hpp"
#include "lanes.hpp"
#include "launch_shape.hpp"
#include "quantize_row.hpp"

namespace qasr {
namespace {

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
      for (int w = 0; w < N / 4; ++w)
        out.word[w] = codes_of(element<T>(raw[i], 4 * w), element<T>(raw[i], 4 * w + 1), element<T>(raw[i], 4 * w + 2), element<T>(raw[i], 4 * w + 3), S);
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
