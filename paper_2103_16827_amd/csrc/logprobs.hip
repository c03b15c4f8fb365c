// Log probabilities of given tokens, the entropy and the top alternatives of rows of logits: one workgroup a row, a pass
// for the maximum, one for the sums, and one for each alternative.
#include "floats.hpp"
#include "kernels.hpp"
#include "launch_shape.hpp"

namespace qasr {
namespace {

// order of a float as an unsigned number; zeros of either sign are equal
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
  return b >> 31 ? ~b : b | 0x80000000u;
}

constexpr int kWaves = 4;

__device__ __forceinline__ float row_sum(float v, float* part) {
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}

template <typename T>
__global__ __launch_bounds__(64 * kWaves) void logprobs_kernel(LogprobParams p) {
  __shared__ float part[kWaves];
  __shared__ uint64_t best[kWaves];
  const int64_t row = ((int64_t)blockIdx.y << kGridShift) + blockIdx.x;
  if (row >= p.rows) return;
  const T* x = (const T*)p.x + row * p.xs;
  const float ninf = -__builtin_inff();
  float m = ninf;
  for (int v = threadIdx.x; v < p.V; v += 64 * kWaves) m = fmaxf(m, to_float(x[v]));
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = m;
  __syncthreads();
  m = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  const float base = m == ninf ? 0.0f : m;             // (a row of nothing but -infinity: every exponential is 0)
  float s = 0.0f, t = 0.0f;
  for (int v = threadIdx.x; v < p.V; v += 64 * kWaves) {
    const float d = to_float(x[v]) - base, e = __expf(d);
    s += e;
    t += e > 0.0f ? e * d : 0.0f;
  }
  s = row_sum(s, part);
  t = row_sum(t, part);
  const bool bad = s != s, none = s == 0.0f;
  const float ls = __logf(s);
  if (threadIdx.x == 0 && p.entropy) p.entropy[row] = bad ? s : none ? 0.0f : ls - t / s;
  for (int j = threadIdx.x; j < p.n; j += 64 * kWaves) {
    const int tok = p.tokens[row * p.n + j];
    p.logprob[row * p.n + j] = tok < 0 ? 0.0f : tok >= p.V || bad ? __builtin_nanf("") : none ? ninf : (to_float(x[tok]) - base) - ls;
  }
  uint64_t last = ~0ull;                               // keys below it are still to come
  for (int j = 0; j < p.top; ++j) {
    uint64_t b = 0;
    for (int v = threadIdx.x; v < p.V; v += 64 * kWaves) {
      const uint64_t key = (uint64_t)order_of(to_float(x[v])) << 32 | (uint32_t)~v;
      b = key < last && key > b ? key : b;
    }
    for (int d = 32; d > 0; d >>= 1) {
      const uint64_t o = __shfl_xor((unsigned long long)b, d);
      b = o > b ? o : b;
    }
    __syncthreads();
    if (threadIdx.x % 64 == 0) best[threadIdx.x / 64] = b;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) b = best[w] > b ? best[w] : b;
    last = b;
    if (threadIdx.x == 0) {
      const int id = bad ? -1 : (int)~(uint32_t)b;
      p.top_ids[row * p.top + j] = id;
      p.top_logprob[row * p.top + j] = bad ? s : none ? ninf : (to_float(x[id]) - base) - ls;
    }
  }
}

}  // namespace

size_t logprobs_workspace_bytes(int64_t, int, int) { return 0; }

hipError_t launch_logprobs(const LogprobParams& p, int x_type, void*, hipStream_t st) {
  const GridShape g = grid_shape(p.rows);
  return with_type(x_type, [&](auto t) {
    return launch_kernel(logprobs_kernel<decltype(t)>, dim3(g.x, g.y), dim3(64 * kWaves), 0, st, p);
  });
}

}  // namespace qasr
