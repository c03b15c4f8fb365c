// Matrix products of int8 codes with a scale per token and per channel, one matrix or one per group of rows.
//
// A wave computes 16 channels x 16 tokens: the operands of v_mfma_i32_16x16x64_i8 are 16 consecutive bytes of a row per lane
// (lane = 16 g + r: row r, bytes 16 g .. 16 g + 15 of a chunk of 64), the weights as the first operand, so that a lane
// ends with four consecutive channels of one token.
#include "floats.hpp"
#include "kernels.hpp"
#include "launch_shape.hpp"

namespace qasr {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

// bytes [k, k + 16) of a row of K bytes, zeros past its end
__device__ __forceinline__ v4i row_chunk(const int8_t* row, int k, int K) {
  if (k + 16 <= K) return *reinterpret_cast<const unaligned_chunk16*>(row + k);
  v4i v = (v4i){0, 0, 0, 0};
  for (int i = 0; k + i < K; ++i) v[i >> 2] |= (int)((uint32_t)(uint8_t)row[k + i] << (8 * (i & 3)));
  return v;
}

// The group and the rows [lo, hi) of tile t where every group's rows are cut into tiles of BM; false past the last tile.
template <int BM>
__device__ __forceinline__ bool group_tile(const LinearParams& p, int64_t t, int& e, int& lo, int& hi) {
  const int lane = threadIdx.x & 63;
  for (int e0 = 0; e0 < p.E; e0 += 64) {
    int a = 0, b = 0;
    if (e0 + lane < p.E) {
      a = min(max(p.offsets[e0 + lane], 0), p.M);
      b = min(max(p.offsets[e0 + lane + 1], 0), p.M);
    }
    const int n = b > a ? (b - a + BM - 1) / BM : 0;
    int upto = n;                                      // tiles of this and the groups before it among the 64
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      upto += lane >= d ? o : 0;
    }
    const int all = __shfl(upto, 63);
    if (t < all) {
      const int src = __popcll(__ballot(upto <= (int)t));
      e = e0 + src;
      lo = __shfl(a, src) + ((int)t - __shfl(upto - n, src)) * BM;
      hi = min(__shfl(b, src), lo + BM);
      return true;
    }
    t -= all;
  }
  return false;
}

template <typename T>
__global__ __launch_bounds__(256) void linear_kernel(LinearParams p, int64_t tiles) {
  const int64_t unit = (((int64_t)blockIdx.y << kGridShift) + blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  if (unit >= tiles) return;
  const int n16 = (p.N + 15) / 16;
  const int n0 = (int)(unit % n16) * 16;
  int e = 0, lo = (int)(unit / n16) * 16, hi = min(p.M, lo + 16);
  if (p.offsets && !group_tile<16>(p, unit / n16, e, lo, hi)) return;
  const int m = min(lo + r, hi - 1);
  int i = p.index ? p.index[m] : m;
  const bool known = i >= 0 && i < p.x_rows;
  i = known ? i : 0;
  const int8_t* wr = p.w + e * p.wes + min(n0 + r, p.N - 1) * p.ws;
  const int8_t* xr = p.x + i * p.xs;
  v4i acc = (v4i){0, 0, 0, 0};
  for (int k = 16 * g; k - 16 * g < p.K; k += 64)
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(row_chunk(wr, k, p.K), row_chunk(xr, k, p.K), acc, 0, 0, 0);
  if (lo + r >= hi) return;
  const float sx = p.x_scale[i];
  T* yr = (T*)p.y + (int64_t)m * p.ys;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int n = n0 + 4 * g + c;
    if (n >= p.N) break;
    const int64_t at = (int64_t)e * p.N + n;
    float v = __fmul_rn(__fmul_rn((float)(known ? acc[c] : 0), sx), p.w_scale[at]);
    if (p.bias) v = __fadd_rn(v, p.bias[at]);
    yr[n] = from_float<T>(v);
  }
}

}  // namespace

hipError_t launch_linear(const LinearParams& p, hipStream_t st) {
  const int64_t m16 = p.offsets ? p.M / 16 + (p.E < p.M ? p.E : p.M) : (p.M + 15) / 16;
  const int64_t tiles = m16 * ((p.N + 15) / 16);
  const GridShape g = grid_shape((tiles + 3) / 4);
  return with_type(p.y_type, [&](auto t) {
    return launch_kernel(linear_kernel<decltype(t)>, dim3(g.x, g.y), dim3(256), 0, st, p, tiles);
  });
}

}  // namespace qasr
