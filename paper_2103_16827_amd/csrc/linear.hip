// Matrix products of int8 codes with a scale per token and per channel, one matrix or one per group of rows:
//   y[m,n] = ((float)(sum_k x[m,k] w[n,k]) x_scale[m]) w_scale[n] + bias[n].
//
// Both operands are rows of K consecutive codes, which is what v_mfma_i32_16x16x64_i8 wants: lane 16 g + r brings 16
// consecutive codes of row r (chunk g of 64).  Rows go to LDS by direct loads (1 KiB each) in steps of 128 codes, whole cache lines; the
// lane of a load that writes slot s of a row brings chunk s ^ f(row), so that the 16-byte reads of an operand (one chunk of
// many rows) touch every bank once.  Weights are the first operand: a lane ends up with four consecutive channels of one
// token, and which channels the rows of an operand are is chosen so that a lane has 16 bytes of y over one or two products.
//
// linear_few (few tokens): the weights pass once from memory to one workgroup, which is all such a product costs.  The waves
// of a workgroup split K, each with a ring of its own in LDS and no barrier before the end, where the exact int32
// partial sums meet in LDS.  Bound by memory, and below 16 MB of weights by one launch and its chain of loads: 1 token of 4096 x 4096
// 4.9 us with the weights in the 256 MB cache and 6.8 from memory, 32 of 11008 x 4096 10.6 and 15.3 (3.0 TB/s), 1 of 32768 x 4096 29.8 from
// memory (4.5 TB/s).
// linear_tile (more): tiles of BM x BN through a ring in LDS that the waves share, a barrier per step.  8192 x 14336 x 4096 372 to 400 us by
// the card = 2.4 to 2.6 POP/s, 8192^3 384 to 438 = 2.5 to 2.9: matrix pipes 62 % busy at the 1.9 GHz that the operands' power leaves (zeros instead of
// codes, on a card that takes 400 us: 300).  A step of a 256 x 256 tile keeps the LDS port (192 KiB read, 64 written, 128 bytes a cycle) as long as the products keep the
// pipes.  Four waves of 128 x 128 each instead of eight of 128 x 64, which read a third less, have one wave per SIMD and were 3 to 6 % slower;
// stages of 64 codes, three of them, too, at half the vector cache's rate; tiles in turn with the results of one leaving under the
// products of the next spilled registers.
// linear_rows: the same tiles for rows of any alignment, through registers.  777 x 1029 x 1003 7.6 to 8.0 us, 2000 x 2001 x 2001 24.4
// (0.66 POP/s): its chain of loads, two steps ahead.
#include "floats.hpp"
#include "kernels.hpp"
#include "lanes.hpp"
#include "launch_shape.hpp"
#include "quantize_row.hpp"
#include "tuning.hpp"
#include "vmem.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace qasr {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kLdsBytes = 160 * 1024;

__device__ __align__(16) const uint8_t kZeros[16] = {};   // what stands for codes past the end of a row

// Rows that begin anywhere or end inside a chunk: chunk k (bytes [k, k + 16), zeros past the end of the K bytes) is loaded from
// chunk_at(k, K), no branch around the load, and moved down by what that lies ahead of k once it is there.  (Byte by byte a
// row's end would be a chain of up to 15 round trips to memory.)  K >= 16.
__device__ __forceinline__ int chunk_at(int k, int K) { return min(k, K - 16); }
__device__ __forceinline__ v4i moved_down(v4i all, int by) {               // by 0 .. 16 bytes, without a branch
  const uint32_t eight = -(by >> 3 & 1), four = -(by >> 2 & 1), none = (by >> 4) - 1;
  uint32_t w[5] = {(uint32_t)all[0], (uint32_t)all[1], (uint32_t)all[2], (uint32_t)all[3], 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = ((i < 2 ? w[i + 2] : 0) & eight) | (w[i] & ~eight);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = ((w[i + 1] & four) | (w[i] & ~four)) & none;
  v4i v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (int)__builtin_amdgcn_alignbyte(w[i + 1], w[i], by & 3);
  return v;
}
// ... of a row shorter than 16
__device__ __forceinline__ v4i short_row(const int8_t* row, int k, int K) {
  v4i v = (v4i){0, 0, 0, 0};
  for (int i = 0; k + i < K; ++i) v[i >> 2] |= (int)((uint32_t)(uint8_t)row[k + i] << (8 * (i & 3)));
  return v;
}

struct Tile {
  int e;            // group
  int lo, hi;       // its rows
  int n0;           // first channel
};

// offsets[i] held to [0, M]
__device__ __forceinline__ int offset_at(const LinearParams& L, int i) { return min(max(L.offsets[i], 0), L.M); }

// How the launch's workgroups are shared out.  Workgroup b runs on XCD b mod 8: an XCD gets consecutive tiles, which read the
// same rows of x or w, so that these come to its L2 once.
struct Order {
  int nt;           // tiles of channels
  int mt;           // tiles of rows (groups: the most there can be)
  int along;        // tiles of rows that take turns before the next tile of channels
};

// the unit-th of n units (fewer than 2^31), in runs of consecutive ones per XCD; -1 past the last
__device__ __forceinline__ int xcd_order(uint32_t unit, uint32_t n) {
  const uint32_t per = (n + 7) / 8, t = (unit & 7) * per + (unit >> 3);
  return (unit >> 3) < per && t < n ? (int)t : -1;
}
__device__ __forceinline__ uint32_t first_unit() { return (blockIdx.y << kGridShift) + blockIdx.x; }

// The tile of this workgroup where every group's rows are cut into tiles of BM; false if there is none.  Rows are counted 64
// groups at a time by a scan over the lanes; every wave does it for itself.  Their tiles are unsigned numbers: offsets that fall
// and rise again (which may give wrong values, never an access out of range) make up to 32 M / BM + 64 of them, 2^31 + 64.
template <int BM>
__device__ __forceinline__ bool group_tile(const LinearParams& L, const Order& o, uint32_t unit, int BN, Tile& t) {
  const int lane = threadIdx.x & 63;
  int a, b;                                 // the lane's group among the 64 from e0 on, and its tiles
  auto upto = [&](int e0, uint32_t& n) __attribute__((always_inline)) {
    const int e = min(e0 + lane, L.E - 1);
    a = offset_at(L, e);
    b = offset_at(L, e + 1);
    n = e0 + lane < L.E && b > a ? (b - a + BM - 1) / BM : 0;
    return wave_scan(n, 0u, [](uint32_t x, uint32_t y) { return x + y; });
  };
  auto of_lane = [](uint32_t v, int from) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readlane((int)v, from); };
  const uint32_t most = o.mt;
  uint32_t n, before = upto(0, n), total = of_lane(before, 63);
  for (int e0 = 64; e0 < L.E && total < most; e0 += 64) total += of_lane(upto(e0, n), 63);
  if (L.E > 64) before = upto(0, n);
  // (more than that only where offsets decrease)
  const int u = xcd_order(unit, min(total, most) * o.nt);
  if (u < 0) return false;
  uint32_t left = u / o.nt;
  t.n0 = (u - (int)left * o.nt) * BN;
  for (int e0 = 0;;) {
    const uint32_t all = of_lane(before, 63);
    if (left < all) {
      const int src = __popcll(__ballot(before <= left));
      t.e = e0 + src;
      t.lo = __builtin_amdgcn_readlane(a, src) + (int)(left - of_lane(before - n, src)) * BM;
      t.hi = min(__builtin_amdgcn_readlane(b, src), t.lo + BM);
      return true;
    }
    left -= all;
    e0 += 64;
    if (e0 >= L.E) return false;
    before = upto(e0, n);
  }
}

// the same for one matrix: `along` tiles of rows by all tiles of channels, the rows going first
template <int BM>
__device__ __forceinline__ bool plain_tile(const LinearParams& L, const Order& o, uint32_t unit, int BN, Tile& t) {
  const int u = xcd_order(unit, (uint32_t)o.mt * o.nt);
  if (u < 0) return false;
  const int band = u / (o.along * o.nt), in = u - band * o.along * o.nt;
  const int rows = min(o.along, o.mt - band * o.along), across = in / rows;
  t.e = 0;
  t.lo = (band * o.along + in - across * rows) * BM;
  t.hi = min(L.M, t.lo + BM);
  t.n0 = across * BN;
  return true;
}

template <int BM>
__device__ __forceinline__ bool find_tile(const LinearParams& L, const Order& o, uint32_t unit, int BN, Tile& t) {
  if (!L.offsets) return plain_tile<BM>(L, o, unit, BN, t);
  return group_tile<BM>(L, o, unit, BN, t);
}

// row of x that row m of y reads, -1 for one that is not there
__device__ __forceinline__ int x_row(const LinearParams& L, int m) {
  if (!L.index) return m;
  const int i = L.index[m];
  return i >= 0 && i < L.x_rows ? i : -1;
}

// Slot of a row's chunk c is c ^ f: what eight consecutive lanes read of as many rows then lies in different banks, which a row
// of 128 codes fills.  Rows are counted as an operand's lanes read them (r = lane & 15).
__device__ __forceinline__ int swizzle(int r) { return r & 7; }

// Row r of product nt of a wave is its channel channel_of: lanes 16 g .. end with 4 P consecutive channels of a token over P
// products, 16 bytes of y.
template <int P>
__device__ __forceinline__ int channel_of(int nt, int r) { return 16 * P * (nt / P) + 4 * P * (r >> 2) + 4 * (nt % P) + (r & 3); }
template <int P>
__device__ __forceinline__ int row_of(int n) { return 4 * ((n / (4 * P)) & 3) + (n & 3); }      // the r of channel n

// how many products a lane's 16 bytes of y come from
template <typename T>
constexpr int products_of(int NT) { return NT < 4 / (int)sizeof(T) ? NT : 4 / (int)sizeof(T); }

// each operation rounds once, as the ABI says; the sum itself rounds where it passes 2^24.  No bias is an addition of 0.
template <typename T>
__device__ __forceinline__ T result(int acc, float sx, float ws, float bias) {
#pragma clang fp contract(off)
  const float v = ((float)acc * sx) * ws;
  return from_float<T>(v + bias);
}

// the scale of row m of y's tokens: a row that is not there counts as zeros
__device__ __forceinline__ float token_scale(const LinearParams& L, int m) {
  const int xr = x_row(L, m);
  return xr >= 0 ? L.x_scale[xr] : 0.0f;
}
__device__ __forceinline__ float channel_scale(const LinearParams& L, const Tile& t, int n) {
  return L.w_scale[(int64_t)t.e * L.N + min(n, L.N - 1)];
}
__device__ __forceinline__ float channel_bias(const LinearParams& L, const Tile& t, int n) {
  return L.bias ? L.bias[(int64_t)t.e * L.N + min(n, L.N - 1)] : 0.0f;
}

// ---- few tokens

// Elements of x that linear_few quantises by itself: they are in registers in between.
constexpr int kFloats = 8192;
// W waves; wave w takes the steps w, w + W, ...; DIRECT: rows 16-byte aligned, K a multiple of 16.
// X: int8_t, or the type of float tokens, up to 16 of them and kFloats elements, that every workgroup quantises for itself while its
// weights are on their way (a launch less, which for one token is half of the time); their rows 16-byte aligned.
template <int MT, int NT, int W, int S, bool DIRECT, bool ONCE, typename X, typename T>
__global__ __launch_bounds__(64 * W) void linear_few_kernel(LinearParams L, Order o) {
  constexpr bool FLOATS = !__is_same(X, int8_t);
  static_assert(!FLOATS || (DIRECT && MT == 1), "floats: one product of tokens");
  constexpr int STEP = 128, P = products_of<T>(NT);
  constexpr int BM = 16 * MT, BN = 16 * NT, TOKENS = FLOATS ? 0 : BM;          // rows of tokens in a stage
  constexpr int kLoads = (TOKENS + BN) / 8, kStage = (TOKENS + BN) * STEP;
  static_assert(S * kStage >= MT * NT * 1024, "a wave's partial sums go where its ring was");
  extern __shared__ __align__(1024) unsigned char lds[];
  Tile t;
  if (!find_tile<BM>(L, o, first_unit(), BN, t)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  unsigned char* ring = lds + wave * (S * kStage);

  const int steps = (L.K + STEP - 1) / STEP, rows = t.hi - t.lo;
  const int mine = wave < steps ? (steps - wave + W - 1) / W : 0;
  const int8_t* row[kLoads];
  int chunk[kLoads];
  bool brings[kLoads];             // rows that there are, and a row of every load: the waits count loads
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int i = 8 * j + (lane >> 3);
    if (8 * j < TOKENS) {
      const int xr = x_row(L, t.lo + min(i, rows - 1));
      row[j] = L.x + (int64_t)max(xr, 0) * L.xs;
      chunk[j] = (lane & 7) ^ swizzle(i & 15);
      brings[j] = i < rows || i % 8 == 0;
    } else {
      const int n = i - TOKENS;
      row[j] = L.w + t.e * L.wes + (int64_t)min(t.n0 + n, L.N - 1) * L.ws;
      chunk[j] = (lane & 7) ^ swizzle(row_of<P>(n));
      brings[j] = true;
    }
  }

  // At the end every wave puts some of the 16 x 16 results together; what they are scaled by is asked for now.
  struct Item { int m, n; float sx; v4f ws, bias; };
  auto item = [&](int i) __attribute__((always_inline)) {
    Item it;
    it.m = t.lo + 16 * (i / NT) + r;
    it.n = t.n0 + channel_of<P>(i % NT, 4 * g);
    it.sx = FLOATS ? 0.0f : token_scale(L, min(it.m, t.hi - 1));
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      it.ws[c] = channel_scale(L, t, it.n + c);
      it.bias[c] = channel_bias(L, t, it.n + c);
    }
    return it;
  };
  Item mine_at_end = item(min(wave, MT * NT - 1));

  v4i acc[MT][NT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = (v4i){0, 0, 0, 0};

  // FLOATS: the tokens' codes, rows of `pitch` bytes whose chunk c of 128 bytes is at c ^ (row & 7), and their scales
  unsigned char* codes = lds + W * S * kStage;
  const int pitch = steps * STEP, own = min(r, rows - 1);
  float* code_scale = (float*)(codes + rows * pitch);
  auto products = [&](const unsigned char* stage, int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = 16 * ((4 * h + g) ^ swizzle(r));
      v4i a[MT], b[NT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if constexpr (FLOATS) a[mt] = *(const v4i*)(codes + own * pitch + k0 + 16 * ((4 * h + g) ^ (own & 7)));
        else a[mt] = *(const v4i*)(stage + (16 * mt + r) * STEP + at);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) b[nt] = *(const v4i*)(stage + (TOKENS + channel_of<P>(nt, r)) * STEP + at);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[nt], a[mt], acc[mt][nt], 0, 0, 0);
    }
  };

  if constexpr (DIRECT) {
    auto ask = [&](int i) __attribute__((always_inline)) {
      const int k0 = (wave + i * W) * STEP;
      unsigned char* stage = ring + (i % S) * kStage;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int k = k0 + 16 * chunk[j];
        const void* p = k < L.K ? (const void*)(row[j] + k) : (const void*)kZeros;
        if (ONCE && 8 * j >= TOKENS) direct_load16(Once(), p, stage + 1024 * j);
        else if (brings[j]) direct_load16(p, stage + 1024 * j);
      }
    };
    for (int i = 0; i < min(S, mine); ++i) ask(i);
    if constexpr (FLOATS) {
      constexpr int N = kPer<X>, R = kFloats / N / (64 * W);
      const int per = L.K / N, all = rows * per;               // pieces of 16 bytes
      uint32_t* most = (uint32_t*)(code_scale + 16);
      if (threadIdx.x < 16) most[threadIdx.x] = 0;
      v4u raw[R];
      int of[R];
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int c = threadIdx.x + j * 64 * W;
        of[j] = c / per;
        raw[j] = (v4u){0, 0, 0, 0};
        if (c < all) raw[j] = *reinterpret_cast<const v4u*>((const X*)L.xf + (int64_t)(t.lo + of[j]) * L.xs + (c - of[j] * per) * N);
      }
      // zeros behind the codes, up to a whole step
      const int pad = (pitch - L.K) / 16;
      for (int j = threadIdx.x; j < rows * pad; j += 64 * W) {
        const int m = j / pad, c = L.K / 16 + (j - m * pad);
        *(v4i*)(codes + m * pitch + 16 * (c ^ (m & 7))) = (v4i){0, 0, 0, 0};
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < R; ++j) {
        if (threadIdx.x - lane + j * 64 * W >= all) break;       // (the whole wave)
        uint32_t a = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t word = sign_off<X>(raw[j][k]);
          if constexpr (sizeof(X) == 4) a = max(a, word < kInf<X> ? word : 0u);
          else a = max(a, max((word & 0xffffu) < kInf<X> ? word & 0xffffu : 0u, word >> 16 < kInf<X> ? word >> 16 : 0u));
        }
        // one update for a wave that is in one row
        if (__builtin_amdgcn_readfirstlane(of[j]) == __builtin_amdgcn_readlane(of[j], 63)) {
          a = wave_max(a);
          if (lane == 0) atomicMax(&most[of[j]], a);
        } else if (of[j] < rows) {
          atomicMax(&most[of[j]], a);
        }
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int c = threadIdx.x + j * 64 * W, k = (c - of[j] * per) * N, m = of[j];
        if (c >= all) break;
        const float S_m = scale_of(magnitude<X>(most[m]));
        if (k == 0) code_scale[m] = S_m;
#pragma unroll
        for (int w = 0; w < N / 4; ++w)
          *(uint32_t*)(codes + m * pitch + 16 * ((k >> 4) ^ (m & 7)) + (k & 15) + 4 * w) =
              codes_of(element<X>(raw[j], 4 * w), element<X>(raw[j], 4 * w + 1), element<X>(raw[j], 4 * w + 2), element<X>(raw[j], 4 * w + 3), S_m);
      }
      __syncthreads();
      mine_at_end.sx = code_scale[own];
    }
    for (int i = 0; i < mine; ++i) {
      if (i + S <= mine) wait_vm<(S - 1) * kLoads>();
      else wait_vm_dyn((mine - 1 - i) * kLoads);
      products(ring + (i % S) * kStage, (wave + i * W) * STEP);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the slot has been read
      if (i + S < mine) ask(i + S);
    }
    wait_vm<0>();
  } else {
    constexpr int D = 2;                           // steps on their way
    v4i next[D][kLoads];
    auto k_of = [&](int i, int j) __attribute__((always_inline)) { return (wave + i * W) * STEP + 16 * chunk[j]; };
    auto fetch = [&](int i, v4i (&to)[kLoads]) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) to[j] = *reinterpret_cast<const unaligned_chunk16*>(row[j] + chunk_at(k_of(i, j), L.K));
    };
    auto multiply = [&](int i, const v4i (&from)[kLoads]) __attribute__((always_inline)) {
      const bool whole = (wave + i * W + 1) * STEP <= L.K;
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        *(v4i*)(ring + 1024 * j + 16 * lane) = whole ? from[j] : moved_down(from[j], min(16, max(0, k_of(i, j) + 16 - L.K)));
      __builtin_amdgcn_wave_barrier();
      products(ring, 0);
      __builtin_amdgcn_wave_barrier();
    };
    if (L.K < 16) {
      if (mine > 0) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) next[0][j] = short_row(row[j], 16 * chunk[j], L.K);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) *(v4i*)(ring + 1024 * j + 16 * lane) = next[0][j];
        __builtin_amdgcn_wave_barrier();
        products(ring, 0);
      }
    } else {
#pragma unroll
      for (int d = 0; d < D; ++d)
        if (d < mine) fetch(d, next[d]);
      for (int i = 0; i < mine; i += D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
          if (i + d >= mine) break;
          multiply(i + d, next[d]);
          if (i + d + D < mine) fetch(i + d + D, next[d]);
        }
      }
    }
  }

#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) *(v4i*)(ring + (mt * NT + nt) * 1024 + 16 * lane) = acc[mt][nt];
  __syncthreads();
#pragma unroll
  for (int i0 = 0; i0 < MT * NT; i0 += W) {
    const int i = i0 + wave;
    if (i >= MT * NT) break;
    if (i0 > 0) mine_at_end = item(i);
    const Item& it = mine_at_end;
    v4i sum = (v4i){0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < W; ++w) sum += *(const v4i*)(lds + w * (S * kStage) + i * 1024 + 16 * lane);
    if (it.m >= t.hi) continue;
    T* y = (T*)L.y + (int64_t)it.m * L.ys + it.n;
    struct __attribute__((packed, aligned(sizeof(T)))) Four { T v[4]; } f;
#pragma unroll
    for (int c = 0; c < 4; ++c) f.v[c] = result<T>(sum[c], it.sx, it.ws[c], it.bias[c]);
    if (it.n + 4 <= L.N) {
      *reinterpret_cast<Four*>(y) = f;
    } else {
#pragma unroll
      for (int c = 0; c < 3; ++c)
        if (it.n + c < L.N) y[c] = f.v[c];
    }
  }
}

// ---- tiles

template <int MT, int NT>
using Sums = v4i[MT][NT];

// A wave's 16 MT x 16 NT products over one half (64 codes) of a stage whose tokens begin at `as` and channels at `bs`, at the
// lane's own row; at: the lane's chunk
template <int MT, int NT, int P, int STEP>
__device__ __forceinline__ void products_of_half(Sums<MT, NT>& acc, const unsigned char* as, const unsigned char* bs) {
  v4i a[MT], b[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) b[nt] = *(const v4i*)(bs + channel_of<P>(nt, 0) * STEP);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) a[mt] = *(const v4i*)(as + 16 * mt * STEP);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[nt], a[mt], acc[mt][nt], 0, 0, 0);
}

// scales in LDS: BM of the tile's tokens, BN of its channels, BN biases
template <int BM, int BN, int THREADS>
struct Scales {
  static constexpr int kEach = (BM + 2 * BN + THREADS - 1) / THREADS;
  float v[kEach];
  __device__ __forceinline__ void load(const LinearParams& L, const Tile& t) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int i = threadIdx.x + j * THREADS;
      v[j] = i < BM ? token_scale(L, min(t.lo + i, t.hi - 1)) : i < BM + BN ? channel_scale(L, t, t.n0 + i - BM) : channel_bias(L, t, t.n0 + i - BM - BN);
    }
  }
  __device__ __forceinline__ void put(float* to) const {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int i = threadIdx.x + j * THREADS;
      if (i < BM + 2 * BN) to[i] = v[j];
    }
  }
};

// The results of a wave go through its share (ROOM bytes) of the LDS that the stages were in, as many tokens at a time as fit,
// so that they leave as whole cache lines: from the registers, where a lane has 16 bytes of every product or two, they would go
// as 64-byte pieces.  Piece p of a row is at p ^ (row & 7).
// Rows that keep to boundaries of 64 bytes are stored past the caches, so that no workgroup leaves a 4 MB L2 full of lines to
// be written out, and the operands stay there: 8192 x 14336 x 4096 401 us for 408 on one card (364 for 402 on another), 4096 x 4096 x 512 15.5
// for 16.1, and no difference for 6400 x 2048 x 512 in float32 (17.7 and 17.9), alone or with the layer that quantises the result behind it
// (44.1 and 43.8 together).  Lines that two workgroups share have to meet in the cache: 4096 x 4104 x 512 took 30.4 us past it, 25 to 28
// through it.
template <int MT, int NT, int BM, int BN, int ROOM, typename T>
__device__ __forceinline__ void store_tile(const LinearParams& L, const Tile& t, const float* scales, unsigned char* room, int m0, int n0,
                                           const Sums<MT, NT>& acc) {
  constexpr int P = products_of<T>(NT), C = 4 * P, PR = NT * (int)sizeof(T);      // C channels are a piece, PR pieces a row
  constexpr int kFit = ROOM / (16 * PR * 16), MB = kFit >= MT ? MT : kFit >= 4 ? 4 : kFit >= 2 ? 2 : 1;
  static_assert(C * sizeof(T) == 16 && PR >= 8 && 64 % PR == 0 && MT % MB == 0 && kFit >= 1, "room for rows of pieces");
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  v4f ws[NT], bias[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    ws[nt] = *(const v4f*)(scales + BM + n0 + channel_of<P>(nt, 4 * g));
    bias[nt] = *(const v4f*)(scales + BM + BN + n0 + channel_of<P>(nt, 4 * g));
  }
  const int p = lane % PR, n = t.n0 + n0 + C * p;
  const bool whole = (((uintptr_t)L.y | (uint64_t)L.ys * sizeof(T)) & 63) == 0;
#pragma unroll
  for (int b = 0; b < MT / MB; ++b) {
    const int mb = m0 + 16 * MB * b;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      const float sx = scales[mb + 16 * i + r];
#pragma unroll
      for (int j = 0; j < NT / P; ++j) {
        struct __attribute__((aligned(16))) { T v[C]; } piece;
#pragma unroll
        for (int c = 0; c < C; ++c)
          piece.v[c] = result<T>(acc[MB * b + i][P * j + c / 4][c % 4], sx, ws[P * j + c / 4][c % 4], bias[P * j + c / 4][c % 4]);
        *(v4i*)(room + ((16 * i + r) * PR + ((4 * j + g) ^ (r & 7))) * 16) = __builtin_bit_cast(v4i, piece);
      }
      __builtin_amdgcn_sched_barrier(0);                     // (else the registers do not last)
    }
    asm volatile("" ::: "memory");                           // other lanes read it: a wave's LDS accesses stay in order
    const int rows = min(16 * MB, t.hi - t.lo - mb);
    T* y = (T*)L.y + (int64_t)(t.lo + mb) * L.ys + n;
    auto piece = [&](int row) __attribute__((always_inline)) { return *(const v4i*)(room + (row * PR + (p ^ (row & 7))) * 16); };
    if (whole && n + C <= L.N) {
#pragma unroll 4
      for (int row = lane / PR; row < rows; row += 64 / PR) __builtin_nontemporal_store(piece(row), (v4i*)(y + row * L.ys));
    } else if (n + C <= L.N) {
#pragma unroll 4
      for (int row = lane / PR; row < rows; row += 64 / PR) *reinterpret_cast<unaligned_chunk16*>(y + row * L.ys) = piece(row);
    } else {
      for (int row = lane / PR; row < rows; row += 64 / PR)
        for (int c = 0; n + c < L.N; ++c) y[row * L.ys + c] = ((const T*)(room + (row * PR + (p ^ (row & 7))) * 16))[c];
    }
    asm volatile("" ::: "memory");
  }
}

// WM x WN waves of 16 MT tokens x 16 NT channels each, S stages of 128 codes.
template <int MT, int NT, int WM, int WN, int S, bool ONCE, typename T>
__global__ __launch_bounds__(64 * WM * WN) void linear_tile_kernel(LinearParams L, Order o) {
  constexpr int STEP = 128, P = products_of<T>(NT), RPL = 1024 / STEP, CPR = STEP / 16;     // rows per load, chunks per row
  constexpr int W = WM * WN, BM = 16 * MT * WM, BN = 16 * NT * WN, kStage = (BM + BN) * STEP;
  constexpr int kTokenLoads = BM / RPL / W, kLoads = kTokenLoads + BN / RPL / W;
  static_assert(BM % (RPL * W) == 0 && BN % (RPL * W) == 0, "whole loads of tokens and of channels for every wave");
  static_assert(RPL * W % 16 == 0, "a lane brings the same chunk in all its loads of tokens, and in all of channels");
  static_assert(MT >= 2 && S * kStage + 4 * (BM + 2 * BN) <= kLdsBytes, "LDS");
  extern __shared__ __align__(1024) unsigned char lds[];
  float* scales = (float*)(lds + S * kStage);
  Tile t;
  if (!find_tile<BM>(L, o, first_unit(), BN, t)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int wm = wave / WN, wn = wave % WN;
  const int steps = (L.K + STEP - 1) / STEP;

  // the rows that this lane brings, by 32-bit offsets from the tile's first rows (the launch sees to it that these do)
  const int first = RPL * wave + lane / CPR;
  const int token_chunk = (lane % CPR) ^ swizzle(first & 15), channel_chunk = (lane % CPR) ^ swizzle(row_of<P>(first));
  const int8_t* xbase = L.x + (L.index ? 0 : (int64_t)t.lo * L.xs);
  const int8_t* wbase = L.w + t.e * L.wes + (int64_t)t.n0 * L.ws;
  uint32_t off[kLoads];
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int i = first + RPL * W * (j < kTokenLoads ? j : j - kTokenLoads);
    const int m = min(i, t.hi - t.lo - 1);
    if (j < kTokenLoads) off[j] = (uint32_t)(L.index ? max(x_row(L, t.lo + m), 0) : m) * (uint32_t)L.xs + 16 * token_chunk;
    else off[j] = (uint32_t)min(i, L.N - 1 - t.n0) * (uint32_t)L.ws + 16 * channel_chunk;
  }
  auto load = [&](int j, const int8_t* from, int slot) __attribute__((always_inline)) {
    if (ONCE && j >= kTokenLoads) direct_load16(Once(), from, off[j], lds + slot + 1024 * (j * W + wave));
    else direct_load16(from, off[j], lds + slot + 1024 * (j * W + wave));
  };
  // load j of stage k, which goes to `slot`; past the end of a row come zeros of the tokens (ask_end), anything of the channels
  auto ask_one = [&](int k, int slot, int j) __attribute__((always_inline)) {
    const int left = L.K - k * STEP;
    if (16 * (j < kTokenLoads ? token_chunk : channel_chunk) < left)
      load(j, (j < kTokenLoads ? xbase : wbase) + k * STEP, slot);
  };
  auto ask_end = [&](int k, int slot) __attribute__((always_inline)) {
    if (16 * token_chunk >= L.K - k * STEP) {
#pragma unroll
      for (int j = 0; j < kTokenLoads; ++j) *(v4i*)(lds + slot + 1024 * (j * W + wave) + 16 * lane) = (v4i){0, 0, 0, 0};
    }
  };
  // Two halves of a stage take turns, each one's operands read under the products of the one before.  Once the second
  // half's are on their way into registers, and the next stage has come, the stage's room is free: it is asked for again there.
  Sums<MT, NT> acc;
  v4i a[MT], b[2][NT];
  const int at[2] = {16 * (g ^ swizzle(r)), 16 * ((4 + g) ^ swizzle(r))};
  const unsigned char* as = lds + (16 * MT * wm + r) * STEP;
  const unsigned char* bs = lds + (BM + 16 * NT * wn + channel_of<P>(0, r)) * STEP;
  auto read_a = [&](int mt, int slot, int h) __attribute__((always_inline)) { a[mt] = *(const v4i*)(as + slot + at[h] + 16 * mt * STEP); };
  auto read_b = [&](int nt, int slot, int h) __attribute__((always_inline)) { b[h][nt] = *(const v4i*)(bs + slot + at[h] + channel_of<P>(nt, 0) * STEP); };
  auto read_bs = [&](int mt, int slot, int h) __attribute__((always_inline)) {
    if (mt < NT) read_b(mt, slot, h);
    if (mt == MT - 1) {
#pragma unroll
      for (int nt = MT; nt < NT; ++nt) read_b(nt, slot, h);
    }
  };
  auto products_of_row = [&](int mt, int h) __attribute__((always_inline)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[h][nt], a[mt], acc[mt][nt], 0, 0, 0);
  };
  auto first_half = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      products_of_row(mt, 0);
      read_a(mt, slot, 1);
      read_bs(mt, slot, 1);
      __builtin_amdgcn_sched_barrier(0);           // (else the reads come early and the registers do not last)
    }
  };
  auto second_half = [&](int next, auto&& among) __attribute__((always_inline)) {
    read_a(0, next, 0);
    read_b(0, next, 0);
#pragma unroll
    for (int mt = 1; mt < MT; ++mt) {
      among(mt);
      products_of_row(mt, 1);
      read_a(mt, next, 0);
      read_bs(mt, next, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  Scales<BM, BN, 64 * W> sc;
  sc.load(L, t);
#pragma unroll 1
  for (int k = 0; k < min(S, steps); ++k) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) ask_one(k, k * kStage, j);
    ask_end(k, k * kStage);
  }
  sc.put(scales);
  if (steps >= S) wait_vm<(S - 1) * kLoads>();
  else wait_vm<0>();
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) read_b(nt, 0, 0);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) read_a(mt, 0, 0);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = (v4i){0, 0, 0, 0};
  int slot = 0, k = 0;
  // while the stage to ask for is a whole one: no branches among the products
  const int8_t *xk = xbase + S * STEP, *wk = wbase + S * STEP;
  for (const int whole = L.K / STEP; k + S < whole; ++k) {
    const int next = slot + kStage == S * kStage ? 0 : slot + kStage;
    first_half(slot);
    products_of_row(0, 1);
    wait_vm<(S - 2) * kLoads>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    second_half(next, [&](int mt) __attribute__((always_inline)) {
      // (the requests of a step, a few at a time: a wave whose request has to queue issues no products meanwhile)
#pragma unroll
      for (int j = kLoads * (mt - 1) / (MT - 1); j < kLoads * mt / (MT - 1); ++j)
        load(j, j < kTokenLoads ? xk : wk, slot);
    });
    xk += STEP;
    wk += STEP;
    slot = next;
  }
  for (; k + 1 < steps; ++k) {
    const int next = slot + kStage == S * kStage ? 0 : slot + kStage;
    first_half(slot);
    products_of_row(0, 1);
    if (k + S - 1 < steps) wait_vm<(S - 2) * kLoads>();
    else wait_vm<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (k + S < steps) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) ask_one(k + S, slot, j);
      ask_end(k + S, slot);
    }
    second_half(next, [](int) {});
    slot = next;
  }
  first_half(slot);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    products_of_row(mt, 1);
    __builtin_amdgcn_sched_barrier(0);
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");     // every stage has been read
  store_tile<MT, NT, BM, BN, S * kStage / W, T>(L, t, scales, lds + S * kStage / W * wave, 16 * MT * wm, 16 * NT * wn, acc);
  wait_vm<0>();
}

// The same tiles where rows begin anywhere or end inside a chunk, of 16 codes and more: rows come through registers.
template <int MT, int NT, int WM, int WN, typename T>
__global__ __launch_bounds__(64 * WM * WN) void linear_rows_kernel(LinearParams L, Order o) {
  constexpr int STEP = 128, P = products_of<T>(NT), RPL = 1024 / STEP, CPR = STEP / 16, D = 2;
  constexpr int W = WM * WN, BM = 16 * MT * WM, BN = 16 * NT * WN, kStage = (BM + BN) * STEP;
  constexpr int kTokenLoads = BM / RPL / W, kLoads = kTokenLoads + BN / RPL / W;
  static_assert(BM % (RPL * W) == 0 && BN % (RPL * W) == 0 && RPL * W % 16 == 0, "see linear_tile_kernel");
  extern __shared__ __align__(1024) unsigned char lds[];
  float* scales = (float*)(lds + 2 * kStage);
  Tile t;
  if (!find_tile<BM>(L, o, first_unit(), BN, t)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int wm = wave / WN, wn = wave % WN, steps = (L.K + STEP - 1) / STEP;
  const int first = RPL * wave + lane / CPR;
  const int token_chunk = (lane % CPR) ^ swizzle(first & 15), channel_chunk = (lane % CPR) ^ swizzle(row_of<P>(first));
  const int8_t* row[kLoads];
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int i = first + RPL * W * (j < kTokenLoads ? j : j - kTokenLoads);
    if (j < kTokenLoads) row[j] = L.x + (int64_t)max(x_row(L, min(t.lo + i, t.hi - 1)), 0) * L.xs;
    else row[j] = L.w + t.e * L.wes + (int64_t)min(t.n0 + i, L.N - 1) * L.ws;
  }
  Scales<BM, BN, 64 * W> sc;
  sc.load(L, t);
  // Step k's rows are asked for D steps before their products, into registers by turns; past the last step they are asked for
  // all the same, so that the compiler can count which are on their way.
  v4i next[D][kLoads];
  auto k_of = [&](int k, int j) __attribute__((always_inline)) { return k * STEP + 16 * (j < kTokenLoads ? token_chunk : channel_chunk); };
  auto fetch = [&](int k, v4i (&to)[kLoads]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) to[j] = *reinterpret_cast<const unaligned_chunk16*>(row[j] + chunk_at(k_of(k, j), L.K));
  };
  auto put = [&](int k, const v4i (&from)[kLoads]) __attribute__((always_inline)) {
    unsigned char* stage = lds + (k & 1) * kStage;
    const bool whole = (k + 1) * STEP <= L.K;
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      *(v4i*)(stage + 1024 * (j * W + wave) + 16 * lane) = whole ? from[j] : moved_down(from[j], min(16, max(0, k_of(k, j) + 16 - L.K)));
  };
  Sums<MT, NT> acc;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = (v4i){0, 0, 0, 0};
#pragma unroll
  for (int d = 0; d < D; ++d) fetch(d, next[d]);
  put(0, next[0]);
  sc.put(scales);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  for (int k0 = 0;; k0 += D) {
    bool more = true;
#pragma unroll
    for (int d = 0; d < D; ++d) {
      if (!more) continue;
      const int k = k0 + d;
      const unsigned char* stage = lds + (k & 1) * kStage;
      fetch(k + D, next[d]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = 16 * ((4 * h + g) ^ swizzle(r));
        products_of_half<MT, NT, P, STEP>(acc, stage + (16 * MT * wm + r) * STEP + at, stage + (BM + 16 * NT * wn + channel_of<P>(0, r)) * STEP + at);
      }
      more = k + 1 < steps;
      if (more) put(k + 1, next[(d + 1) % D]);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    if (!more) break;
  }
  store_tile<MT, NT, BM, BN, 2 * kStage / W, T>(L, t, scales, lds + 2 * kStage / W * wave, 16 * MT * wm, 16 * NT * wn, acc);
}

// ---- launches

// tiles of BM rows (groups: the most that the rows can make)
int64_t row_tiles(const LinearParams& p, int BM) {
  return p.offsets ? p.M / BM + (p.E < p.M ? p.E : p.M) : ((int64_t)p.M + BM - 1) / BM;
}

Order order_of(const LinearParams& p, int BM, int BN) { return Order{(p.N + BN - 1) / BN, (int)row_tiles(p, BM), 8}; }

GridShape grid_of(const Order& o) { return grid_shape(((int64_t)o.mt * o.nt + 7) / 8 * 8); }

// groups with rows, of which only the device knows the sizes: as if rows fell on them by chance
double groups_of(const LinearParams& p) { return p.offsets ? p.E * (1.0 - std::pow(1.0 - 1.0 / p.E, (double)p.M)) : 1.0; }

// ONCE: the weights come past the 256 MB cache behind the L2s.  That is for matrices, all experts' together, that are larger than
// the cache, and for as many rows as a tile has, of one matrix as two tiles that run side by side: 64 experts of 2048 x 2048 with
// 8 rows each 45.2 us for 52.6, with 32 rows 44.9 for 50.5, 128 of 1024 x 2048 with a row each 28.6 for 32.9.  With two tiles to most of
// 64 experts of 2816 x 2048 it is one or the other by the card (163 us for 167, 165 for 152).  Smaller matrices gain less where memory has
// them (32 x 11008 x 4096 14.8 us for 15.2), and lose more where the cache does (12.9 for 10.6).
constexpr int64_t kLargeWeights = 1 << 28;
bool weights_once(const LinearParams& p, int BM) {
  if (const int forced = tuning().linear_once) return forced == 2;
  return (int64_t)(p.offsets ? p.E : 1) * p.N * p.K >= kLargeWeights && p.M <= (p.offsets ? 1 : 2) * BM * groups_of(p);
}

template <int MT, int NT, int W, int S, bool DIRECT, typename X, typename T>
hipError_t launch_few(const LinearParams& p, hipStream_t st) {
  const Order o = order_of(p, 16 * MT, 16 * NT);
  const GridShape g = grid_of(o);
  constexpr bool floats = !__is_same(X, int8_t);
  const int bytes = W * S * 16 * ((floats ? 0 : MT) + NT) * 128 + (floats ? p.M * ((p.K + 127) / 128 * 128) + 128 : 0);
  auto launch = [&](auto once) {
    constexpr auto kernel = linear_few_kernel<MT, NT, W, S, DIRECT, once, X, T>;
    static std::atomic<uint64_t> done;
    const hipError_t e = ensure_max_dynamic_lds((const void*)kernel, done);
    return e != hipSuccess ? e : launch_kernel(kernel, dim3(g.x, g.y), dim3(64 * W), bytes, st, p, o);
  };
  if constexpr (DIRECT && !floats)             // (what takes floats has no weights as large)
    if (weights_once(p, 16 * MT)) return launch(std::true_type());
  return launch(std::false_type());
}

template <int MT, int NT, int WM, int WN, int S, typename T>
hipError_t launch_tile(const LinearParams& p, hipStream_t st) {
  constexpr int BM = 16 * MT * WM, BN = 16 * NT * WN, bytes = S * (BM + BN) * 128 + 4 * (BM + 2 * BN);
  const Order o = order_of(p, BM, BN);
  const GridShape g = grid_of(o);
  auto launch = [&](auto once) {
    constexpr auto kernel = linear_tile_kernel<MT, NT, WM, WN, S, once, T>;
    static std::atomic<uint64_t> done;
    const hipError_t e = ensure_max_dynamic_lds((const void*)kernel, done);
    return e != hipSuccess ? e : launch_kernel(kernel, dim3(g.x, g.y), dim3(64 * WM * WN), bytes, st, p, o);
  };
  if (weights_once(p, BM)) return launch(std::true_type());
  return launch(std::false_type());
}

template <int MT, int NT, int WM, int WN, typename T>
hipError_t launch_rows(const LinearParams& p, hipStream_t st) {
  constexpr int BM = 16 * MT * WM, BN = 16 * NT * WN, bytes = 2 * (BM + BN) * 128 + 4 * (BM + 2 * BN);
  const Order o = order_of(p, BM, BN);
  const GridShape g = grid_of(o);
  static std::atomic<uint64_t> done;
  const hipError_t e = ensure_max_dynamic_lds((const void*)linear_rows_kernel<MT, NT, WM, WN, T>, done);
  if (e != hipSuccess) return e;
  return launch_kernel(linear_rows_kernel<MT, NT, WM, WN, T>, dim3(g.x, g.y), dim3(64 * WM * WN), bytes, st, p, o);
}

// Rows on 16-byte boundaries that hold whole chunks, and whose offsets within a tile (with an index: within x) are 32-bit numbers.
bool direct_ok(const LinearParams& p) {
  if (p.K % 16 || p.xs % 16 || p.ws % 16 || p.wes % 16 || (uintptr_t)p.x % 16 || (uintptr_t)p.w % 16) return false;
  const int64_t most = ((int64_t)1 << 32) - 1024;
  return p.ws < most / 256 && (p.index ? p.xs < most / p.x_rows : p.xs < most / 256);
}

// What a form of the kernels takes for one tile on a compute unit, in us: `end` for its beginning and end, `group` more of that
// where a tile's rows have to be found first, and for a step of 128 codes `alone` with nothing else on the chip, `busy` with
// a tile on every unit.  Fitted to 10 forms x 36 shapes of 1 to 16384 rows, 10 of them in groups, on several copies of the weights in turn; against the
// same shapes timed anew, its times are off by 9 to 20 % rms by form, and the form that it takes is within 1 % of the fastest for 27 of them, within 10 %
// for 34, and 16 % and 31 % slower for 64 and 256 rows of 4096 x 4096 (2.4 % on average; profiles/linear_form_choice.txt has them all).
struct Form { int BM, BN, per_unit; double end, group, alone, busy; };
constexpr Form kForms[] = {
    {16, 16, 5, 0.29, 1.5, 0.085, 0.039},      // linear_few, from here
    {16, 32, 3, 0.44, 1.6, 0.103, 0.062},
    {16, 64, 4, 0.48, 2.2, 0.212, 0.109},
    {32, 32, 2, 0.88, 1.1, 0.128, 0.088},
    {32, 64, 1, 2.2, 1.2, 0.132, 0.185},
    {64, 64, 1, 3.8, 1.1, 0.210, 0.265},
    {64, 128, 2, 0.94, 1.55, 0.318, 0.346},    // linear_tile, from here
    {128, 128, 1, 2.57, 1.12, 0.383, 0.564},
    {128, 256, 1, 3.39, 0.48, 0.556, 0.907},
    {256, 256, 1, 3.11, 1.71, 1.216, 1.216},
};
// ... where rows begin anywhere or end inside a chunk (20 shapes: off by 11 to 13 % rms, the form within 1 % of the fastest for 14 of them, within 7 %
// for five more and 10 % slower for the last)
constexpr Form kRowForms[] = {
    {16, 16, 4, 0.65, 1.43, 0.116, 0.087},     // linear_few, 8 waves
    {16, 32, 6, 0.31, 1.33, 0.204, 0.142},     // 4 waves
    {32, 32, 5, 0.73, 1.58, 0.250, 0.173},
    {64, 64, 4, 0.96, 1.21, 0.539, 0.406},     // linear_rows, from here
    {64, 128, 3, 1.74, 1.23, 0.702, 0.604},
    {128, 256, 1, 3.72, 1.24, 1.355, 1.862},
};
constexpr int kRowFormCount = sizeof(kRowForms) / sizeof(kRowForms[0]), kShortRowForms = 3;      // (linear_rows: K >= 16)
constexpr double kBytesPerUs = 5.3e6;           // of memory

template <int N>
int fastest_form(const LinearParams& p, const Form (&forms)[N], int among) {
  if (const int forced = tuning().linear_form; forced >= 1 && forced <= among) return forced - 1;
  const double steps = (p.K + 127) / 128, units = compute_units();
  const double groups = groups_of(p), rows = p.M / groups;
  const double memory = (groups * p.N * p.K + (double)p.M * (p.K + 2.0 * p.N)) / kBytesPerUs;
  int best = 0;
  double least = 0;
  for (int i = 0; i < among; ++i) {
    const Form& f = forms[i];
    const double in_group = !p.offsets ? std::ceil(rows / f.BM) : rows <= f.BM / 2 ? 1.0 : rows / f.BM + 0.5;
    const double load = groups * in_group * ((p.N + f.BN - 1) / f.BN) / units, group = p.offsets ? f.group : 0.0;
    const double us = std::max(std::ceil(load / f.per_unit) * (f.end + group + steps * f.alone),
                               (load > 1 ? std::ceil(load) : std::sqrt(std::sqrt(load))) * (f.end + group / f.per_unit + steps * f.busy));
    const double cubes = us * us * us + memory * memory * memory;      // (the longer of the two, and a little of the other)
    if (i == 0 || cubes < least) {
      best = i;
      least = cubes;
    }
  }
  return best;
}

template <typename T>
hipError_t launch_typed(const LinearParams& p, hipStream_t st) {
  if (!direct_ok(p)) {
    switch (fastest_form(p, kRowForms, p.K < 16 ? kShortRowForms : kRowFormCount)) {
      case 0: return launch_few<1, 1, 8, 1, false, int8_t, T>(p, st);
      case 1: return launch_few<1, 2, 4, 1, false, int8_t, T>(p, st);
      case 2: return launch_few<2, 2, 4, 1, false, int8_t, T>(p, st);
      case 3: return launch_rows<1, 4, 4, 1, T>(p, st);
      case 4: return launch_rows<2, 4, 2, 2, T>(p, st);
      default: return launch_rows<4, 4, 2, 4, T>(p, st);
    }
  }
  switch (fastest_form(p, kForms, sizeof(kForms) / sizeof(kForms[0]))) {
    case 0: return launch_few<1, 1, 4, 2, true, int8_t, T>(p, st);
    case 1: return launch_few<1, 2, 4, 2, true, int8_t, T>(p, st);
    case 2: return launch_few<1, 4, 4, 1, true, int8_t, T>(p, st);
    case 3: return launch_few<2, 2, 4, 2, true, int8_t, T>(p, st);
    case 4: return launch_few<2, 4, 4, 2, true, int8_t, T>(p, st);
    case 5: return launch_few<4, 4, 4, 2, true, int8_t, T>(p, st);
    case 6: return launch_tile<2, 4, 2, 2, 3, T>(p, st);
    case 7: return launch_tile<4, 4, 2, 2, 4, T>(p, st);
    case 8: return launch_tile<4, 4, 2, 4, 3, T>(p, st);
    default: return launch_tile<8, 4, 2, 4, 2, T>(p, st);
  }
}

}  // namespace

// Few enough floats for every workgroup to quantise them: with kFloats over all rounds of workgroups on the chip it takes
// less than the launch that it saves (one token of 2048 x 2048 in a graph: 4.2 us, 5.7 as two kernels; called from the host 6.7, and 12.2
// as two calls).
bool linear_takes_floats(const LinearParams& p, int x_type) {
  const int64_t size = x_type == 0 ? 4 : 2, all = (int64_t)p.M * p.K;
  LinearParams codes = p;                // as if tokens were codes on a boundary: the weights are what is asked about
  codes.x = nullptr;
  codes.xs = (p.K + 15) / 16 * 16;
  return p.M <= 16 && all * ((p.N + 8191) / 8192) <= kFloats && direct_ok(codes) && (uintptr_t)p.xf % 16 == 0 &&
         (p.M == 1 || p.xs * size % 16 == 0);
}

hipError_t launch_linear_floats(const LinearParams& p, int x_type, hipStream_t st) {
  return with_type(x_type, [&](auto x) {
    return with_type(p.y_type, [&](auto t) { return launch_few<1, 1, 8, 2, true, decltype(x), decltype(t)>(p, st); });
  });
}

hipError_t launch_linear(const LinearParams& p, hipStream_t st) {
  return with_type(p.y_type, [&](auto t) { return launch_typed<decltype(t)>(p, st); });
}

}  // namespace qasr
