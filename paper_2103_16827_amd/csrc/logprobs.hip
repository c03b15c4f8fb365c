// Log probabilities of given tokens, the entropy and the top alternatives of rows of logits, in one pass over the logits.
//
// A row (or a piece of it, where rows are long or few) belongs to one workgroup, or to one wave where it is short, which reads
// it once into registers.  From there:
//   - the maximum m, then s = sum e^(x - m) and t = sum e^(x - m) (x - m): ln s gives the log probabilities, ln s - t / s the
//     entropy.  Two sweeps over registers instead of a running maximum: one exponential per logit and no rescaling.
//   - the alternatives by a threshold: lane l of every wave owns the logits of column l of the 64, and the `top`-th largest of
//     the 64 columns' maxima is reached by at least `top` logits, and hardly more where the best are spread by chance.  Those
//     are gathered in LDS and ranked by counting.  Where more reach it than there is room for (equal logits, mostly), the
//     best are taken out one after the other instead.
// Pieces leave (m, s, t) and their best in the workspace; a second kernel joins them.
// What bounds it: the logits' way from memory, and next to it about ten vector operations per logit, of which the exponential
// takes four times the others' time.
#include "floats.hpp"
#include "kernels.hpp"
#include "launch_shape.hpp"

namespace qasr {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int kMaxTop = 64;
constexpr int kRoom = 256;          // candidates that are ranked at once

// order of a float as an unsigned number; zeros of either sign are equal
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __builtin_bit_cast(float, o >> 31 ? o & 0x7fffffffu : ~o); }
// larger logits first, equal ones by the lower id; 0 is below every logit
__device__ __forceinline__ uint64_t key_of(float v, int id) { return (uint64_t)order_of(v) << 32 | (uint32_t)~id; }

__device__ __forceinline__ float wave_max(float v) {
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  for (int d = 32; d > 0; d >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)v, d);
    v = o > v ? o : v;
  }
  return v;
}

// Logits per 16 bytes, and the e-th of them
template <typename T>
constexpr int kPer = 16 / (int)sizeof(T);
template <typename T>
__device__ __forceinline__ float logit(const v4u& v, int e) {
  const uint32_t word = v[sizeof(T) == 4 ? e : e >> 1];
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, word);
  else if constexpr (__is_same(T, bf16)) return __builtin_bit_cast(float, e & 1 ? word & 0xffff0000u : word << 16);
  else return (float)__builtin_bit_cast(_Float16, (uint16_t)(word >> (16 * (e & 1))));
}

// the largest of three, in one instruction (fmaxf first makes NaNs quiet, an instruction for each operand)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// what one piece of a row leaves
struct Part { float m, s, t; };

struct Pieces {
  int n;             // pieces of a row
  int len;           // logits of a piece (the last one's may be fewer)
  Part* part;        // [rows][n]
  uint64_t* best;    // [rows][n][top]
};

// the outputs of a row from its (m, s, t); its alternatives' keys, best first, in `best`
template <typename T>
__device__ __forceinline__ void finish(const LogprobParams& p, int64_t row, float m, float s, float t, const uint64_t* best, int tid, int threads) {
  const float ninf = -__builtin_inff(), nan = __builtin_nanf("");
  const bool bad = s != s, none = s == 0.0f;           // a NaN or +infinity; nothing but -infinity
  const float base = none ? 0.0f : m, ls = __logf(s);
  auto score = [&](float x) { return bad ? nan : none ? ninf : (x - base) - ls; };
  const T* x = (const T*)p.x + row * p.xs;
  for (int j = tid; j < p.n; j += threads) {
    const int tok = p.tokens[row * p.n + j];
    p.logprob[row * p.n + j] = tok < 0 ? 0.0f : tok >= p.V ? nan : score(to_float(x[tok]));
  }
  if (tid == 0 && p.entropy) p.entropy[row] = bad ? nan : none ? 0.0f : ls - t / s;
  if (tid < p.top) {
    const uint64_t k = best[tid];
    p.top_ids[row * p.top + tid] = bad ? -1 : (int)~(uint32_t)k;
    p.top_logprob[row * p.top + tid] = score(value_of((uint32_t)(k >> 32)));
  }
}

// LDS of a choice of the best
template <int W>
struct Choice {
  uint32_t column[64];               // the largest number in each column
  uint64_t cand[kRoom];
  uint64_t best[kMaxTop];            // the outcome, best first
  uint64_t wave_best[W];
  int count;
};

template <int W>
__device__ __forceinline__ void sync() {
  if constexpr (W > 1) __syncthreads();
  else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// The `top` largest of the keys that W waves hold, at least that many.  own: the order of the thread's largest; each(limit, f)
// calls f(key) for each of its keys of an order of `limit` or more, or for more of them.  c.column and c.count were cleared, with a sync
// after that.
template <int W, typename Each>
__device__ __forceinline__ void choose(Choice<W>& c, int top, uint32_t own, int tid, Each&& each) {
  const int lane = tid & 63;
  atomicMax(&c.column[lane], own);
  sync<W>();
  // the largest number that at least `top` of the columns reach, bit by bit (every wave for itself)
  const uint32_t mine = c.column[lane];
  uint32_t limit = 0;
  if (top < 64) {
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t higher = limit | 1u << bit;
      if (__popcll(__ballot(mine >= higher)) >= top) limit = higher;
    }
  } else {
    limit = mine;
    for (int d = 32; d > 0; d >>= 1) limit = min(limit, (uint32_t)__shfl_xor((int)limit, d));
  }
  if (own >= limit) {
    each(limit, [&](uint64_t key) {
      const int to = atomicAdd(&c.count, 1);
      if (to < kRoom) c.cand[to] = key;
    });
  }
  sync<W>();
  const int found = c.count;
  if (found <= kRoom) {
    for (int i = tid; i < found; i += 64 * W) {
      const uint64_t k = c.cand[i];
      int rank = 0;
      for (int o = 0; o < found; ++o) rank += c.cand[o] > k;
      if (rank < top) c.best[rank] = k;
    }
  } else {
    // one after the other: every thread offers its best that is still to come
    uint64_t last = ~0ull;
    for (int j = 0; j < top; ++j) {
      uint64_t b = 0;
      each(0, [&](uint64_t key) { b = key < last && key > b ? key : b; });
      b = wave_max(b);
      if constexpr (W > 1) {
        sync<W>();
        if (lane == 0) c.wave_best[tid >> 6] = b;
        sync<W>();
#pragma unroll
        for (int w = 0; w < W; ++w) b = c.wave_best[w] > b ? c.wave_best[w] : b;
      }
      last = b;
      if (tid == 0) c.best[j] = b;
    }
  }
  sync<W>();
}

// W waves a row or piece, R loads of 16 bytes a lane: up to 64 W R kPer logits.  W == 1: four rows a workgroup, a wave each.
template <typename T, int W, int R>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void logprobs_kernel(LogprobParams p, Pieces c) {
  constexpr int N = kPer<T>, kRows = W == 1 ? 4 : 1;
  __shared__ float part[kRows][3 * W];
  __shared__ Choice<W> choices[kRows];
  const int sub = W == 1 ? threadIdx.x >> 6 : 0;       // the row among the workgroup's
  const int tid = W == 1 ? threadIdx.x & 63 : threadIdx.x, lane = threadIdx.x & 63, wave = tid >> 6;
  const int64_t unit = (((int64_t)blockIdx.y << kGridShift) + blockIdx.x) * kRows + sub;
  if (unit >= p.rows * c.n) return;                    // (W == 1: no barriers below)
  const int64_t row = c.n == 1 ? unit : unit / c.n;
  const int piece = c.n == 1 ? 0 : (int)(unit - row * c.n);
  const int v0 = piece * c.len, len = min(c.len, p.V - v0);
  const T* x = (const T*)p.x + row * p.xs + v0;
  Choice<W>& choice = choices[sub];

  const float ninf = -__builtin_inff();
  // Whole loads, and what is left of the row, a logit for each of the first threads.  Lanes past the end hold -infinity.
  const int loads = len / N, rest = loads * N + tid;
  struct __attribute__((packed, aligned(sizeof(T)))) Load { v4u v; };
  v4u raw[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : __is_same(T, bf16) ? 0xff80ff80u : 0xfc00fc00u;
    raw[i] = (v4u){kNone, kNone, kNone, kNone};
    if (i * 64 * W + tid < loads) raw[i] = reinterpret_cast<const Load*>(x + (i * 64 * W + tid) * N)->v;
  }
  const float last = rest < len ? to_float(x[rest]) : ninf;
  // calls f(a, b, place of a, whether they are logits) for the lane's logits, two neighbours at a time
  auto sweep = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      asm volatile("" : "+v"(raw[i]));                 // (taken apart anew in every sweep: as floats they would need up to twice the registers)
      if (i * 64 * W < loads) {
#pragma unroll
        for (int k = 0; k < N; k += 2) f(logit<T>(raw[i], k), logit<T>(raw[i], k + 1), (i * 64 * W + tid) * N + k, i * 64 * W + tid < loads);
      }
    }
  };
  float m = last;
  sweep([&](float a, float b, int, bool) { m = max3(m, a, b); });
  const float own = m;                                 // of this thread's logits
  m = wave_max(m);
  if (p.top > 0) {
    if (tid < 64) choice.column[lane] = 0;
    if (tid == 0) choice.count = 0;
  }
  if constexpr (W > 1) {
    if (lane == 0) part[0][wave] = m;
    sync<W>();
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, part[0][w]);
  }
  const float base = m == ninf ? 0.0f : m;             // (nothing but -infinity: every exponential is 0)
  float s = 0.0f, t = 0.0f;
  auto add = [&](float v) __attribute__((always_inline)) {
    const float d = v - base, e = __expf(d);
    s += e;
    t = fmaf(e, fmaxf(d, -1000.0f), t);                // (not 0 times -infinity)
  };
  sweep([&](float a, float b, int, bool) {
    add(a);
    add(b);
  });
  add(last);
  s = wave_sum(s);
  t = wave_sum(t);
  if constexpr (W > 1) {
    if (lane == 0) {
      part[0][W + wave] = s;
      part[0][2 * W + wave] = t;
    }
    if (p.top == 0) sync<W>();                         // (else the choice has one)
  }
  const int top = min(p.top, len);                     // (a piece may be shorter than that)
  if (p.top > 0)
    choose<W>(choice, top, order_of(own), tid, [&](uint32_t limit, auto&& f) __attribute__((always_inline)) {
      const float least = limit == 0 ? ninf : value_of(limit);
      sweep([&](float a, float b, int at, bool there) {
        if (!(a < least) && there) f(key_of(a, v0 + at));
        if (!(b < least) && there) f(key_of(b, v0 + at + 1));
      });
      if (!(last < least) && rest < len) f(key_of(last, v0 + rest));
    });
  if constexpr (W > 1) {
    s = t = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      s += part[0][W + w];
      t += part[0][2 * W + w];
    }
  }
  if (c.n == 1) {
    finish<T>(p, row, m, s, t, choice.best, tid, 64 * W);
    return;
  }
  if (tid == 0) c.part[unit] = Part{m, s, t};
  if (tid < p.top) c.best[unit * p.top + tid] = tid < top ? choice.best[tid] : 0;
}

// A workgroup joins the pieces of a row.
constexpr int kJoinWaves = 4, kHeld = 16;              // keys that a thread holds
template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void join_kernel(LogprobParams p, Pieces c) {
  __shared__ Choice<kJoinWaves> choice;
  const int64_t row = ((int64_t)blockIdx.y << kGridShift) + blockIdx.x;
  if (row >= p.rows) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const uint64_t* keys = c.best + row * c.n * p.top;
  const int64_t n = (int64_t)c.n * p.top;
  uint64_t held[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = i * 64 * kJoinWaves + tid < n ? keys[i * 64 * kJoinWaves + tid] : 0;
  const float ninf = -__builtin_inff();
  float m = ninf;
  for (int i = lane; i < c.n; i += 64) m = fmaxf(m, c.part[row * c.n + i].m);
  m = wave_max(m);
  const float base = m == ninf ? 0.0f : m;
  float s = 0.0f, t = 0.0f;
  for (int i = lane; i < c.n; i += 64) {
    const Part q = c.part[row * c.n + i];
    // (a piece without a logit above -infinity adds nothing: its s and t are 0)
    const float d = (q.m == ninf ? base : q.m) - base, f = __expf(d);
    s += q.s * f;
    t += f * fmaf(q.s, fmaxf(d, -1000.0f), q.t);
  }
  s = wave_sum(s);
  t = wave_sum(t);
  if (p.top > 0) {
    if (tid < 64) choice.column[lane] = 0;
    if (tid == 0) choice.count = 0;
    sync<kJoinWaves>();
    auto each = [&](uint32_t limit, auto&& f) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (held[i] != 0 && (uint32_t)(held[i] >> 32) >= limit) f(held[i]);
      for (int64_t i = kHeld * 64 * kJoinWaves + tid; i < n; i += 64 * kJoinWaves)
        if (keys[i] != 0 && (uint32_t)(keys[i] >> 32) >= limit) f(keys[i]);
    };
    uint64_t own = 0;
    each(0, [&](uint64_t k) { own = k > own ? k : own; });
    choose<kJoinWaves>(choice, p.top, (uint32_t)(own >> 32), tid, each);
  }
  finish<T>(p, row, m, s, t, choice.best, tid, 64 * kJoinWaves);
}

int size_of(int type) { return type == 0 ? 4 : 2; }

// Bytes of logits that the largest workgroup takes: 16 waves of 8 loads a lane.
constexpr int kWhole = 16 * 64 * 8 * 16;

Pieces pieces_of(int64_t rows, int V, int bytes) {
  Pieces c{};
  const int64_t all = (int64_t)V * bytes;
  int64_t n = (all + kWhole - 1) / kWhole;
  // few long rows: pieces for the whole chip, of 8 KiB and more
  const int64_t want = 256 / rows, most = (all + 8191) / 8192;
  if (want > n) n = want < most ? want : most > n ? most : n;
  const int per = 16 / bytes;
  c.len = (int)(((V + n - 1) / n + per - 1) / per * per);
  c.n = (int)((V + (int64_t)c.len - 1) / c.len);
  return c;
}

}  // namespace

size_t logprobs_workspace_bytes(int64_t rows, int V, int top) {
  size_t most = 0;
  for (int bytes = 2; bytes <= 4; bytes += 2) {
    const Pieces c = rows > 0 ? pieces_of(rows, V, bytes) : Pieces{1};
    const size_t need = c.n == 1 ? 0 : (size_t)rows * c.n * (16 + 8 * (size_t)top);
    most = need > most ? need : most;
  }
  return (most + 255) & ~(size_t)255;
}

hipError_t launch_logprobs(const LogprobParams& p, int x_type, void* workspace, hipStream_t st) {
  const int bytes = size_of(x_type);
  Pieces c = pieces_of(p.rows, p.V, bytes);
  if (c.n > 1) {
    c.best = (uint64_t*)workspace;
    c.part = (Part*)(c.best + (size_t)p.rows * c.n * p.top);
  }
  return with_type(x_type, [&](auto t) {
    using T = decltype(t);
    const int64_t units = p.rows * c.n;
    const int loads = c.len / kPer<T>;                           // of 16 bytes, of a piece
    hipError_t e;
    auto launch = [&](auto kernel, int waves) {
      const GridShape g = grid_shape(waves == 1 ? (units + 3) / 4 : units);
      return launch_kernel(kernel, dim3(g.x, g.y), dim3(waves == 1 ? 256 : 64 * waves), 0, st, p, c);
    };
    if (loads <= 64) e = launch(logprobs_kernel<T, 1, 1>, 1);
    else if (loads <= 256) e = launch(logprobs_kernel<T, 1, 4>, 1);
    else if (loads <= 512) e = launch(logprobs_kernel<T, 4, 2>, 4);
    else if (loads <= 1024) e = launch(logprobs_kernel<T, 4, 4>, 4);
    else if (loads <= 2048) e = launch(logprobs_kernel<T, 4, 8>, 4);
    else if (loads <= 4096) e = launch(logprobs_kernel<T, 8, 8>, 8);
    else e = launch(logprobs_kernel<T, 16, 8>, 16);
    if (e != hipSuccess || c.n == 1) return e;
    const GridShape g = grid_shape(p.rows);
    return launch_kernel(join_kernel<T>, dim3(g.x, g.y), dim3(64 * kJoinWaves), 0, st, p, c);
  });
}

}  // namespace qasr
