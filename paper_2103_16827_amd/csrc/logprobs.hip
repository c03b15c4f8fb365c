// Log probabilities of given tokens, the entropy and the top alternatives of rows of logits, in one pass over the logits.
//
// A row (or a piece of it, where rows are long or few) belongs to one workgroup, or to one wave where it is short, which reads
// it once into registers.  From there:
//   - the maximum m, then s = sum e^(x - m) and t = sum e^(x - m) (x - m): ln s gives the log probabilities, ln s - t / s the
//     entropy.  Two sweeps over registers instead of a running maximum: one exponential per logit and no rescaling.
//   - the alternatives by a threshold.  Threads are columns, 64 of them or four times as many (some threads each): the `top`-th
//     largest of the columns' maxima is reached by `top` logits at least, and hardly more where the best are spread by
//     chance.  The few threads whose maximum reaches it put their logits in LDS, where all threads look for those
//     that do; these are ranked by counting.  Where they are too many for the room, most often because the best end among equal
//     logits (a mask of -infinity or of the type's lowest value that leaves fewer than `top`), the larger ones are taken, and of the
//     equal ones those up to a limit on their ids, found in the same way.  Where these are too many as well (hundreds of
//     unequal logits in few columns), the best are taken out one after the other, from memory.
// Pieces leave (m, s, t) and their best in the workspace; a second kernel joins them.
// What bounds it: the logits' way from memory, and next to it about eleven vector operations per logit, of which the
// exponential takes four times the others' time.  4096 rows of 50257 bf16 logits 73 us (5.6 TB/s), with 5 alternatives 79, with 20 81;
// 64 of 151936 fp16 11.3 and with 20 alternatives 15.1 (12.3 and 16.0 from memory); 1 of 128256 float32 5.4 and 10.3, of which a launch and its
// first loads are half, the second kernel another half.  With 3 logits left of 50257 and 20 alternatives, 512 rows take 43 us for 20 (657 when they
// were taken out one after the other).
// The exponential and the logarithm are the hardware's (__expf, __logf: an ulp of their own, and of an exponential's argument d another 2^-24 |d|): an
// exponential that matters has a small |d|, and a sum's rounding is of the same size.
#include "floats.hpp"
#include "kernels.hpp"
#include "lanes.hpp"
#include "launch_shape.hpp"
#include <algorithm>

namespace qasr {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int kRoom = 512;          // candidates that are ranked at once

// order of a float as an unsigned number; zeros of either sign are equal
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __builtin_bit_cast(float, o >> 31 ? o & 0x7fffffffu : ~o); }
// larger logits first, equal ones by the lower id; 0 is below every logit
__device__ __forceinline__ uint64_t key_of(float v, int id) { return (uint64_t)order_of(v) << 32 | (uint32_t)~id; }

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

// a given token and its logit
struct Ahead {
  int tok = -1;
  float x = 0.0f;
  __device__ __forceinline__ void ask(const LogprobParams& p, int64_t row, int j) {
    if (j < p.n) tok = p.tokens[row * p.n + j];
  }
  template <typename T>
  __device__ __forceinline__ void look(const LogprobParams& p, int64_t row) {
    if (tok >= 0 && tok < p.V) x = to_float(((const T*)p.x + row * p.xs)[tok]);
  }
  template <typename T>
  __device__ __forceinline__ void load(const LogprobParams& p, int64_t row, int j) {
    ask(p, row, j);
    look<T>(p, row);
  }
};

// the outputs of a row from its (m, s, t)
struct Scorer {
  float base, ls, entropy;
  bool bad, none;              // a NaN or +infinity; nothing but -infinity
  __device__ __forceinline__ Scorer(float m, float s, float t) {
    bad = s != s;
    none = s == 0.0f;
    base = none ? 0.0f : m;
    ls = __logf(s);
    entropy = bad ? __builtin_nanf("") : none ? 0.0f : ls - t / s;
  }
  __device__ __forceinline__ float operator()(float x) const {
    return bad ? __builtin_nanf("") : none ? -__builtin_inff() : (x - base) - ls;
  }
  // the entropy and the given tokens' scores; `ahead`: the thread's first token, asked for when the kernel began
  template <typename T>
  __device__ __forceinline__ void tokens(const LogprobParams& p, int64_t row, int tid, int threads, Ahead ahead) const {
    for (int j = tid; j < p.n; j += threads) {
      if (j != tid) ahead.load<T>(p, row, j);
      p.logprob[row * p.n + j] = ahead.tok < 0 ? 0.0f : ahead.tok >= p.V ? __builtin_nanf("") : (*this)(ahead.x);
    }
    if (tid == 0 && p.entropy) p.entropy[row] = entropy;
  }
  // the alternative of rank j
  __device__ __forceinline__ void alternative(const LogprobParams& p, int64_t row, int j, uint64_t key) const {
    p.top_ids[row * p.top + j] = bad ? -1 : (int)~(uint32_t)key;
    p.top_logprob[row * p.top + j] = (*this)(value_of((uint32_t)(key >> 32)));
  }
};

template <int W>
__device__ __forceinline__ void sync() {
  if constexpr (W > 1) __syncthreads();
  else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// LDS of a choice of the best: the largest number in each column, and the candidates
template <int W>
struct Choice {
  static constexpr int kQuarters = 4;                  // columns / 64, where there are many (`wide`)
  __align__(16) uint32_t column[64 * kQuarters];
  uint64_t cand[kRoom];
  uint64_t wave_best[W];
  int count, holders;
  uint32_t least;                    // what limit() said

  __device__ __forceinline__ void clear(int tid) {
    if (tid < 64) {
#pragma unroll
      for (int q = 0; q < kQuarters; ++q) column[64 * q + tid] = 0;
    }
    if (tid == 0) count = holders = 0;
  }
  // own: the order of the thread's largest.  (A sync comes before it and after it.)
  __device__ __forceinline__ void offer(bool wide, uint32_t own, int tid) {
    atomicMax(&column[(tid & 63) + (wide ? 64 * ((tid >> 6) % kQuarters) : 0)], own);
  }
  // One wave: the largest number that at least n of the columns reach, 0 if there is none (where there are four times 64 in its bits from
  // `low` on).
  __device__ __forceinline__ uint32_t limit(bool wide, int n, int low) const {
    const int lane = threadIdx.x & 63;
    if (!wide) {
      const uint32_t mine = column[lane];
      int above = 0;
#pragma unroll 2
      for (int o = 0; o < 64; o += 4) {
        const v4u c = *reinterpret_cast<const v4u*>(column + o);
        above += (c[0] > mine) + (c[1] > mine) + (c[2] > mine) + (c[3] > mine);
      }
      return wave_min(above < n ? mine : ~0u);
    }
    uint32_t mine[kQuarters], found = 0;
#pragma unroll
    for (int q = 0; q < kQuarters; ++q) mine[q] = column[64 * q + lane];
    for (int bit = 31; bit >= low; --bit) {
      const uint32_t higher = found | 1u << bit;
      int reach = 0;
#pragma unroll
      for (int q = 0; q < kQuarters; ++q) reach += __popcll(__ballot(mine[q] >= higher));
      if (reach >= n) found = higher;
    }
    return found;
  }
  // The candidates where those that reach the limit are too many, most often because the `top` best end among equal logits (a mask that
  // leaves fewer than `top`): the larger ones, and of the equal ones those whose ids reach a limit found in the same way.  each(f)
  // calls f(order, ~id) for the thread's logits.  False if these are too many as well.  (A sync comes before it.)
  template <typename Each>
  __device__ __forceinline__ bool among_equals(bool wide, int top, int tid, Each&& each) {
    if (W == 1 || tid < 64) {
      const uint32_t l = limit(wide, top, 0);
      if ((tid & 63) == 0) least = l;
    }
    sync<W>();
    const uint32_t value = least;
    clear(tid);
    sync<W>();
    uint32_t first = 0;
    each([&](uint32_t order, uint32_t id) __attribute__((always_inline)) {
      if (order > value) add((uint64_t)order << 32 | id);
      else if (order == value) first = max(first, id);
    });
    offer(wide, first, tid);
    sync<W>();
    const int larger = count;
    if (larger > kRoom) return false;
    if (W == 1 || tid < 64) {
      const uint32_t l = larger < top ? limit(wide, top - larger, 0) : ~0u;
      if ((tid & 63) == 0) least = l;
    }
    sync<W>();
    const uint32_t lowest = least;
    each([&](uint32_t order, uint32_t id) __attribute__((always_inline)) {
      if (order == value && id >= lowest) add((uint64_t)order << 32 | id);
    });
    sync<W>();
    return count <= kRoom;
  }
  __device__ __forceinline__ void add(uint64_t key) {
    const int to = atomicAdd(&count, 1);
    if (to < kRoom) cand[to] = key;
  }
  // Calls f(rank, key) for the `top` best candidates.  (A sync comes before it.)
  template <typename F>
  __device__ __forceinline__ void rank(int top, int tid, F&& f) const {
    constexpr int B = kRoom > 64 * W ? (kRoom / (64 * W) < 4 ? kRoom / (64 * W) : 4) : 1;
    const int found = count;
    if (found <= 64 * W) rank_some<1>(top, tid, found, f);
    else for (int i = tid; i < found; i += 64 * W * B) rank_some<B>(top, i, found, f);
  }
  // ... of the candidates i, i + 64 W ..: each that is read is compared with B
  template <int B, typename F>
  __device__ __forceinline__ void rank_some(int top, int i, int found, F&& f) const {
    uint64_t k[B];
    int r[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      k[b] = i + b * 64 * W < found ? cand[i + b * 64 * W] : 0;
      r[b] = 0;
    }
    if (k[0] == 0) return;
    for (int o = 0; o < found; ++o) {
      const uint64_t other = cand[o];
#pragma unroll
      for (int b = 0; b < B; ++b) r[b] += other > k[b];
    }
#pragma unroll
    for (int b = 0; b < B; ++b)
      if (k[b] != 0 && r[b] < top) f(r[b], k[b]);
  }
  // The same for all keys next(i), i = tid, tid + 64 W .. < n, one after the other
  template <typename Next, typename F>
  __device__ __forceinline__ void one_by_one(int top, int n, int tid, Next&& next, F&& f) {
    uint64_t last = ~0ull;
    for (int j = 0; j < top; ++j) {
      uint64_t b = 0;
#pragma unroll 1
      for (int i = tid; i < n; i += 64 * W) {
        const uint64_t key = next(i);
        b = key < last && key > b ? key : b;
      }
      b = wave_max(b);
      if constexpr (W > 1) {
        sync<W>();
        if ((tid & 63) == 0) wave_best[tid >> 6] = b;
        sync<W>();
        b = wave_max(wave_best[tid % W]);
      }
      last = b;
      if (tid == 0) f(j, b);
    }
  }
};

// W waves a row or piece, R loads of 16 bytes a lane: up to 64 W R kPer logits.  W == 1: four rows a workgroup, a wave each.
template <typename T, int W, int R>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void logprobs_kernel(LogprobParams p, Pieces c) {
  constexpr int N = kPer<T>, kRows = W == 1 ? 4 : 1;
  constexpr int kHolders = W == 1 ? 32 : 128;          // threads whose logits fit the LDS at once
  __shared__ float part[kRows][3 * W];
  __shared__ Choice<W> choices[kRows];
  __shared__ v4u held[kRows][kHolders * R];
  __shared__ float held_last[kRows][kHolders];
  __shared__ int holder[kRows][kHolders];
  const int sub = W == 1 ? threadIdx.x >> 6 : 0;       // the row among the workgroup's
  const int tid = W == 1 ? threadIdx.x & 63 : threadIdx.x, lane = threadIdx.x & 63, wave = tid >> 6;
  const int64_t unit = (((int64_t)blockIdx.y << kGridShift) + blockIdx.x) * kRows + sub;
  if (unit >= p.rows * c.n) return;                    // (W == 1: no barriers below)
  int64_t row = unit;
  int piece = 0;
  if (c.n > 1) {
    row = unit >> 31 ? unit / c.n : (int64_t)((uint32_t)unit / (uint32_t)c.n);
    piece = (int)(unit - row * c.n);
  }
  const int v0 = piece * c.len, len = min(c.len, p.V - v0);
  const T* x = (const T*)p.x + row * p.xs + v0;
  Choice<W>& choice = choices[sub];
  const int top = min(p.top, len);                     // (a piece may be shorter than p.top)

  // Whole loads from a 16-byte boundary on, and what is before and behind them, a logit for each of the first threads.  Lanes
  // past the end hold -infinity.  (Loads that straddle boundaries ran at three quarters of the rate.)
  const float ninf = -__builtin_inff();
  const int head = min(len, (int)(-(uintptr_t)x & 15) / (int)sizeof(T));
  const int loads = (len - head) / N, rest = tid < head ? tid : loads * N + tid;
  const v4u* aligned = reinterpret_cast<const v4u*>(x + head);
  v4u raw[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : __is_same(T, bf16) ? 0xff80ff80u : 0xfc00fc00u;
    raw[i] = (v4u){kNone, kNone, kNone, kNone};
    if (i * 64 * W + tid < loads) raw[i] = aligned[i * 64 * W + tid];
  }
  const float last = rest < len ? to_float(x[rest]) : ninf;
  Ahead ahead;
  if (c.n == 1) ahead.load<T>(p, row, tid);
  if (top > 0) {
    choice.clear(tid);
    sync<W>();                                         // (the logits are on their way)
  }
  // calls f(a, b) for the lane's logits, two neighbours at a time
  auto sweep = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      asm volatile("" : "+v"(raw[i]));                 // (taken apart anew in every sweep: as floats they would need up to twice the registers)
      if (i * 64 * W < loads) {
#pragma unroll
        for (int k = 0; k < N; k += 2) f(logit<T>(raw[i], k), logit<T>(raw[i], k + 1));
      }
    }
  };
  float m = last;
  sweep([&](float a, float b) { m = max3(m, a, b); });
  const uint32_t own = order_of(m);                    // of this thread's logits
  m = wave_max(m);
  // Four times 64 columns for many alternatives, and for a wave on its own where few of its lanes hold logits; there a lane's loads,
  // or the words of its only one, are four.
  const bool by_load = W == 1 && (top > 24 || loads < 2 * top), wide = top > 24 || by_load;
  if (by_load) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float most = q == 0 ? last : ninf;
      if constexpr (R == 1) {
#pragma unroll
        for (int k = q * N / 4; k < (q + 1) * N / 4; ++k) most = fmaxf(most, logit<T>(raw[0], k));
      } else {
#pragma unroll
        for (int k = 0; k < N; ++k) most = fmaxf(most, logit<T>(raw[q % R], k));
      }
      choice.column[64 * q + lane] = order_of(most);
    }
  } else if (top > 0) {
    choice.offer(wide, own, tid);
  }
  if constexpr (W > 1) {
    if (lane == 0) part[0][wave] = m;
  }
  sync<W>();
  if constexpr (W > 1) m = wave_max(part[0][lane % W]);
  if (top > 0 && (W == 1 || wave == 0)) {              // (meanwhile the others go on)
    const uint32_t l = choice.limit(wide, top, 12);
    if (lane == 0) choice.least = l;
  }
  const float base = m == ninf ? 0.0f : m;             // (nothing but -infinity: every exponential is 0)
  float s = 0.0f, t = 0.0f;
  auto add = [&](float v) __attribute__((always_inline)) {
    const float d = v - base, e = __expf(d);
    s += e;
    t = fmaf(e, fmaxf(d, -1000.0f), t);                // (not 0 times -infinity)
  };
  sweep([&](float a, float b) {
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
  }
  sync<W>();
  if constexpr (W > 1) {
    s = wave_sum(lane < W ? part[0][W + lane] : 0.0f);
    t = wave_sum(lane < W ? part[0][2 * W + lane] : 0.0f);
  }
  const uint32_t limit = top > 0 ? choice.least : 0;
  if (top > 0 && !by_load && own >= limit && (tid < loads || rest < len)) {
    const int h = atomicAdd(&choice.holders, 1);
    if (h < kHolders) {
#pragma unroll
      for (int i = 0; i < R; ++i) held[sub][h * R + i] = raw[i];
      held_last[sub][h] = last;
      holder[sub][h] = tid;
    }
  }
  const Scorer score(m, s, t);
  if (c.n == 1) score.template tokens<T>(p, row, tid, 64 * W, ahead);
  else if (tid == 0) c.part[unit] = Part{m, s, t};
  if (top == 0) return;
  if (score.bad) {                                     // (who joins the pieces asks for none of this one's)
    if (c.n == 1 && tid < top) score.alternative(p, row, tid, 0);
    return;
  }
  sync<W>();

  auto leave = [&](int j, uint64_t key) __attribute__((always_inline)) {
    if (c.n == 1) score.alternative(p, row, j, key);
    else c.best[unit * p.top + j] = key;
  };
  // calls f(order, ~id) for the thread's logits (read again, but by a wave on its own: few rows come here, and registers are short)
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    auto all_of = [&](const v4u& v, int at) __attribute__((always_inline)) {
      if (at >= loads) return;
#pragma unroll
      for (int k = 0; k < N; ++k) f(order_of(logit<T>(v, k)), (uint32_t)~(v0 + head + at * N + k));
    };
    if constexpr (W == 1) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        asm volatile("" : "+v"(raw[i]));
        all_of(raw[i], i * 64 + tid);
      }
    } else {
#pragma unroll 4
      for (int at = tid; at < loads; at += 64 * W) all_of(aligned[at], at);
    }
    if (rest < len) f(order_of(last), (uint32_t)~(v0 + rest));
  };
  const int holders = choice.holders;
  bool fits = holders <= kHolders;
  if (by_load) {
    each([&](uint32_t order, uint32_t id) __attribute__((always_inline)) {
      if (order >= limit) choice.add((uint64_t)order << 32 | id);
    });
    sync<W>();
    fits = choice.count <= kRoom;
  } else if (fits) {
    // a load of a holder for each thread, then the holders' last logits
    for (int i = tid; i < holders * R; i += 64 * W) {
      const int h = i / R, at = ((i % R) * 64 * W + holder[sub][h]);
      const v4u v = held[sub][i];
      if (at < loads) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float f = logit<T>(v, k);
          if (order_of(f) >= limit) choice.add(key_of(f, v0 + head + at * N + k));
        }
      }
    }
    for (int h = tid; h < holders; h += 64 * W) {
      const int at = holder[sub][h] < head ? holder[sub][h] : loads * N + holder[sub][h];
      if (at < len && order_of(held_last[sub][h]) >= limit) choice.add(key_of(held_last[sub][h], v0 + at));
    }
    sync<W>();
    fits = choice.count <= kRoom;
  }
  if (!fits) fits = choice.among_equals(wide, top, tid, each);
  if (fits) choice.rank(top, tid, leave);
  else choice.one_by_one(top, len, tid, [&](int i) { return key_of(to_float(x[i]), v0 + i); }, leave);
  if (c.n > 1 && tid >= top && tid < p.top) c.best[unit * p.top + tid] = 0;
}

// Rows of up to B G = 16, 32, 64, 128 or 256 logits: G lanes of B logits each (l, G + l, ..), 64 / G rows a wave.  Reductions by
// exchanges within 16 lanes; the alternatives one after the other, or (B == 4) their ranks by comparing every logit with all.
// Bound by the instructions: 25600 rows of 29 float32 logits and 3 alternatives 4.5 us, with a lane for every logit and two to
// eight times the exchanges 6.5.
template <int G, typename V, typename Op>
__device__ __forceinline__ V row_reduce(V v, Op op) {
  auto moved = [&](auto ctrl) __attribute__((always_inline)) {
    constexpr int C = decltype(ctrl)::value;
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    return __builtin_bit_cast(V, lane_move<C, 0xf>(b, b));
  };
  using std::integral_constant;
  v = op(v, moved(integral_constant<int, 0xb1>()));    // neighbours, pairs, halves of eight, of sixteen
  v = op(v, moved(integral_constant<int, 0x4e>()));
  if constexpr (G >= 8) v = op(v, moved(integral_constant<int, 0x141>()));
  if constexpr (G >= 16) v = op(v, moved(integral_constant<int, 0x140>()));
  return v;
}

template <typename T, int G, int B>
__global__ __launch_bounds__(256) void logprobs_small_kernel(LogprobParams p) {
  constexpr int kRows = 64 / G;
  __shared__ __align__(16) uint32_t orders[4][B == 4 ? 64 * B : 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane % G;
  const int64_t row = ((((int64_t)blockIdx.y << kGridShift) + blockIdx.x) * 4 + wave) * kRows + lane / G;
  if (row >= p.rows) return;                           // (no barriers below)
  const float ninf = -__builtin_inff();
  float x[B];
#pragma unroll
  for (int b = 0; b < B; ++b) x[b] = b * G + l < p.V ? to_float(((const T*)p.x + row * p.xs)[b * G + l]) : ninf;
  Ahead ahead;
  ahead.load<T>(p, row, l);
  float m = x[0];
#pragma unroll
  for (int b = 1; b < B; ++b) m = fmaxf(m, x[b]);
  m = row_reduce<G>(m, [](float a, float b) { return fmaxf(a, b); });
  const float base = m == ninf ? 0.0f : m;
  float s = 0.0f, t = 0.0f;
#pragma unroll
  for (int b = 0; b < B; ++b) {
    const float d = x[b] - base, e = __expf(d);
    s += e;
    t = fmaf(e, fmaxf(d, -1000.0f), t);
  }
  s = row_reduce<G>(s, [](float a, float b) { return a + b; });
  t = row_reduce<G>(t, [](float a, float b) { return a + b; });
  const Scorer score(m, s, t);
  score.template tokens<T>(p, row, l, G, ahead);
  if (p.top == 0) return;
  if (score.bad) {
    for (int j = l; j < p.top; j += G) score.alternative(p, row, j, 0);
    return;
  }
  uint32_t own[B];                                     // 0: no logit, or taken
#pragma unroll
  for (int b = 0; b < B; ++b) own[b] = b * G + l < p.V ? order_of(x[b]) : 0;
  if (B > 4 || 4 * p.top < p.V) {
    // few: taken out one after the other, of equal ones the lowest
    for (int j = 0; j < p.top; ++j) {
      auto most_of = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
      uint32_t most = own[0];
#pragma unroll
      for (int b = 1; b < B; ++b) most = most_of(most, own[b]);
      most = row_reduce<G>(most, most_of);
      uint32_t id = ~0u;
#pragma unroll
      for (int b = B - 1; b >= 0; --b) id = own[b] == most ? b * G + l : id;
      id = row_reduce<G>(id, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
      if (id % G == l) score.alternative(p, row, j, (uint64_t)most << 32 | ~id);
#pragma unroll
      for (int b = 0; b < B; ++b) own[b] = b * G + l == id ? 0 : own[b];
    }
    return;
  }
  if constexpr (B == 4) {
    uint32_t* all = &orders[wave][lane / G * G * B];
#pragma unroll
    for (int b = 0; b < B; ++b) all[b * G + l] = own[b];
    sync<1>();
    int rank[B] = {};
#pragma unroll 1
    for (int o = 0; o < p.V; o += 4) {                 // (past the row there are zeros)
      const v4u c = *reinterpret_cast<const v4u*>(all + o);
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) rank[b] += c[k] > own[b] - (uint32_t)(o + k < b * G + l);      // (an equal one before it is ahead)
    }
#pragma unroll
    for (int b = 0; b < B; ++b)
      if (rank[b] < p.top && b * G + l < p.V) score.alternative(p, row, rank[b], (uint64_t)own[b] << 32 | (uint32_t)~(b * G + l));
  }
}

// A workgroup joins the pieces of a row.
constexpr int kJoinWaves = 4, kHeld = 16;              // keys that a thread holds
template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void join_kernel(LogprobParams p, Pieces c) {
  constexpr int W = kJoinWaves;
  __shared__ Choice<W> choice;
  const int64_t row = ((int64_t)blockIdx.y << kGridShift) + blockIdx.x;
  if (row >= p.rows) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const float ninf = -__builtin_inff();
  // (a token, keys and parts are on their way together: what is waited for here is two loads one after the other)
  Ahead ahead;
  ahead.ask(p, row, tid);
  const uint64_t* keys = c.best + row * c.n * p.top;
  const int n = c.n * p.top;
  uint64_t held[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    // (a piece's keys are in order: with the rotation a thread holds some of every rank where 64 W is a multiple of p.top too)
    const int at = i * 64 * W + (tid + 37 * i) % (64 * W);
    held[i] = at < n ? keys[at] : 0;
  }
  const Part mine = lane < c.n ? c.part[row * c.n + lane] : Part{ninf, 0.0f, 0.0f};
  ahead.look<T>(p, row);
  float m = mine.m;
  for (int i = lane + 64; i < c.n; i += 64) m = fmaxf(m, c.part[row * c.n + i].m);
  m = wave_max(m);
  const float base = m == ninf ? 0.0f : m;
  float s = 0.0f, t = 0.0f;
  for (int i = lane; i < c.n; i += 64) {
    const Part q = i == lane ? mine : c.part[row * c.n + i];
    // (a piece without a logit above -infinity adds nothing: its s and t are 0)
    const float d = (q.m == ninf ? base : q.m) - base, f = __expf(d);
    s += q.s * f;
    t += f * fmaf(q.s, fmaxf(d, -1000.0f), q.t);
  }
  s = wave_sum(s);
  t = wave_sum(t);
  const Scorer score(m, s, t);
  score.template tokens<T>(p, row, tid, 64 * W, ahead);
  if (p.top == 0) return;
  if (score.bad) {
    if (tid < p.top) score.alternative(p, row, tid, 0);
    return;
  }
  auto leave = [&](int j, uint64_t key) __attribute__((always_inline)) { score.alternative(p, row, j, key); };
  if (n > kHeld * 64 * W) {
    choice.one_by_one(p.top, n, tid, [&](int i) { return keys[i]; }, leave);
    return;
  }
  if (n <= 64 * W) {                                   // few: each is compared with all
    if (tid < n) choice.cand[tid] = held[0];
    if (tid == 0) choice.count = n;
    sync<W>();
    choice.rank(p.top, tid, leave);
    return;
  }
  choice.clear(tid);
  sync<W>();
  uint64_t own = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) own = held[i] > own ? held[i] : own;
  const bool wide = p.top > 24;
  choice.offer(wide, (uint32_t)(own >> 32), tid);
  sync<W>();
  // (where fewer columns than that have a key the limit is 0 and every key is a candidate)
  const uint32_t limit = choice.limit(wide, p.top, 12);
  if ((uint32_t)(own >> 32) >= limit) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (held[i] != 0 && (uint32_t)(held[i] >> 32) >= limit) choice.add(held[i]);
  }
  sync<W>();
  bool fits = choice.count <= kRoom;
  if (!fits)
    fits = choice.among_equals(wide, p.top, tid, [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (held[i] != 0) f((uint32_t)(held[i] >> 32), (uint32_t)held[i]);
    });
  if (fits) choice.rank(p.top, tid, leave);
  else choice.one_by_one(p.top, n, tid, [&](int i) { return keys[i]; }, leave);
}

int size_of(int type) { return type == 0 ? 4 : 2; }

// Bytes of logits that the largest workgroup takes (16 waves of 8 loads a lane), and one of 8 waves of 13.
constexpr int kWhole = 16 * 64 * 8 * 16, kPiece = 8 * 64 * 13 * 16;

// A row that one workgroup can take is one piece: it is done before a second kernel would begin (32000 float32 logits and five
// alternatives 6.6 us, 8.4 in two pieces, 9.9 in 15; 256 such rows 10.9 and 13.9 in two; but 1000 of them 39.5 and 31.0: 16 waves of 8 loads
// have a unit to themselves, of 8 waves two share it).  Few long rows: pieces for the whole chip, of 8 KiB and
// more, whose best the workgroup that joins them can hold.  Else the number of them that leaves the busiest compute unit the least
// to do, up to twice as many as it takes (128 rows of 128256 fp16 logits with 20 alternatives 18.7 to 20.1 us in 4 pieces, 20.9 in 2, 22.4
// in 3; 1000 of 100000 49.4 in 2, 52.4 in 3, 54.7 in 4).  256: the chip's units, as a number, because the workspace's size has to be the same
// whichever device is current, or none.
Pieces pieces_of(int64_t rows, int V, int bytes, int top) {
  Pieces c{};
  const int64_t all = (int64_t)V * bytes;
  int64_t n = 1;
  if (all > kWhole) {
    const int64_t least = (all + kPiece - 1) / kPiece, want = 256 / rows,
                  most = std::min<int64_t>((all + 8191) / 8192, kHeld * 64 * kJoinWaves / std::max(top, 1));
    auto turns = [&](int64_t k) { return (rows * k + 255) / 256; };
    n = std::max(least, std::min(want, most));
    for (int64_t k = least + 1; k <= 2 * least && k <= 64; ++k)
      if (turns(k) * n < turns(n) * k) n = k;
  }
  const int per = 16 / bytes;
  c.len = (int)(((V + n - 1) / n + per - 1) / per * per);
  c.n = (int)((V + (int64_t)c.len - 1) / c.len);
  return c;
}

}  // namespace

size_t logprobs_workspace_bytes(int64_t rows, int V, int top) {
  size_t most = 0;
  for (int bytes = 2; bytes <= 4; bytes += 2) {
    const Pieces c = rows > 0 ? pieces_of(rows, V, bytes, top) : Pieces{1};
    const size_t need = c.n == 1 ? 0 : (size_t)rows * c.n * (16 + 8 * (size_t)top);
    most = need > most ? need : most;
  }
  return (most + 255) & ~(size_t)255;
}

hipError_t launch_logprobs(const LogprobParams& p, int x_type, void* workspace, hipStream_t st) {
  const int bytes = size_of(x_type);
  Pieces c = pieces_of(p.rows, p.V, bytes, p.top);
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
    // (25600 rows of 128 float32 logits and 5 alternatives 9.4 us, a wave a row 22.6, 16 rows 3.7 and 4.7; 25600 of 256 bf16 and 8 alternatives
    // 19.8 and 25.2, but 1000 rows 6.6 and 5.4; with more alternatives a wave a row is the faster one for 256 logits, 28.6 for 33.3 with 20,
    // not for 128, 25.2 for 20.4)
    if (p.V <= 64 || (p.V <= 128 && p.top <= 5) || (p.V <= 256 && p.top <= 8 && p.rows >= 4096)) {
      const int G = p.V <= 16 ? 4 : p.V <= 32 ? 8 : 16, rows = 4 * 64 / G;
      const GridShape g = grid_shape((p.rows + rows - 1) / rows);
      return launch_kernel(G == 4 ? logprobs_small_kernel<T, 4, 4> : G == 8 ? logprobs_small_kernel<T, 8, 4> : p.V <= 64 ? logprobs_small_kernel<T, 16, 4>
                           : p.V <= 128 ? logprobs_small_kernel<T, 16, 8> : logprobs_small_kernel<T, 16, 16>,
                           dim3(g.x, g.y), dim3(256), 0, st, p);
    }
    // As many registers as a row needs and as few waves as then hold it: rows meet fewer barriers, and more of them share a unit.
    // (4096 rows of 50257 bf16 logits and 20 alternatives: 8 waves of 13 loads 81 us, 16 of 8 168; of 18000: 4 of 10 37 us, 8 of 8 48, but
    // where there are few rows, 16 of 20000, 7.8 us against 6.9; profiles/logprobs_form_choice.txt has every kernel beside the choice)
    if (loads <= 64) e = launch(logprobs_kernel<T, 1, 1>, 1);
    else if (loads <= 256) e = launch(logprobs_kernel<T, 1, 4>, 1);
    else if (loads <= 512) e = launch(logprobs_kernel<T, 4, 2>, 4);
    else if (loads <= 1024) e = launch(logprobs_kernel<T, 4, 4>, 4);
    else if (loads <= 2048) e = launch(logprobs_kernel<T, 4, 8>, 4);
    else if (loads <= 2560 && units >= 1024) e = launch(logprobs_kernel<T, 4, 10>, 4);
    else if (loads <= 4096) e = launch(logprobs_kernel<T, 8, 8>, 8);
    else if (loads <= 8 * 64 * 13) e = launch(logprobs_kernel<T, 8, 13>, 8);
    else e = launch(logprobs_kernel<T, 16, 8>, 16);
    if (e != hipSuccess || c.n == 1) return e;
    const GridShape g = grid_shape(p.rows);
    return launch_kernel(join_kernel<T>, dim3(g.x, g.y), dim3(64 * kJoinWaves), 0, st, p, c);
  });
}

}  // namespace qasr
