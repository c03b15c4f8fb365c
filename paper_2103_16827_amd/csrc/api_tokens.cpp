// C ABI of the language-model operators: argument validation (before any HIP call) and launches.
#include "../../include/qasr.h"
#include "kernels.hpp"

namespace {

qasr_status hip_status(hipError_t e) { return (qasr_status)qasr::status_of(e); }

bool overlaps(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a && b && na > 0 && nb > 0 && a0 < b0 + (uint64_t)nb && b0 < a0 + (uint64_t)na;
}

// bytes per element, 0 for an unknown type
int64_t size_of(int32_t type) { return type == QASR_F32 ? 4 : type == QASR_F16 || type == QASR_BF16 ? 2 : 0; }

bool misaligned(const void* p, int64_t size) { return (uintptr_t)p % (uintptr_t)size != 0; }

// elements from the first to behind the last of `rows` rows of n, `stride` apart
int64_t extent(int64_t rows, int64_t stride, int64_t n) { return (rows - 1) * stride + n; }

// rows of n elements `stride` apart (0: dense): the stride is 0 or at least n, and addresses of twice the extent stay in 62 bits
bool rows_ok(int64_t rows, int64_t stride, int64_t n) {
  if (stride == 0) stride = n;
  return stride >= n && stride <= ((int64_t)1 << 58) / (rows < 1 ? 1 : rows);
}

constexpr int32_t kMaxK = 131071;          // 128 x 128 x K < 2^31
constexpr int32_t kMaxExperts = 4096;
constexpr int32_t kMaxSide = 1 << 30;      // of rows, channels and elements of a row: with a tile or a workgroup more they are int32 still
constexpr int64_t kMaxTiles = ((int64_t)1 << 31) - 16;      // (16 x 16 is the smallest tile)

size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }
int64_t round16(int64_t n) { return (n + 15) & ~(int64_t)15; }

// the descriptor's own checks and the strides that 0 stands for
qasr_status check_linear(const qasr_linear_desc* d, int32_t groups, qasr_linear_desc& out) {
  if (!d) return QASR_ERR_NULL;
  if (d->M < 0 || d->M > kMaxSide || d->N < 1 || d->N > kMaxSide || d->K < 1 || d->K > kMaxK) return QASR_ERR_SHAPE;
  if (((int64_t)d->M / 16 + groups) * ((int64_t)d->N / 16 + 1) > kMaxTiles) return QASR_ERR_SHAPE;
  if (!rows_ok(d->M, d->x_stride, d->K) || !rows_ok(d->N, d->w_stride, d->K) || !rows_ok(d->M, d->y_stride, d->N))
    return QASR_ERR_SHAPE;
  if (size_of(d->y_type) == 0 || d->reserved != 0) return QASR_ERR_PARAM;
  out = *d;
  if (out.x_stride == 0) out.x_stride = out.K;
  if (out.w_stride == 0) out.w_stride = out.K;
  if (out.y_stride == 0) out.y_stride = out.N;
  return QASR_OK;
}

qasr::LinearParams linear_params(const qasr_linear_desc& d, const int8_t* x, const float* x_scale, const int8_t* w,
                                 const float* w_scale, const float* bias, void* y) {
  qasr::LinearParams p{};
  p.x = x; p.x_scale = x_scale; p.w = w; p.w_scale = w_scale; p.bias = bias; p.y = y;
  p.xs = d.x_stride; p.ws = d.w_stride; p.ys = d.y_stride;
  p.M = d.M; p.N = d.N; p.K = d.K; p.y_type = d.y_type;
  p.x_rows = d.M;
  return p;
}

}  // namespace

extern "C" {

qasr_status qasr_quantize_tokens(const void* x, int32_t x_type, int64_t M, int32_t K, int64_t x_stride, int8_t* q,
                                 int64_t q_stride, float* scale, void* stream) {
  const int64_t size = size_of(x_type);
  if (size == 0) return QASR_ERR_PARAM;
  if (M < 0 || K < 1 || K > kMaxSide || M > ((int64_t)1 << 40) || !rows_ok(M, x_stride, K) || !rows_ok(M, q_stride, K)) return QASR_ERR_SHAPE;
  if (M == 0) return QASR_OK;
  if (!x || !q || !scale) return QASR_ERR_NULL;
  if (misaligned(x, size) || misaligned(scale, 4)) return QASR_ERR_PARAM;
  if (x_stride == 0) x_stride = K;
  if (q_stride == 0) q_stride = K;
  const int64_t nx = size * extent(M, x_stride, K), nq = extent(M, q_stride, K);
  if (overlaps(q, nq, x, nx) || overlaps(scale, 4 * M, x, nx) || overlaps(scale, 4 * M, q, nq)) return QASR_ERR_ALIAS;
  return hip_status(qasr::launch_quantize_tokens(x, x_type, M, K, x_stride, q, q_stride, scale, (hipStream_t)stream));
}

qasr_status qasr_linear_int8(const qasr_linear_desc* desc, const int8_t* x, const float* x_scale, const int8_t* w,
                             const float* w_scale, const float* bias, void* y, void* stream) {
  qasr_linear_desc d;
  const qasr_status st = check_linear(desc, 1, d);
  if (st != QASR_OK) return st;
  if (d.M == 0) return QASR_OK;
  if (!x || !x_scale || !w || !w_scale || !y) return QASR_ERR_NULL;
  const int64_t size = size_of(d.y_type), ny = size * extent(d.M, d.y_stride, d.N);
  if (misaligned(y, size) || misaligned(x_scale, 4) || misaligned(w_scale, 4) || misaligned(bias, 4)) return QASR_ERR_PARAM;
  if (overlaps(y, ny, x, extent(d.M, d.x_stride, d.K)) || overlaps(y, ny, w, extent(d.N, d.w_stride, d.K)) ||
      overlaps(y, ny, x_scale, 4 * (int64_t)d.M) || overlaps(y, ny, w_scale, 4 * (int64_t)d.N) ||
      overlaps(y, ny, bias, 4 * (int64_t)d.N))
    return QASR_ERR_ALIAS;
  return hip_status(qasr::launch_linear(linear_params(d, x, x_scale, w, w_scale, bias, y), (hipStream_t)stream));
}

size_t qasr_linear_workspace_bytes(int32_t M, int32_t K) {
  if (M < 0 || K < 1 || K > kMaxK) return 0;
  return round256((size_t)M * (size_t)round16(K)) + round256(4 * (size_t)M);
}

qasr_status qasr_linear_int8_dynamic(const qasr_linear_desc* desc, const void* x, int32_t x_type, const int8_t* w,
                                     const float* w_scale, const float* bias, void* y, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  qasr_linear_desc d;
  const qasr_status st = check_linear(desc, 1, d);
  if (st != QASR_OK) return st;
  const int64_t xsize = size_of(x_type), size = size_of(d.y_type);
  if (xsize == 0) return QASR_ERR_PARAM;
  if (d.M == 0) return QASR_OK;
  if (!x || !w || !w_scale || !y) return QASR_ERR_NULL;
  if (misaligned(x, xsize) || misaligned(y, size) || misaligned(w_scale, 4) || misaligned(bias, 4)) return QASR_ERR_PARAM;
  const size_t need = qasr_linear_workspace_bytes(d.M, d.K);
  if (!workspace || misaligned(workspace, 256) || workspace_bytes < need) return QASR_ERR_WORKSPACE;
  const int64_t nx = xsize * extent(d.M, d.x_stride, d.K), nw = extent(d.N, d.w_stride, d.K),
                ny = size * extent(d.M, d.y_stride, d.N), nn = 4 * (int64_t)d.N;
  if (overlaps(y, ny, x, nx) || overlaps(y, ny, w, nw) || overlaps(y, ny, w_scale, nn) || overlaps(y, ny, bias, nn))
    return QASR_ERR_ALIAS;
  const int64_t nws = (int64_t)need;
  if (overlaps(workspace, nws, x, nx) || overlaps(workspace, nws, w, nw) || overlaps(workspace, nws, w_scale, nn) ||
      overlaps(workspace, nws, bias, nn) || overlaps(workspace, nws, y, ny))
    return QASR_ERR_ALIAS;
  qasr::LinearParams p = linear_params(d, nullptr, nullptr, w, w_scale, bias, y);
  p.xf = x;
  if (qasr::linear_takes_floats(p, x_type)) return hip_status(qasr::launch_linear_floats(p, x_type, (hipStream_t)stream));
  const int64_t pitch = round16(d.K);
  int8_t* codes = (int8_t*)workspace;
  float* scale = (float*)(codes + round256((size_t)d.M * (size_t)pitch));
  const hipError_t e = qasr::launch_quantize_tokens(x, x_type, d.M, d.K, d.x_stride, codes, pitch, scale, (hipStream_t)stream);
  if (e != hipSuccess) return hip_status(e);
  d.x_stride = pitch;
  return hip_status(qasr::launch_linear(linear_params(d, codes, scale, w, w_scale, bias, y), (hipStream_t)stream));
}

qasr_status qasr_experts_int8(const qasr_experts_desc* desc, const int8_t* x, const float* x_scale, const int32_t* offsets,
                              const int32_t* index, const int8_t* w, const float* w_scale, const float* bias, void* y,
                              void* stream) {
  if (!desc) return QASR_ERR_NULL;
  qasr_linear_desc d;
  if (desc->E < 1 || desc->E > kMaxExperts) return QASR_ERR_SHAPE;
  const qasr_status st = check_linear(&desc->l, desc->E, d);
  if (st != QASR_OK) return st;
  const int64_t matrix = extent(d.N, d.w_stride, d.K);
  const int64_t wes = desc->w_expert_stride ? desc->w_expert_stride : (int64_t)d.N * d.w_stride;
  if (desc->x_rows < 1 || wes < matrix || wes > ((int64_t)1 << 58) / desc->E ||
      !rows_ok(desc->x_rows, d.x_stride, d.K) || (!index && desc->x_rows < d.M))
    return QASR_ERR_SHAPE;
  if (d.M == 0) return QASR_OK;
  if (!x || !x_scale || !offsets || !w || !w_scale || !y) return QASR_ERR_NULL;
  const int64_t size = size_of(d.y_type), ny = size * extent(d.M, d.y_stride, d.N), nn = 4 * (int64_t)desc->E * d.N;
  if (misaligned(y, size) || misaligned(x_scale, 4) || misaligned(w_scale, 4) || misaligned(bias, 4) ||
      misaligned(offsets, 4) || misaligned(index, 4))
    return QASR_ERR_PARAM;
  if (overlaps(y, ny, x, extent(desc->x_rows, d.x_stride, d.K)) || overlaps(y, ny, w, (desc->E - 1) * wes + matrix) ||
      overlaps(y, ny, x_scale, 4 * (int64_t)desc->x_rows) || overlaps(y, ny, w_scale, nn) || overlaps(y, ny, bias, nn) ||
      overlaps(y, ny, offsets, 4 * ((int64_t)desc->E + 1)) || overlaps(y, ny, index, 4 * (int64_t)d.M))
    return QASR_ERR_ALIAS;
  qasr::LinearParams p = linear_params(d, x, x_scale, w, w_scale, bias, y);
  p.offsets = offsets; p.index = index;
  p.E = desc->E; p.x_rows = desc->x_rows; p.wes = wes;
  return hip_status(qasr::launch_linear(p, (hipStream_t)stream));
}

static bool logprobs_shape_ok(int64_t rows, int32_t V, int32_t top) {
  return rows >= 0 && rows <= ((int64_t)1 << 40) && V >= 1 && top >= 0 && top <= QASR_MAX_TOP && top <= V && rows_ok(rows, 0, V);
}

size_t qasr_logprobs_workspace_bytes(int64_t rows, int32_t V, int32_t top) {
  return logprobs_shape_ok(rows, V, top) ? qasr::logprobs_workspace_bytes(rows, V, top) : 0;
}

qasr_status qasr_token_logprobs(const void* x, int32_t x_type, int64_t rows, int32_t V, int64_t x_stride, const int32_t* tokens,
                                int32_t n, float* logprob, float* entropy, int32_t top, int32_t* top_ids, float* top_logprob,
                                void* workspace, size_t workspace_bytes, void* stream) {
  const int64_t size = size_of(x_type);
  if (size == 0) return QASR_ERR_PARAM;
  if (!logprobs_shape_ok(rows, V, top) || n < 0 || !rows_ok(rows, x_stride, V) || !rows_ok(rows, 0, n)) return QASR_ERR_SHAPE;
  if (rows == 0 || (n == 0 && !entropy && top == 0)) return QASR_OK;
  if (!x || (n > 0 && (!tokens || !logprob)) || (top > 0 && (!top_ids || !top_logprob))) return QASR_ERR_NULL;
  if (x_stride == 0) x_stride = V;
  if (misaligned(x, size) || misaligned(entropy, 4) || (n > 0 && (misaligned(tokens, 4) || misaligned(logprob, 4))) ||
      (top > 0 && (misaligned(top_ids, 4) || misaligned(top_logprob, 4))))
    return QASR_ERR_PARAM;
  const size_t need = qasr::logprobs_workspace_bytes(rows, V, top);
  if (need > 0 && (!workspace || misaligned(workspace, 256) || workspace_bytes < need)) return QASR_ERR_WORKSPACE;
  const struct { const void* p; int64_t bytes; } t[] = {
      {x, size * extent(rows, x_stride, V)}, {n > 0 ? tokens : nullptr, 4 * rows * n},
      {n > 0 ? logprob : nullptr, 4 * rows * n}, {entropy, 4 * rows}, {top > 0 ? top_ids : nullptr, 4 * rows * top},
      {top > 0 ? top_logprob : nullptr, 4 * rows * top}, {need > 0 ? workspace : nullptr, (int64_t)need}};
  for (int a = 2; a < 7; ++a)                        // the written ones against all before them
    for (int b = 0; b < a; ++b)
      if (overlaps(t[a].p, t[a].bytes, t[b].p, t[b].bytes)) return QASR_ERR_ALIAS;
  qasr::LogprobParams p{};
  p.x = x; p.tokens = tokens; p.logprob = logprob; p.entropy = entropy; p.top_ids = top_ids; p.top_logprob = top_logprob;
  p.rows = rows; p.xs = x_stride; p.V = V; p.n = n; p.top = top;
  return hip_status(qasr::launch_logprobs(p, x_type, workspace, (hipStream_t)stream));
}

}  // extern "C"
