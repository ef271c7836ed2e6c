// Log probabilities behind a dense head, and the gradients for its input and
// its matrix, without holding the logits.
#include <cmath>

#include "externd_decode.hpp"

namespace externd {

constexpr int TILE = 64, DEPTH = 16;
constexpr int64_t FORWARD_ROWS = 8192;      // of a pass, so that the parts stay small

// C(i, j) = sum over k of A(i, k) B(j, k) of a 64 x 64 tile; 256 threads, 4 x 4 entries each.
template <typename LA, typename LB>
__device__ __forceinline__ void tile_product(LA A, LB B, int64_t k0, int64_t k1, float (*sum)[4]) {
  __shared__ float a[DEPTH][TILE + 4], b[DEPTH][TILE + 4];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int64_t k = k0; k < k1; k += DEPTH) {
    for (int e = threadIdx.x; e < TILE * DEPTH; e += 256) {
      const int i = e / DEPTH, q = e % DEPTH;
      a[q][i] = k + q < k1 ? A(i, k + q) : 0.f;
      b[q][i] = k + q < k1 ? B(i, k + q) : 0.f;
    }
    __syncthreads();
    for (int q = 0; q < DEPTH; q++)
      for (int i = 0; i < 4; i++)
        for (int j = 0; j < 4; j++) sum[i][j] = fmaf(a[q][ty * 4 + i], b[q][tx * 4 + j], sum[i][j]);
    __syncthreads();
  }
}

struct Part {
  float top, sum, mean, none;      // largest z, sum of e = exp(z - top), sum of e (z - top)
};

struct LinearArgs {
  const void *x, *weight;
  int64_t x_stride, weight_stride, rows, vocab, width;
  const int64_t* targets;
  float scale;
  // forward
  float *logprob, *entropy, *lse;
  Part* parts;          // rows x tiles
  int64_t tiles;
  float* at_target;     // z of the target
  // backward
  const float *lse_in, *entropy_in, *g_logprob, *g_entropy;
  void *grad_x, *grad_weight;
  int64_t grad_x_stride, grad_weight_stride, v0, v1;      // this piece of the vocabulary
  float *G, *dx;        // rows x piece; rows x width
  int64_t piece;
};

__device__ __forceinline__ float propagating_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// What a row's gradient is made of; false: the row takes no part.
__device__ __forceinline__ bool row_gradients(const LinearArgs& a, int64_t r, float* g, float* ge, int64_t* y) {
  *y = a.targets ? a.targets[r] : -1;
  *g = a.g_logprob && *y >= 0 && *y < a.vocab ? a.g_logprob[r] : 0.f;
  *ge = a.g_entropy ? a.g_entropy[r] : 0.f;
  return *g != 0.f || *ge != 0.f;
}

// Rows of x against 64 rows of weight.  BACK: G of the tile, else the tile's part of each row's softmax.
template <int DT, bool BACK>
__global__ __launch_bounds__(256) void k_logits(LinearArgs a) {
  typedef typename Elem<DT>::T T;
  __shared__ float z[TILE][TILE + 1];
  const int64_t r0 = (int64_t)blockIdx.y * TILE, c0 = a.v0 + (int64_t)blockIdx.x * TILE;
  const T *x = (const T*)a.x, *w = (const T*)a.weight;
  float sum[4][4] = {};
  tile_product([&](int i, int64_t k) { return r0 + i < a.rows ? Elem<DT>::load(x[(r0 + i) * a.x_stride + k]) : 0.f; },
               [&](int i, int64_t k) { return c0 + i < a.v1 ? Elem<DT>::load(w[(c0 + i) * a.weight_stride + k]) : 0.f; }, 0, a.width, sum);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int i = 0; i < 4; i++)
    for (int j = 0; j < 4; j++) z[ty * 4 + i][tx * 4 + j] = c0 + tx * 4 + j < a.v1 ? sum[i][j] * a.scale : -INFINITY;
  __syncthreads();
  if (threadIdx.x >= TILE || r0 + threadIdx.x >= a.rows) return;
  const float* row = z[threadIdx.x];
  const int64_t r = r0 + threadIdx.x;
  if constexpr (BACK) {
    float g, ge;
    int64_t y;
    const bool present = row_gradients(a, r, &g, &ge, &y);
    for (int c = 0; c < TILE && c0 + c < a.v1; c++) {
      float o = 0.f;
      if (present) {
        const float lp = row[c] - a.lse_in[r], p = expf(lp);
        o = p == 0.f ? 0.f : -p * (ge == 0.f ? g : fmaf(ge, lp + a.entropy_in[r], g));
        if (c0 + c == y) o += g;
      }
      a.G[r * a.piece + c0 - a.v0 + c] = o;
    }
  } else {
    float top = -INFINITY;
    for (int c = 0; c < TILE; c++) top = fmaxf(top, row[c]);
    Part p = {top, 0.f, 0.f, 0.f};
    const float ref = fmaxf(top, -3.402823466e38f);
    for (int c = 0; c < TILE; c++) {
      const float d = propagating_max(row[c] - ref, -150.f), e = expf(d);
      p.sum += row[c] == -INFINITY ? 0.f : e;
      p.mean += row[c] == -INFINITY ? 0.f : e * d;
    }
    a.parts[r * a.tiles + blockIdx.x] = p;
    if (a.targets && a.targets[r] >= c0 && a.targets[r] < min(c0 + TILE, a.v1)) a.at_target[r] = row[a.targets[r] - c0];
  }
}

// A wave joins a row's parts.
__global__ __launch_bounds__(64) void k_logits_join(LinearArgs a) {
  const int64_t r = blockIdx.x;
  const Part* p = a.parts + r * a.tiles;
  float top = -3.402823466e38f, sum = 0.f, mean = 0.f;
  for (int64_t i = threadIdx.x; i < a.tiles; i += 64) top = fmaxf(top, p[i].top);
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  for (int64_t i = threadIdx.x; i < a.tiles; i += 64) {
    if (p[i].sum == 0.f) continue;
    const float d = fmaxf(p[i].top, -3.402823466e38f) - top, f = expf(d);
    sum += p[i].sum * f;
    mean += f == 0.f ? 0.f : fmaf(p[i].sum, d, p[i].mean) * f;
  }
  for (int d = 32; d; d >>= 1) {
    sum += __shfl_xor(sum, d);
    mean += __shfl_xor(mean, d);
  }
  if (threadIdx.x) return;
  const bool none = sum == 0.f;
  const float l = logf(sum), lse = none ? -INFINITY : top + l;
  if (a.lse) a.lse[r] = lse;
  if (a.entropy) a.entropy[r] = none ? 0.f : l - mean / sum;
  if (a.logprob) {
    const int64_t y = a.targets[r];
    a.logprob[r] = y < 0 ? 0.f : y >= a.vocab ? NAN : none ? -INFINITY : a.at_target[r] - lse;
  }
}

// grad_x (+)= G weight over this piece, in fp32.
template <int DT>
__global__ __launch_bounds__(256) void k_grad_x(LinearArgs a) {
  typedef typename Elem<DT>::T T;
  const int64_t r0 = (int64_t)blockIdx.y * TILE, c0 = (int64_t)blockIdx.x * TILE;
  const T* w = (const T*)a.weight;
  float sum[4][4] = {};
  tile_product([&](int i, int64_t k) { return r0 + i < a.rows ? a.G[(r0 + i) * a.piece + k] : 0.f; },
               [&](int i, int64_t k) { return c0 + i < a.width ? Elem<DT>::load(w[(a.v0 + k) * a.weight_stride + c0 + i]) : 0.f; }, 0,
               a.v1 - a.v0, sum);
  for (int i = 0; i < 4; i++)
    for (int j = 0; j < 4; j++) {
      const int64_t r = r0 + (threadIdx.x >> 4) * 4 + i, c = c0 + (threadIdx.x & 15) * 4 + j;
      if (r >= a.rows || c >= a.width) continue;
      float* d = a.dx + r * a.width + c;
      const float all = (a.v0 ? *d : 0.f) + sum[i][j];
      *d = all;
      if (a.v1 == a.vocab) {
        float g, ge;
        int64_t y;
        ((T*)a.grad_x)[r * a.grad_x_stride + c] = Elem<DT>::store(row_gradients(a, r, &g, &ge, &y) ? all * a.scale : 0.f);
      }
    }
}

template <int DT>
__global__ __launch_bounds__(256) void k_grad_weight(LinearArgs a) {
  typedef typename Elem<DT>::T T;
  const int64_t r0 = (int64_t)blockIdx.y * TILE, c0 = (int64_t)blockIdx.x * TILE;
  const T* x = (const T*)a.x;
  float sum[4][4] = {};
  tile_product([&](int i, int64_t k) { return a.v0 + r0 + i < a.v1 ? a.G[k * a.piece + r0 + i] : 0.f; },
               [&](int i, int64_t k) {
                 float g, ge;
                 int64_t y;
                 return c0 + i < a.width && row_gradients(a, k, &g, &ge, &y) ? Elem<DT>::load(x[k * a.x_stride + c0 + i]) : 0.f;
               },
               0, a.rows, sum);
  for (int i = 0; i < 4; i++)
    for (int j = 0; j < 4; j++) {
      const int64_t r = r0 + (threadIdx.x >> 4) * 4 + i, c = c0 + (threadIdx.x & 15) * 4 + j;
      if (a.v0 + r < a.v1 && c < a.width) ((T*)a.grad_weight)[(a.v0 + r) * a.grad_weight_stride + c] = Elem<DT>::store(sum[i][j] * a.scale);
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

static bool linear_sizes(int64_t rows, int64_t vocab, int64_t width) {
  return rows <= (1 << 22) && vocab < INT32_MAX - 1023 && width <= (1 << 20);
}

struct LinearWork {
  size_t parts, at_target, G, dx, bytes;
  int64_t tiles, piece;
};

static LinearWork forward_work(int64_t rows, int64_t vocab) {
  LinearWork w = {};
  const int64_t r = rows < FORWARD_ROWS ? rows : FORWARD_ROWS;
  w.tiles = ceil_div(vocab, TILE);
  w.parts = 0;
  w.at_target = round256((size_t)(r * w.tiles) * sizeof(Part));
  w.bytes = w.at_target + round256((size_t)r * 4);
  return w;
}

static LinearWork backward_work(int64_t rows, int64_t vocab, int64_t width, bool need_x) {
  LinearWork w = {};
  w.piece = ((int64_t)1 << 25) / (rows ? rows : 1);
  w.piece = ceil_div(w.piece < 1024 ? 1024 : w.piece, TILE) * TILE;
  if (w.piece > ceil_div(vocab, TILE) * TILE) w.piece = ceil_div(vocab, TILE) * TILE;
  w.G = 0;
  w.dx = round256((size_t)(rows * w.piece) * 4);
  w.bytes = w.dx + (need_x ? round256((size_t)(rows * width) * 4) : 0);
  return w;
}

template <int DT>
static void launch_forward(LinearArgs a, hipStream_t s) {
  k_logits<DT, false><<<dim3((unsigned)a.tiles, (unsigned)ceil_div(a.rows, TILE)), 256, 0, s>>>(a);
  k_logits_join<<<(unsigned)a.rows, 64, 0, s>>>(a);
}

template <int DT>
static void launch_backward(LinearArgs a, hipStream_t s) {
  const unsigned rows = (unsigned)ceil_div(a.rows, TILE), cols = (unsigned)ceil_div(a.width, TILE);
  for (a.v0 = 0; a.v0 < a.vocab; a.v0 = a.v1) {
    a.v1 = a.v0 + a.piece < a.vocab ? a.v0 + a.piece : a.vocab;
    const unsigned tiles = (unsigned)ceil_div(a.v1 - a.v0, TILE);
    if (rows) k_logits<DT, true><<<dim3(tiles, rows), 256, 0, s>>>(a);
    if (rows && a.grad_x) k_grad_x<DT><<<dim3(cols, rows), 256, 0, s>>>(a);
    if (a.grad_weight) k_grad_weight<DT><<<dim3(cols, tiles), 256, 0, s>>>(a);
  }
}

}  // namespace externd

using namespace externd;

extern "C" {

size_t externd_linear_logprobs_workspace_bytes(int32_t dtype, int64_t rows, int64_t vocab, int64_t width) {
  if (!dtype_ok(dtype) || rows < 0 || vocab < 1 || width < 1 || !linear_sizes(rows, vocab, width)) return 0;
  return forward_work(rows ? rows : 1, vocab).bytes;
}

int externd_linear_logprobs(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride, int32_t dtype,
                            int64_t rows, int64_t vocab, int64_t width, const int64_t* targets, float scale,
                            float* logprob, float* entropy, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream) {
  if (!dtype_ok(dtype) || rows < 0 || vocab < 1 || width < 1 || x_stride < width || weight_stride < width || !(scale > 0) ||
      !std::isfinite(scale) || (rows && (!x || !weight)) || (rows && logprob && !targets))
    return EXTERND_EINVAL;
  if (!linear_sizes(rows, vocab, width) || x_stride >= (1 << 22) || weight_stride >= (1 << 22)) return EXTERND_EUNSUPPORTED;
  if (!rows) return EXTERND_OK;
  if ((uintptr_t)workspace & 255) return EXTERND_EINVAL;
  const LinearWork w = forward_work(rows, vocab);
  if (!workspace || workspace_bytes < w.bytes) return EXTERND_EWORKSPACE;
  const hipStream_t s = (hipStream_t)stream;
  for (int64_t r = 0; r < rows; r += FORWARD_ROWS) {
    LinearArgs a = {};
    a.x = (const char*)x + r * x_stride * dtype_bytes(dtype);
    a.weight = weight;
    a.x_stride = x_stride;
    a.weight_stride = weight_stride;
    a.rows = rows - r < FORWARD_ROWS ? rows - r : FORWARD_ROWS;
    a.vocab = a.v1 = vocab;
    a.width = width;
    a.targets = logprob ? targets + r : nullptr;
    a.scale = scale;
    a.logprob = logprob ? logprob + r : nullptr;
    a.entropy = entropy ? entropy + r : nullptr;
    a.lse = lse ? lse + r : nullptr;
    a.parts = (Part*)((char*)workspace + w.parts);
    a.at_target = (float*)((char*)workspace + w.at_target);
    a.tiles = w.tiles;
    if (dtype == EXTERND_F32) launch_forward<EXTERND_F32>(a, s);
    else if (dtype == EXTERND_BF16) launch_forward<EXTERND_BF16>(a, s);
    else launch_forward<EXTERND_F16>(a, s);
  }
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

size_t externd_linear_logprobs_backward_workspace_bytes(int32_t dtype, int64_t rows, int64_t vocab, int64_t width,
                                                        int32_t need_x, int32_t need_weight) {
  (void)need_weight;
  if (!dtype_ok(dtype) || rows < 0 || vocab < 1 || width < 1 || !linear_sizes(rows, vocab, width)) return 0;
  return backward_work(rows ? rows : 1, vocab, width, need_x).bytes;
}

int externd_linear_logprobs_backward(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride,
                                     int32_t dtype, int64_t rows, int64_t vocab, int64_t width, const int64_t* targets,
                                     float scale, const float* lse, const float* entropy, const float* g_logprob,
                                     const float* g_entropy, void* grad_x, int64_t grad_x_stride, void* grad_weight,
                                     int64_t grad_weight_stride, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dtype) || rows < 0 || vocab < 1 || width < 1 || x_stride < width || weight_stride < width ||
      (grad_x && grad_x_stride < width) || (grad_weight && grad_weight_stride < width) || !(scale > 0) || !std::isfinite(scale))
    return EXTERND_EINVAL;
  if (rows && (!x || !weight || !lse || (g_logprob && !targets) || (g_entropy && !entropy))) return EXTERND_EINVAL;
  if (!linear_sizes(rows, vocab, width) || x_stride >= (1 << 22) || weight_stride >= (1 << 22)) return EXTERND_EUNSUPPORTED;
  if (!grad_weight && (!grad_x || !rows)) return EXTERND_OK;
  if ((uintptr_t)workspace & 255) return EXTERND_EINVAL;
  const LinearWork w = backward_work(rows ? rows : 1, vocab, width, grad_x);
  if (!workspace || workspace_bytes < w.bytes) return EXTERND_EWORKSPACE;
  LinearArgs a = {};
  a.x = x;
  a.weight = weight;
  a.x_stride = x_stride;
  a.weight_stride = weight_stride;
  a.rows = rows;
  a.vocab = vocab;
  a.width = width;
  a.targets = targets;
  a.scale = scale;
  a.lse_in = lse;
  a.entropy_in = entropy;
  a.g_logprob = g_logprob;
  a.g_entropy = g_entropy;
  a.grad_x = grad_x;
  a.grad_weight = grad_weight;
  a.grad_x_stride = grad_x_stride;
  a.grad_weight_stride = grad_weight_stride;
  a.G = (float*)((char*)workspace + w.G);
  a.dx = (float*)((char*)workspace + w.dx);
  a.piece = w.piece;
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) launch_backward<EXTERND_F32>(a, s);
  else if (dtype == EXTERND_BF16) launch_backward<EXTERND_BF16>(a, s);
  else launch_backward<EXTERND_F16>(a, s);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
