// Log probabilities of given tokens, the entropy and the largest logits of
// each row, and the gradient.
#include <math.h>

#include "externd_decode.hpp"

namespace externd {

struct LogprobArgs {
  const void* logits;
  int64_t rows, vocab, stride;
  const int64_t* targets;
  float scale;
  int top;
  float *logprob, *entropy, *lse, *top_logprobs;
  int64_t* top_ids;
};

// An order of (logit, index) pairs in one whole number: larger logits first,
// then lower indices.  Minus zero counts as zero.
__device__ __forceinline__ uint64_t order_key(float x, unsigned index) {
  int b = __float_as_int(x + 0.f);
  b = b < 0 ? b ^ 0x7FFFFFFF : b;
  return (uint64_t)((unsigned)b ^ 0x80000000u) << 32 | (0xFFFFFFFFu - index);
}

template <typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V* lds, F f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int d = 32; d; d >>= 1) v = f(v, (V)__shfl_xor(v, d));
  __syncthreads();
  if (lane == 0) lds[wave] = v;
  __syncthreads();
  v = lds[0];
  for (int i = 1; i < (int)(blockDim.x >> 6); i++) v = f(v, lds[i]);
  return v;
}

// One workgroup per row: the maximum, then the sums, then the largest logits
// one after another.
template <int DT>
__global__ __launch_bounds__(256) void k_logprobs(LogprobArgs a) {
  typedef typename Elem<DT>::T T;
  __shared__ float lf[4];
  __shared__ unsigned long long lk[4];
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.logits + r * a.stride;
  const int n = (int)a.vocab;
  float m = -INFINITY, nan = 0.f;
  for (int i = threadIdx.x; i < n; i += 256) {
    const float z = Elem<DT>::load(x[i]) * a.scale;
    m = fmaxf(m, z);
    nan = z == z && z < INFINITY ? nan : NAN;
  }
  m = block_reduce(m, lf, [](float p, float q) { return fmaxf(p, q); });
  float sum = 0.f, mean = 0.f;
  if (m > -INFINITY)
    for (int i = threadIdx.x; i < n; i += 256) {
      const float z = Elem<DT>::load(x[i]) * a.scale - m, e = expf(z);
      sum += e;
      mean += z == -INFINITY ? 0.f : e * z;
    }
  const auto plus = [](float p, float q) { return p + q; };
  sum = block_reduce(sum, lf, plus);
  mean = block_reduce(mean, lf, plus);
  nan = block_reduce(nan, lf, plus);
  const float lse = m == -INFINITY ? nan == 0.f ? -INFINITY : NAN : m + logf(sum) + nan;
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[r] = lse;
    if (a.entropy) a.entropy[r] = lse == -INFINITY ? 0.f : logf(sum) - mean / sum + nan;
    if (a.logprob) {
      const int64_t y = a.targets[r];
      const float z = y >= 0 && y < n ? Elem<DT>::load(x[y]) * a.scale : 0.f;
      a.logprob[r] = y < 0 ? 0.f : y >= n ? NAN : z == -INFINITY && !(lse != lse) ? -INFINITY : z - lse;
    }
  }
  uint64_t last = ~0ull;
  for (int j = 0; j < a.top; j++) {
    unsigned long long best = 0;
    for (int i = threadIdx.x; i < n; i += 256) {
      const uint64_t key = order_key(Elem<DT>::load(x[i]), (unsigned)i);
      if (key < last && key > best) best = key;
    }
    best = block_reduce(best, lk, [](unsigned long long p, unsigned long long q) { return p > q ? p : q; });
    last = best;
    if (threadIdx.x == 0) {
      const int i = (int)(0xFFFFFFFFu - (unsigned)best);
      const float z = Elem<DT>::load(x[i]) * a.scale;
      a.top_ids[r * a.top + j] = i;
      a.top_logprobs[r * a.top + j] = z == -INFINITY && !(lse != lse) ? -INFINITY : z - lse;
    }
  }
}

struct LogprobGradArgs {
  const void* logits;
  void* grad;
  int64_t rows, vocab, stride, grad_stride;
  const int64_t* targets;
  float scale;
  const float *lse, *entropy, *g_logprob, *g_entropy;
};

template <int DT>
__global__ __launch_bounds__(256) void k_logprobs_grad(LogprobGradArgs a) {
  typedef typename Elem<DT>::T T;
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.logits + r * a.stride;
  T* d = (T*)a.grad + r * a.grad_stride;
  const int n = (int)a.vocab;
  const int64_t y = a.targets ? a.targets[r] : -1;
  const float lse = a.lse[r], g = a.g_logprob && y >= 0 ? a.g_logprob[r] : 0.f;
  const float ge = a.g_entropy ? a.g_entropy[r] : 0.f, h = a.g_entropy ? a.entropy[r] : 0.f;
  for (int i = threadIdx.x; i < n; i += 256) {
    const float lp = lse == -INFINITY ? lse : Elem<DT>::load(x[i]) * a.scale - lse, p = expf(lp);
    float v = p == 0.f ? 0.f : -p * (g + ge * (lp + h));
    if (i == y) v += g;
    d[i] = Elem<DT>::store(v * a.scale);
  }
}

static bool logprob_sizes_ok(int64_t rows, int64_t vocab, int32_t top) {
  return rows >= 0 && vocab >= 1 && top >= 0 && top <= EXTERND_LOGPROBS_MAX_TOP && top <= vocab;
}

}  // namespace externd

using namespace externd;

extern "C" {

size_t externd_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int32_t top) {
  if (!logprob_sizes_ok(rows, vocab, top)) return 0;
  return 0;
}

int externd_token_logprobs(const void* logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t row_stride,
                           const int64_t* targets, float scale, int32_t top, float* logprob, float* entropy,
                           float* lse, float* top_logprobs, int64_t* top_ids, void* workspace,
                           size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dtype) || !logprob_sizes_ok(rows, vocab, top) || row_stride < vocab || !(scale > 0) ||
      !std::isfinite(scale) || (top && (!top_logprobs || !top_ids)) || (rows && !logits) || (logprob && rows && !targets))
    return EXTERND_EINVAL;
  if (rows > INT32_MAX || vocab > INT32_MAX) return EXTERND_EUNSUPPORTED;
  const size_t need = externd_token_logprobs_workspace_bytes(rows, vocab, top);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) return EXTERND_EWORKSPACE;
  if (!rows) return EXTERND_OK;
  const LogprobArgs a = {logits, rows, vocab, row_stride, targets, scale, top, logprob, entropy, lse, top_logprobs, top_ids};
  const hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)rows);
  if (dtype == EXTERND_F32) k_logprobs<EXTERND_F32><<<grid, 256, 0, s>>>(a);
  else if (dtype == EXTERND_BF16) k_logprobs<EXTERND_BF16><<<grid, 256, 0, s>>>(a);
  else k_logprobs<EXTERND_F16><<<grid, 256, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

int externd_token_logprobs_backward(const void* logits, int32_t dtype, int64_t rows, int64_t vocab,
                                    int64_t row_stride, const int64_t* targets, float scale, const float* lse,
                                    const float* entropy, const float* g_logprob, const float* g_entropy, void* grad,
                                    int64_t grad_row_stride, void* stream) {
  if (!dtype_ok(dtype) || !logprob_sizes_ok(rows, vocab, 0) || row_stride < vocab || grad_row_stride < vocab ||
      !(scale > 0) || !std::isfinite(scale))
    return EXTERND_EINVAL;
  if (rows && (!logits || !grad || !lse || (g_logprob && !targets) || (g_entropy && !entropy))) return EXTERND_EINVAL;
  if (rows > INT32_MAX || vocab > INT32_MAX) return EXTERND_EUNSUPPORTED;
  if (!rows) return EXTERND_OK;
  const LogprobGradArgs a = {logits, grad, rows, vocab, row_stride, grad_row_stride, targets, scale, lse, entropy,
                             g_logprob, g_entropy};
  const hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)rows);
  if (dtype == EXTERND_F32) k_logprobs_grad<EXTERND_F32><<<grid, 256, 0, s>>>(a);
  else if (dtype == EXTERND_BF16) k_logprobs_grad<EXTERND_BF16><<<grid, 256, 0, s>>>(a);
  else k_logprobs_grad<EXTERND_F16><<<grid, 256, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
