// Attention over the cache in 4 bits.
#include <math.h>

#include "externd_decode.hpp"

namespace externd {

struct AttnArgs {
  const uint8_t* cache;
  Kv4Shape c;
  Kv4Sequences s;
  const void* q;
  int64_t q_ts, q_hs;
  int heads_q, each;      // query heads, and how many of them share a cache head
  void* out;
  float* lse;
  float scale;
  int window;
};

// One wave per new token and query head, over 64 keys at a time: a lane scores
// one key, then the wave forms the weighted sum of the values, a lane holding
// DIM / 64 channels.
template <int DT, int DIM>
__global__ __launch_bounds__(64) void k_attention_rows(AttnArgs a) {
  typedef typename Elem<DT>::T T;
  constexpr int NG = DIM / KV4_GROUP, HALF = DIM / 2;
  __shared__ float qs[DIM], w[64];
  __shared__ int64_t base[64];
  const int lane = threadIdx.x;
  const int64_t t = blockIdx.x;
  const int hq = blockIdx.y, h = hq / a.each;
  const int b = sequence_of(a.s, t);
  const int64_t pos = position_of(a.s, b, t);
  const T* q = (const T*)a.q + t * a.q_ts + hq * a.q_hs;
#pragma unroll
  for (int g = 0; g < NG; g++) qs[g * 64 + lane] = Elem<DT>::load(q[g * 64 + lane]) * a.scale;
  __syncthreads();
  const int P = 1 << a.c.page_log2;
  int64_t first = a.window > 0 && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0;
  float m = -INFINITY, l = 0.f, o[NG] = {};
  for (int64_t j0 = first; j0 <= pos; j0 += 64) {
    const int64_t j = j0 + lane, page = j <= pos ? page_of(a.c, a.s, b, j) : -1;
    const int off = (int)(j & (P - 1));
    float x = -INFINITY;
    base[lane] = page < 0 ? -1 : (page * a.c.heads + h) * a.c.head_bytes;
    if (page >= 0) {
      const uint8_t* pg = a.cache + base[lane];
      const uint8_t* kc = pg + (size_t)off * HALF;
      const uint16_t* words = (const uint16_t*)(pg + (size_t)P * DIM) + off * 2 * NG;
      x = 0.f;
#pragma unroll
      for (int g = 0; g < NG; g++) {
        const float z = (float)(words[g] & 15);
        float sum = 0.f;
        for (int i = 0; i < 64; i++) {
          const int d = g * 64 + i;
          const unsigned byte = kc[d % HALF];
          sum = fmaf(qs[d], (float)(d < HALF ? byte & 15 : byte >> 4) - z, sum);
        }
        x = fmaf((float)__builtin_bit_cast(_Float16, (uint16_t)(words[g] & 0xFFF0u)), sum, x);
      }
    }
    float top = x;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float mn = fmaxf(m, top);
    // no key seen so far (mn -infinity): nothing to rescale and no weight;
    // a NaN score (x == x fails) stays a NaN weight
    const float keep = mn == -INFINITY ? 0.f : expf(m - mn);
    const float p = x == -INFINITY ? 0.f : mn == -INFINITY ? x : expf(x - mn);
    float sum = p;
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    m = mn;
    l = l * keep + sum;
    w[lane] = p;
    __syncthreads();
#pragma unroll
    for (int g = 0; g < NG; g++) {
      const int d = g * 64 + lane;
      float acc = o[g] * keep;
      for (int i = 0; i < 64; i++) {
        if (base[i] < 0) continue;
        const int oi = (int)((j0 + i) & (P - 1));
        const uint8_t* pg = a.cache + base[i];
        const unsigned byte = pg[(size_t)P * HALF + (size_t)(oi >> 4) * (HALF * 16) + (d % HALF) * 16 + (oi & 15)];
        const unsigned word = ((const uint16_t*)(pg + (size_t)P * DIM))[(oi * 2 + 1) * NG + g];
        const float v = (float)__builtin_bit_cast(_Float16, (uint16_t)(word & 0xFFF0u)) *
                        ((float)(d < HALF ? byte & 15 : byte >> 4) - (float)(word & 15));
        acc = fmaf(w[i], v, acc);
      }
      o[g] = acc;
    }
    __syncthreads();
  }
  const bool none = l == 0.f && m == -INFINITY;
  T* out = (T*)a.out + (t * a.heads_q + hq) * DIM;
#pragma unroll
  for (int g = 0; g < NG; g++) out[g * 64 + lane] = Elem<DT>::store(none ? 0.f : o[g] / l);
  if (a.lse && lane == 0) a.lse[t * a.heads_q + hq] = none ? -INFINITY : m + logf(l);
}

template <int DT>
static void launch_rows(const AttnArgs& a, dim3 grid, hipStream_t s) {
  if (a.c.dim == 64) k_attention_rows<DT, 64><<<grid, 64, 0, s>>>(a);
  else if (a.c.dim == 128) k_attention_rows<DT, 128><<<grid, 64, 0, s>>>(a);
  else k_attention_rows<DT, 256><<<grid, 64, 0, s>>>(a);
}

// Heads, types and counts of an attention call.
static bool attention_sizes_ok(int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t dtype, int64_t tokens,
                               int32_t batch, int32_t max_new, int64_t max_len) {
  return heads_kv >= 1 && heads_kv <= 4096 && heads_q >= heads_kv && heads_q % heads_kv == 0 && heads_q / heads_kv <= 64 &&
         (head_dim == 64 || head_dim == 128 || head_dim == 256) && dtype_ok(dtype) && tokens >= 0 && batch >= 1 &&
         max_new >= 1 && max_len >= 0;
}

}  // namespace externd

using namespace externd;

extern "C" {

size_t externd_kv4_attention_workspace_bytes(int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t dtype,
                                             int64_t tokens, int32_t batch, int32_t max_new, int64_t max_len) {
  if (!attention_sizes_ok(heads_q, heads_kv, head_dim, dtype, tokens, batch, max_new, max_len)) return 0;
  return 0;
}

int externd_kv4_attention(const void* cache, int64_t num_pages, int32_t heads_kv, int32_t head_dim,
                          int32_t page_tokens, const void* q, int32_t dtype, int64_t q_token_stride,
                          int64_t q_head_stride, int32_t heads_q, void* out, float* lse, int64_t tokens,
                          int32_t batch, int32_t max_new, int64_t max_len, const int32_t* starts,
                          const int32_t* lens, const int32_t* table, int64_t table_pages, float scale,
                          int32_t window, void* workspace, size_t workspace_bytes, void* stream) {
  AttnArgs a;
  if (!kv4_shape(num_pages, heads_kv, head_dim, page_tokens, &a.c)) return EXTERND_EINVAL;
  if (!attention_sizes_ok(heads_q, heads_kv, head_dim, dtype, tokens, batch, max_new, max_len)) return EXTERND_EINVAL;
  if (!cache || ((uintptr_t)cache & 15) || !lens || !table || table_pages < 1 || window < 0 || !std::isfinite(scale) ||
      (!starts && tokens != batch) || (tokens && (!q || !out)))
    return EXTERND_EINVAL;
  if (tokens > INT32_MAX || batch > 65535 || heads_q > 65535 || table_pages > INT32_MAX) return EXTERND_EUNSUPPORTED;
  const size_t need =
      externd_kv4_attention_workspace_bytes(heads_q, heads_kv, head_dim, dtype, tokens, batch, max_new, max_len);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) return EXTERND_EWORKSPACE;
  if (!tokens) return EXTERND_OK;
  a.cache = (const uint8_t*)cache;
  a.s = {starts, lens, table, table_pages, tokens, batch};
  a.q = q;
  a.q_ts = q_token_stride;
  a.q_hs = q_head_stride;
  a.heads_q = heads_q;
  a.each = heads_q / heads_kv;
  a.out = out;
  a.lse = lse;
  a.scale = scale;
  a.window = window;
  const dim3 grid((unsigned)tokens, (unsigned)heads_q);
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) launch_rows<EXTERND_F32>(a, grid, s);
  else if (dtype == EXTERND_BF16) launch_rows<EXTERND_BF16>(a, grid, s);
  else launch_rows<EXTERND_F16>(a, grid, s);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
