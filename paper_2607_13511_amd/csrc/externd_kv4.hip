// The cache in 4 bits: storing new tokens and reading values back.
#include "externd_decode.hpp"

namespace externd {

// Scale of 64 values that span `range` (0 within it): range / 15 rounded up
// to seven significant bits, or to a multiple of 2^-20 below 2^-14, so that
// scale x (-15 .. 15) is exactly an fp16 number and the fp16 scale's low four
// bits are free for the zero point.
__device__ __forceinline__ float kv4_scale(float range) {
  const float s = range / 15.f;
  const float seven = __uint_as_float((__float_as_uint(s) + 0x1FFFFu) & ~0x1FFFFu);
  const float small = ceilf(s * 1048576.f) * 9.5367431640625e-7f;
  return fminf(s < 6.103515625e-5f ? small : seven, KV4_SCALE_MAX);
}

__device__ __forceinline__ float wave_max(float v) {
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// Quantizes a wave's 64 values (one a lane): the lane's code; *word the group's.
__device__ __forceinline__ unsigned kv4_quantize(float x, unsigned* word) {
  const bool bad = __any(!__builtin_isfinite(x));
  const float hi = wave_max(fmaxf(x, 0.f)), lo = -wave_max(fmaxf(-x, 0.f));
  const float s = kv4_scale(hi - lo);
  const float by = s > 0.f ? s : 1.f;
  const float z = fminf(fmaxf(rintf(-lo / by), 0.f), 15.f);
  const float c = fminf(fmaxf(rintf(x / by) + z, 0.f), 15.f);
  *word = bad ? KV4_NAN : (unsigned)__builtin_bit_cast(uint16_t, (_Float16)s) | (unsigned)z;
  return bad ? 0u : (unsigned)c;
}

struct Kv4Source {
  const void* x;
  int64_t ts, hs;
};

// One wave per new token, cache head, and K or V; lane l has channels
// l, l + 64, ...
template <int DT, int DIM>
__global__ __launch_bounds__(256) void k_kv4_append(uint8_t* cache, Kv4Shape c, Kv4Sequences q, Kv4Source k, Kv4Source v) {
  typedef typename Elem<DT>::T T;
  constexpr int NG = DIM / KV4_GROUP, HALF = DIM / 2;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (unit >= q.tokens * c.heads) return;
  const int64_t t = unit / c.heads;
  const int h = (int)(unit - t * c.heads), which = blockIdx.y;
  const int b = sequence_of(q, t);
  const int64_t p = position_of(q, b, t), page = page_of(c, q, b, p);
  if (page < 0) return;
  const int P = 1 << c.page_log2, off = (int)(p & (P - 1));
  const Kv4Source src = which ? v : k;
  const T* x = (const T*)src.x + t * src.ts + h * src.hs;
  unsigned code[NG], word[NG];
#pragma unroll
  for (int g = 0; g < NG; g++) code[g] = kv4_quantize(Elem<DT>::load(x[g * 64 + lane]), &word[g]);
  uint8_t* base = cache + (page * c.heads + h) * c.head_bytes;
  // byte i of the token: K side by side, V 16 bytes apart
  uint8_t* to = which ? base + (size_t)P * HALF + (size_t)(off >> 4) * (HALF * 16) + (off & 15) : base + (size_t)off * HALF;
  const int step = which ? 16 : 1;
  if constexpr (DIM == 64) {
    const unsigned other = __shfl_xor(code[0], 32);
    if (lane < 32) to[lane * step] = (uint8_t)(code[0] | other << 4);
  } else {
#pragma unroll
    for (int g = 0; g < NG / 2; g++) to[(g * 64 + lane) * step] = (uint8_t)(code[g] | code[g + NG / 2] << 4);
  }
  uint16_t* words = (uint16_t*)(base + (size_t)P * DIM) + (off * 2 + which) * NG;
  if (lane == 0)
#pragma unroll
    for (int g = 0; g < NG; g++) words[g] = (uint16_t)word[g];
}

// One wave per new token, cache head, and K or V.
template <int DT, int DIM>
__global__ __launch_bounds__(256) void k_kv4_read(const uint8_t* cache, Kv4Shape c, Kv4Sequences q, void* k, void* v) {
  typedef typename Elem<DT>::T T;
  constexpr int NG = DIM / KV4_GROUP, HALF = DIM / 2;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (unit >= q.tokens * c.heads) return;
  const int64_t t = unit / c.heads;
  const int h = (int)(unit - t * c.heads), which = blockIdx.y;
  const int b = sequence_of(q, t);
  const int64_t p = position_of(q, b, t), page = page_of(c, q, b, p);
  T* out = (T*)(which ? v : k) + unit * DIM;
  const int P = 1 << c.page_log2, off = (int)(p & (P - 1));
  const uint8_t* base = cache + (page * c.heads + h) * c.head_bytes;
  const uint8_t* from = which ? base + (size_t)P * HALF + (size_t)(off >> 4) * (HALF * 16) + (off & 15) : base + (size_t)off * HALF;
  const int step = which ? 16 : 1;
  const uint16_t* words = (const uint16_t*)(base + (size_t)P * DIM) + (off * 2 + which) * NG;
#pragma unroll
  for (int g = 0; g < NG; g++) {
    const int d = g * 64 + lane;
    float x = 0.f;
    if (page >= 0) {
      const unsigned w = words[g], byte = from[(d % HALF) * step], code = d < HALF ? byte & 15 : byte >> 4;
      x = (float)__builtin_bit_cast(_Float16, (uint16_t)(w & 0xFFF0u)) * ((float)code - (float)(w & 15));
    }
    out[d] = Elem<DT>::store(x);
  }
}

template <int DT>
static void launch_append(const Kv4Shape& c, dim3 grid, hipStream_t s, uint8_t* cache, const Kv4Sequences& q, Kv4Source k,
                          Kv4Source v) {
  if (c.dim == 64) k_kv4_append<DT, 64><<<grid, 256, 0, s>>>(cache, c, q, k, v);
  else if (c.dim == 128) k_kv4_append<DT, 128><<<grid, 256, 0, s>>>(cache, c, q, k, v);
  else k_kv4_append<DT, 256><<<grid, 256, 0, s>>>(cache, c, q, k, v);
}

template <int DT>
static void launch_read(const Kv4Shape& c, dim3 grid, hipStream_t s, const uint8_t* cache, const Kv4Sequences& q, void* k,
                        void* v) {
  if (c.dim == 64) k_kv4_read<DT, 64><<<grid, 256, 0, s>>>(cache, c, q, k, v);
  else if (c.dim == 128) k_kv4_read<DT, 128><<<grid, 256, 0, s>>>(cache, c, q, k, v);
  else k_kv4_read<DT, 256><<<grid, 256, 0, s>>>(cache, c, q, k, v);
}

// Argument checks that append and read share; > 0: nothing to do.
static int check_cache_args(const void* cache, const Kv4Shape& c, int64_t tokens, int32_t batch, const int32_t* starts,
                            const int32_t* lens, const int32_t* table, int64_t table_pages, int32_t dtype) {
  if (!cache || ((uintptr_t)cache & 15) || !dtype_ok(dtype) || tokens < 0 || batch < 1 || table_pages < 1 || !lens || !table)
    return EXTERND_EINVAL;
  if (!starts && tokens != batch) return EXTERND_EINVAL;
  if (tokens > INT32_MAX || tokens * c.heads > INT32_MAX || table_pages > INT32_MAX) return EXTERND_EUNSUPPORTED;
  return tokens ? EXTERND_OK : 1;
}

}  // namespace externd

using namespace externd;

extern "C" {

size_t externd_kv4_page_bytes(int32_t head_dim, int32_t page_tokens) {
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return 0;
  if (page_tokens < 16 || page_tokens > 1024 || (page_tokens & (page_tokens - 1))) return 0;
  return (size_t)page_tokens * (size_t)(head_dim + head_dim / 16);
}

int externd_kv4_append(void* cache, int64_t num_pages, int32_t heads_kv, int32_t head_dim, int32_t page_tokens,
                       const void* k, const void* v, int32_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                       int64_t v_token_stride, int64_t v_head_stride, int64_t tokens, int32_t batch,
                       const int32_t* starts, const int32_t* lens, const int32_t* table, int64_t table_pages,
                       void* stream) {
  Kv4Shape c;
  if (!kv4_shape(num_pages, heads_kv, head_dim, page_tokens, &c)) return EXTERND_EINVAL;
  const int st = check_cache_args(cache, c, tokens, batch, starts, lens, table, table_pages, dtype);
  if (st) return st > 0 ? EXTERND_OK : st;
  if (!k || !v) return EXTERND_EINVAL;
  const Kv4Sequences q = {starts, lens, table, table_pages, tokens, batch};
  const Kv4Source ks = {k, k_token_stride, k_head_stride}, vs = {v, v_token_stride, v_head_stride};
  const dim3 grid((unsigned)((tokens * c.heads + 3) / 4), 2);
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) launch_append<EXTERND_F32>(c, grid, s, (uint8_t*)cache, q, ks, vs);
  else if (dtype == EXTERND_BF16) launch_append<EXTERND_BF16>(c, grid, s, (uint8_t*)cache, q, ks, vs);
  else launch_append<EXTERND_F16>(c, grid, s, (uint8_t*)cache, q, ks, vs);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

int externd_kv4_read(const void* cache, int64_t num_pages, int32_t heads_kv, int32_t head_dim, int32_t page_tokens,
                     void* k, void* v, int32_t dtype, int64_t tokens, int32_t batch, const int32_t* starts,
                     const int32_t* lens, const int32_t* table, int64_t table_pages, void* stream) {
  Kv4Shape c;
  if (!kv4_shape(num_pages, heads_kv, head_dim, page_tokens, &c)) return EXTERND_EINVAL;
  const int st = check_cache_args(cache, c, tokens, batch, starts, lens, table, table_pages, dtype);
  if (st) return st > 0 ? EXTERND_OK : st;
  if (!k || !v) return EXTERND_EINVAL;
  const Kv4Sequences q = {starts, lens, table, table_pages, tokens, batch};
  const dim3 grid((unsigned)((tokens * c.heads + 3) / 4), 2);
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) launch_read<EXTERND_F32>(c, grid, s, (const uint8_t*)cache, q, k, v);
  else if (dtype == EXTERND_BF16) launch_read<EXTERND_BF16>(c, grid, s, (const uint8_t*)cache, q, k, v);
  else launch_read<EXTERND_F16>(c, grid, s, (const uint8_t*)cache, q, k, v);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
