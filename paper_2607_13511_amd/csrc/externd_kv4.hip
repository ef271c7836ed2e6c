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

struct Kv4Source {
  const void* x;
  int64_t ts, hs;
};

// New tokens are taken by blocks of 16 positions, as the cache holds V.  The
// blocks of sequence b (at most n / 16 + 2 for n tokens) have the numbers from
// first_block(b) on, so that a block finds its sequence by bisection and no
// prefix sum is needed; numbers behind a sequence's last block are empty.
__device__ __forceinline__ int64_t first_block(const Kv4Sequences& q, int b) {
  return q.starts ? q.starts[b] / 16 + 2 * (int64_t)b : b;
}
static int64_t block_count(const Kv4Sequences& q) { return q.starts ? q.tokens / 16 + 2 * (int64_t)q.batch : q.batch; }

struct Kv4Block {
  int64_t page;        // -1: the cache has no place for the block
  int64_t token;       // call's token at the block's first position (below the sequence's first: not new)
  int64_t first, end;  // new positions
  int64_t at;          // the block's first position
};
__device__ __forceinline__ bool find_block(const Kv4Shape& c, const Kv4Sequences& q, int64_t number, Kv4Block* k) {
  int lo = 0, hi = q.batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first_block(q, mid) <= number) lo = mid; else hi = mid - 1;
  }
  const int64_t t0 = q.starts ? q.starts[lo] : lo, t1 = q.starts ? q.starts[lo + 1] : lo + 1;
  k->end = max(q.lens[lo], 0);
  k->first = k->end - (t1 - t0);
  const int64_t i = number - first_block(q, lo), b0 = k->first >> 4;      // rounds down below 0 too
  k->at = (b0 + i) * 16;
  if (i < 0 || t0 < 0 || t1 > q.tokens || k->at >= k->end) return false;
  k->token = t0 + (k->at - k->first);
  k->page = page_of(c, q, lo, k->at);
  return true;
}

// Across the lanes that hold a group: all four of a token, or two at 256 channels.
template <int DIM>
__device__ __forceinline__ float group_max(float v) {
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, true)));
  if (DIM < 256) v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, true)));
  return v;
}

// Codes of N values of this lane, their group spread over lanes; returns the group's word.
template <int DIM, int N>
__device__ __forceinline__ unsigned kv4_quantize(float* x) {
  float hi = 0.f, lo = 0.f, odd = 0.f;      // odd: above 0 where an entry is not finite
#pragma unroll
  for (int i = 0; i < N; i++) {
    hi = fmaxf(hi, x[i]);
    lo = fmaxf(lo, -x[i]);
    odd = __builtin_isfinite(x[i]) ? odd : 1.f;
  }
  hi = group_max<DIM>(hi);
  lo = -group_max<DIM>(lo);
  const bool bad = group_max<DIM>(odd) > 0.f;
  const float s = kv4_scale(hi - lo);
  const float by = s > 0.f ? s : 1.f;
  const float z = fminf(fmaxf(rintf(-lo / by), 0.f), 15.f);
#pragma unroll
  for (int i = 0; i < N; i++) x[i] = bad ? 0.f : fminf(fmaxf(rintf(x[i] / by) + z, 0.f), 15.f);
  return bad ? KV4_NAN : (unsigned)__builtin_bit_cast(uint16_t, (_Float16)s) | (unsigned)z;
}

// One wave per block of 16 positions, cache head, and K or V.  Lane 4 t + c has
// token t's byte columns c H / 4 ..: as many channels below D / 2 and, in the
// high nibbles, above.  V's bytes are turned through LDS, so that a lane writes
// 16 tokens' bytes of one column at once.  Bound by memory: 6.8 K tokens of 8
// heads of 128 in bf16, 28 MB read and 7 written, in 15.6 us (2.3 TB/s).
// Entries are read one by one (VEC false) only where heads do not start at
// multiples of 16 bytes; so, and with V's bytes scattered, this and reading
// back took 82 us together, now 24.
template <int DT, int DIM, bool VEC>
__global__ __launch_bounds__(256) void k_kv4_append(uint8_t* cache, Kv4Shape c, Kv4Sequences q, Kv4Source k, Kv4Source v,
                                                    int64_t blocks) {
  typedef typename Elem<DT>::T T;
  constexpr int NG = DIM / KV4_GROUP, HALF = DIM / 2, N = HALF / 4;
  __shared__ __align__(16) uint8_t turn[4][16][HALF + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = lane >> 2, part = lane & 3;
  const int64_t unit = (int64_t)blockIdx.x * 4 + wave;
  const int64_t number = unit / (2 * c.heads);
  if (number >= blocks) return;
  const int rest = (int)(unit - number * 2 * c.heads), which = rest >= c.heads, h = rest - which * c.heads;
  Kv4Block B;
  if (!find_block(c, q, number, &B) || B.page < 0) return;
  const int P = 1 << c.page_log2, off = (int)(B.at & (P - 1));
  const bool in = B.at + t >= B.first && B.at + t < B.end;
  const bool full = B.at >= B.first && B.at + 16 <= B.end;
  const Kv4Source src = which ? v : k;
  float x[2][N];
  if (in) {
    const T* p = (const T*)src.x + (B.token + t) * src.ts + h * src.hs + part * N;
    load_n<DT, N, VEC>(p, x[0]);
    load_n<DT, N, VEC>(p + HALF, x[1]);
  } else {
#pragma unroll
    for (int i = 0; i < 2 * N; i++) x[i / N][i % N] = 0.f;
  }
  unsigned word[2];
  if constexpr (DIM == 64) word[0] = word[1] = kv4_quantize<DIM, 2 * N>(&x[0][0]);
  else {
    word[0] = kv4_quantize<DIM, N>(x[0]);
    word[1] = kv4_quantize<DIM, N>(x[1]);
  }
  unsigned bytes[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; i++) {
    bytes[i] = 0;
#pragma unroll
    for (int j = 0; j < 4; j++) bytes[i] |= ((unsigned)x[0][4 * i + j] | (unsigned)x[1][4 * i + j] << 4) << (8 * j);
  }
  uint8_t* base = cache + (B.page * c.heads + h) * c.head_bytes;
  uint16_t* words = (uint16_t*)(base + (size_t)P * DIM) + ((off + t) * 2 + which) * NG;
  if (in) {
    if (DIM == 64 && part == 0) words[0] = (uint16_t)word[0];
    if (DIM == 128 && part == 0) *(unsigned*)words = word[0] | word[1] << 16;
    if (DIM == 256 && !(part & 1)) {
      words[part >> 1] = (uint16_t)word[0];
      words[2 + (part >> 1)] = (uint16_t)word[1];
    }
  }
  if (!which) {
    if (in) {
      unsigned* to = (unsigned*)(base + (size_t)(off + t) * HALF + part * N);
#pragma unroll
      for (int i = 0; i < N / 4; i++) to[i] = bytes[i];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N / 4; i++) *(unsigned*)&turn[wave][t][part * N + 4 * i] = bytes[i];
  __builtin_amdgcn_wave_barrier();      // the wave's own LDS, in order
  uint8_t* to = base + (size_t)P * HALF + (size_t)(off >> 4) * (HALF * 16);
  const int t0 = (int)max((int64_t)0, B.first - B.at), t1 = (int)min((int64_t)16, B.end - B.at);
#pragma unroll
  for (int col0 = 0; col0 < HALF; col0 += 64) {
    const int col = col0 + lane;
    if (col >= HALF) break;
    if (full) {
      v4u o;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        o[i] = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) o[i] |= (unsigned)turn[wave][4 * i + j][col] << (8 * j);
      }
      *(v4u*)(to + col * 16) = o;
    } else {
      for (int j = t0; j < t1; j++) to[col * 16 + j] = turn[wave][j][col];
    }
  }
}

// The same units, the other way: 6.8 K tokens in 10.8 us (3.3 TB/s).
template <int DT, int DIM>
__global__ __launch_bounds__(256) void k_kv4_read(const uint8_t* cache, Kv4Shape c, Kv4Sequences q, void* k, void* v,
                                                  int64_t blocks) {
  typedef typename Elem<DT>::T T;
  constexpr int NG = DIM / KV4_GROUP, HALF = DIM / 2, N = HALF / 4;
  __shared__ __align__(16) uint8_t turn[4][HALF][16 + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = lane >> 2, part = lane & 3;
  const int64_t unit = (int64_t)blockIdx.x * 4 + wave;
  const int64_t number = unit / (2 * c.heads);
  if (number >= blocks) return;
  const int rest = (int)(unit - number * 2 * c.heads), which = rest >= c.heads, h = rest - which * c.heads;
  Kv4Block B;
  if (!find_block(c, q, number, &B)) return;
  const int P = 1 << c.page_log2, off = (int)(B.at & (P - 1));
  const bool in = B.at + t >= B.first && B.at + t < B.end;
  const uint8_t* base = cache + (max(B.page, (int64_t)0) * c.heads + h) * c.head_bytes;
  const uint16_t* words = (const uint16_t*)(base + (size_t)P * DIM) + ((off + t) * 2 + which) * NG;
  const unsigned w0 = words[DIM == 256 ? part >> 1 : 0], w1 = words[DIM == 64 ? 0 : DIM == 128 ? 1 : 2 + (part >> 1)];
  unsigned bytes[N / 4];
  if (!which) {
    const unsigned* from = (const unsigned*)(base + (size_t)(off + t) * HALF + part * N);
#pragma unroll
    for (int i = 0; i < N / 4; i++) bytes[i] = from[i];
  } else {
    const uint8_t* from = base + (size_t)P * HALF + (size_t)(off >> 4) * (HALF * 16);
#pragma unroll
    for (int col0 = 0; col0 < HALF; col0 += 64) {
      const int col = col0 + lane;
      if (col >= HALF) break;
      const v4u o = *(const v4u*)(from + col * 16);
#pragma unroll
      for (int i = 0; i < 4; i++) *(unsigned*)&turn[wave][col][4 * i] = o[i];
    }
    __builtin_amdgcn_wave_barrier();      // the wave's own LDS, in order
#pragma unroll
    for (int i = 0; i < N / 4; i++) {
      bytes[i] = 0;
#pragma unroll
      for (int j = 0; j < 4; j++) bytes[i] |= (unsigned)turn[wave][part * N + 4 * i + j][t] << (8 * j);
    }
  }
  if (!in) return;
  const float s0 = (float)__builtin_bit_cast(_Float16, (uint16_t)(w0 & 0xFFF0u)), z0 = (float)(w0 & 15);
  const float s1 = (float)__builtin_bit_cast(_Float16, (uint16_t)(w1 & 0xFFF0u)), z1 = (float)(w1 & 15);
  float x[2][N];
#pragma unroll
  for (int i = 0; i < N; i++) {
    const unsigned byte = bytes[i / 4] >> (8 * (i % 4)) & 0xFF;
    x[0][i] = B.page < 0 ? 0.f : s0 * ((float)(byte & 15) - z0);
    x[1][i] = B.page < 0 ? 0.f : s1 * ((float)(byte >> 4) - z1);
  }
  T* out = (T*)(which ? v : k) + ((B.token + t) * c.heads + h) * DIM + part * N;
  store_n<DT, N, true>(out, x[0]);
  store_n<DT, N, true>(out + HALF, x[1]);
}

template <int DT, bool VEC>
static void launch_append(const Kv4Shape& c, int64_t n, dim3 grid, hipStream_t s, uint8_t* cache, const Kv4Sequences& q,
                          Kv4Source k, Kv4Source v) {
  if (c.dim == 64) k_kv4_append<DT, 64, VEC><<<grid, 256, 0, s>>>(cache, c, q, k, v, n);
  else if (c.dim == 128) k_kv4_append<DT, 128, VEC><<<grid, 256, 0, s>>>(cache, c, q, k, v, n);
  else k_kv4_append<DT, 256, VEC><<<grid, 256, 0, s>>>(cache, c, q, k, v, n);
}
template <int DT>
static void launch_append(bool vec, const Kv4Shape& c, int64_t n, dim3 grid, hipStream_t s, uint8_t* cache,
                          const Kv4Sequences& q, Kv4Source k, Kv4Source v) {
  if (vec) launch_append<DT, true>(c, n, grid, s, cache, q, k, v);
  else launch_append<DT, false>(c, n, grid, s, cache, q, k, v);
}

template <int DT>
static void launch_read(const Kv4Shape& c, int64_t n, dim3 grid, hipStream_t s, const uint8_t* cache, const Kv4Sequences& q,
                        void* k, void* v) {
  if (c.dim == 64) k_kv4_read<DT, 64><<<grid, 256, 0, s>>>(cache, c, q, k, v, n);
  else if (c.dim == 128) k_kv4_read<DT, 128><<<grid, 256, 0, s>>>(cache, c, q, k, v, n);
  else k_kv4_read<DT, 256><<<grid, 256, 0, s>>>(cache, c, q, k, v, n);
}

// Argument checks that append and read share; > 0: nothing to do.
static int check_cache_args(const void* cache, const Kv4Shape& c, int64_t tokens, int32_t batch, const int32_t* starts,
                            const int32_t* lens, const int32_t* table, int64_t table_pages, int32_t dtype) {
  if (!cache || ((uintptr_t)cache & 15) || !dtype_ok(dtype) || tokens < 0 || batch < 1 || table_pages < 1 || !lens || !table)
    return EXTERND_EINVAL;
  if (!starts && tokens != batch) return EXTERND_EINVAL;
  if (tokens > INT32_MAX || tokens * c.heads > INT32_MAX || batch > (1 << 24) || table_pages > INT32_MAX) return EXTERND_EUNSUPPORTED;
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
  const int64_t n = block_count(q);
  if ((n * 2 * c.heads + 3) / 4 > MAX_THREADS / 256) return EXTERND_EUNSUPPORTED;
  const dim3 grid((unsigned)((n * 2 * c.heads + 3) / 4));
  const hipStream_t s = (hipStream_t)stream;
  const int es = dtype_bytes(dtype);
  const bool vec = rows_aligned(k, k_token_stride, k_head_stride, es) && rows_aligned(v, v_token_stride, v_head_stride, es);
  if (dtype == EXTERND_F32) launch_append<EXTERND_F32>(vec, c, n, grid, s, (uint8_t*)cache, q, ks, vs);
  else if (dtype == EXTERND_BF16) launch_append<EXTERND_BF16>(vec, c, n, grid, s, (uint8_t*)cache, q, ks, vs);
  else launch_append<EXTERND_F16>(vec, c, n, grid, s, (uint8_t*)cache, q, ks, vs);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

int externd_kv4_read(const void* cache, int64_t num_pages, int32_t heads_kv, int32_t head_dim, int32_t page_tokens,
                     void* k, void* v, int32_t dtype, int64_t tokens, int32_t batch, const int32_t* starts,
                     const int32_t* lens, const int32_t* table, int64_t table_pages, void* stream) {
  Kv4Shape c;
  if (!kv4_shape(num_pages, heads_kv, head_dim, page_tokens, &c)) return EXTERND_EINVAL;
  const int st = check_cache_args(cache, c, tokens, batch, starts, lens, table, table_pages, dtype);
  if (st) return st > 0 ? EXTERND_OK : st;
  if (!k || !v || (((uintptr_t)k | (uintptr_t)v) & 15)) return EXTERND_EINVAL;
  const Kv4Sequences q = {starts, lens, table, table_pages, tokens, batch};
  const int64_t n = block_count(q);
  if ((n * 2 * c.heads + 3) / 4 > MAX_THREADS / 256) return EXTERND_EUNSUPPORTED;
  const dim3 grid((unsigned)((n * 2 * c.heads + 3) / 4));
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) launch_read<EXTERND_F32>(c, n, grid, s, (const uint8_t*)cache, q, k, v);
  else if (dtype == EXTERND_BF16) launch_read<EXTERND_BF16>(c, n, grid, s, (const uint8_t*)cache, q, k, v);
  else launch_read<EXTERND_F16>(c, n, grid, s, (const uint8_t*)cache, q, k, v);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
