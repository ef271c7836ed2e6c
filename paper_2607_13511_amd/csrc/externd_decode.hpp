// What the decoding operators share: the three storage types, where a new
// token is, and where a cache keeps it.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "externd.h"

namespace externd {

// A launch holds fewer than 2^32 threads a dimension.
constexpr int64_t MAX_THREADS = ((int64_t)1 << 32) - 1;

inline bool dtype_ok(int32_t d) { return d == EXTERND_F32 || d == EXTERND_BF16 || d == EXTERND_F16; }
inline int dtype_bytes(int32_t d) { return d == EXTERND_F32 ? 4 : 2; }

// Storage type of a dtype code, widened to and rounded from fp32 (to nearest,
// ties to even; a NaN stays one).
template <int DT> struct Elem;
template <> struct Elem<EXTERND_F32> {
  typedef float T;
  static __device__ __forceinline__ float load(float v) { return v; }
  static __device__ __forceinline__ float store(float v) { return v; }
};
template <> struct Elem<EXTERND_F16> {
  typedef _Float16 T;
  static __device__ __forceinline__ float load(_Float16 v) { return (float)v; }
  static __device__ __forceinline__ _Float16 store(float v) { return (_Float16)v; }
};
template <> struct Elem<EXTERND_BF16> {
  typedef __bf16 T;
  static __device__ __forceinline__ float load(__bf16 v) {
    return __uint_as_float((unsigned)__builtin_bit_cast(uint16_t, v) << 16);
  }
  static __device__ __forceinline__ __bf16 store(float v) { return (__bf16)v; }
};

typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

// 16 bytes of a type.
template <int DT> struct Vec {
  static constexpr int E = DT == EXTERND_F32 ? 4 : 8;      // entries
  static __device__ __forceinline__ void unpack(v4u v, float* x) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if constexpr (DT == EXTERND_F32) x[i] = __uint_as_float(v[i]);
      else if constexpr (DT == EXTERND_BF16) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
      } else {
        x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)v[i]);
        x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(v[i] >> 16));
      }
    }
  }
  static __device__ __forceinline__ v4u pack(const float* x) {
    v4u v;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if constexpr (DT == EXTERND_F32) v[i] = __float_as_uint(x[i]);
      else
        v[i] = (unsigned)__builtin_bit_cast(uint16_t, Elem<DT>::store(x[2 * i])) |
               (unsigned)__builtin_bit_cast(uint16_t, Elem<DT>::store(x[2 * i + 1])) << 16;
    }
    return v;
  }
};

// N entries at p, in 16-byte loads or stores where VEC (p is 16-byte aligned then).
template <int DT, int N, bool VEC>
__device__ __forceinline__ void load_n(const typename Elem<DT>::T* p, float* x) {
  constexpr int E = Vec<DT>::E;
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < N / E; i++) Vec<DT>::unpack(((const v4u*)p)[i], x + i * E);
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = Elem<DT>::load(p[i]);
  }
}
template <int DT, int N, bool VEC>
__device__ __forceinline__ void store_n(typename Elem<DT>::T* p, const float* x) {
  constexpr int E = Vec<DT>::E;
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < N / E; i++) ((v4u*)p)[i] = Vec<DT>::pack(x + i * E);
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = Elem<DT>::store(x[i]);
  }
}
// Whether every head of an array starts at a multiple of 16 bytes.
inline bool rows_aligned(const void* p, int64_t token_stride, int64_t head_stride, int bytes) {
  return !(((uintptr_t)p | (uint64_t)(token_stride * bytes) | (uint64_t)(head_stride * bytes)) & 15);
}

// The cache's layout for one page size and head width (include/externd.h).
struct Kv4Shape {
  int64_t num_pages;
  int heads, dim, page_log2;
  int64_t head_bytes;   // of one head of one page
};
constexpr int KV4_GROUP = 64;          // channels that share a scale
constexpr float KV4_SCALE_MAX = 4352.f;
constexpr unsigned KV4_NAN = 0x7E00u;  // word of a group that held a NaN or an infinity

struct Kv4Sequences {
  const int32_t* starts;
  const int32_t* lens;
  const int32_t* table;
  int64_t table_pages, tokens;
  int batch;
};

// Page of position p of sequence b, or -1.
__device__ __forceinline__ int64_t page_of(const Kv4Shape& c, const Kv4Sequences& s, int b, int64_t p) {
  if (p < 0) return -1;
  const int64_t i = p >> c.page_log2;
  if (i >= s.table_pages) return -1;
  const int64_t page = s.table[(int64_t)b * s.table_pages + i];
  return page >= 0 && page < c.num_pages ? page : -1;
}

// Fills the shape; false where the arguments are not a cache's.
inline bool kv4_shape(int64_t num_pages, int32_t heads, int32_t dim, int32_t page_tokens, Kv4Shape* c) {
  const size_t bytes = externd_kv4_page_bytes(dim, page_tokens);
  if (!bytes || num_pages < 1 || num_pages > INT32_MAX || heads < 1 || heads > 4096) return false;
  c->num_pages = num_pages;
  c->heads = heads;
  c->dim = dim;
  c->page_log2 = __builtin_ctz((unsigned)page_tokens);
  c->head_bytes = (int64_t)bytes;
  return true;
}

}  // namespace externd
