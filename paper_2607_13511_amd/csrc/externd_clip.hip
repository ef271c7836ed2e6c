// The norm over many tensors, and clipping by it.
#include <cmath>

#include "externd_decode.hpp"

namespace externd {

constexpr int CLIP_TENSORS = 120;       // of a launch: their descriptions are its arguments, so nothing is copied ahead of it
constexpr int64_t CLIP_CHUNK = 16384;    // entries of a chunk; a chunk is one tensor's
constexpr int CLIP_BLOCKS = 2048;       // workgroups of a launch, each with equally many chunks, and as many partial sums

struct ClipList {
  const void* in[CLIP_TENSORS];
  void* out[CLIP_TENSORS];
  int64_t size[CLIP_TENSORS];
  uint32_t first[CLIP_TENSORS];         // chunks before the tensor's
  uint8_t dtype[CLIP_TENSORS];
  int count;
  uint32_t chunks, each;                // in all, and of a workgroup
};

// The tensor that a chunk belongs to.
__device__ __forceinline__ int tensor_of(const ClipList& l, uint32_t chunk) {
  int lo = 0, hi = l.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.first[mid] <= chunk) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ double sum_of_wave(double v) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
// Over 256 threads; every thread receives it.
__device__ __forceinline__ double sum_of_block(double v, double* lds) {
  v = sum_of_wave(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Entries before the first 16-byte boundary.
template <int DT>
__device__ __forceinline__ int lead_of(const void* p, int n) {
  const int lead = (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(typename Elem<DT>::T);
  return min(lead, n);
}

template <int DT>
__device__ __forceinline__ void add_squares(const void* p, int n, double* sum) {
  typedef typename Elem<DT>::T T;
  constexpr int E = Vec<DT>::E, U = 8;
  const T* x = (const T*)p;
  const int lead = lead_of<DT>(p, n), nv = (n - lead) / E, tail = n - lead - nv * E;
  const v4u* v = (const v4u*)(x + lead);
  for (int i = threadIdx.x; i < nv; i += 256 * U) {
    v4u x[U];
#pragma unroll
    for (int u = 0; u < U; u++) x[u] = i + u * 256 < nv ? v[i + u * 256] : v4u{0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < U; u++) {
      float f[E];
      Vec<DT>::unpack(x[u], f);
#pragma unroll
      for (int e = 0; e < E; e++) sum[e & 3] = fma((double)f[e], (double)f[e], sum[e & 3]);
    }
  }
  const int i = threadIdx.x;
  if (i < lead + tail) {
    const double f = Elem<DT>::load(x[i < lead ? i : nv * E + i]);
    sum[0] = fma(f, f, sum[0]);
  }
}

__global__ __launch_bounds__(256) void k_squares(ClipList l, double* partial) {
  __shared__ double lds[4];
  double sum[4] = {};
  const uint32_t c0 = blockIdx.x * l.each, c1 = min(c0 + l.each, l.chunks);
  int t = c0 < c1 ? tensor_of(l, c0) : 0;
  for (uint32_t c = c0; c < c1; c++) {
    while (t + 1 < l.count && l.first[t + 1] <= c) t++;
    const int64_t at = (int64_t)(c - l.first[t]) * CLIP_CHUNK;
    const int n = (int)min(CLIP_CHUNK, l.size[t] - at);
    if (l.dtype[t] == EXTERND_F32) add_squares<EXTERND_F32>((const float*)l.in[t] + at, n, sum);
    else if (l.dtype[t] == EXTERND_BF16) add_squares<EXTERND_BF16>((const uint16_t*)l.in[t] + at, n, sum);
    else add_squares<EXTERND_F16>((const uint16_t*)l.in[t] + at, n, sum);
  }
  const double all = sum_of_block((sum[0] + sum[1]) + (sum[2] + sum[3]), lds);
  if (threadIdx.x == 0) partial[blockIdx.x] = all;
}

template <int DT>
__device__ __forceinline__ void scale_entries(const void* p, void* q, int n, float before, float factor) {
  typedef typename Elem<DT>::T T;
  constexpr int E = Vec<DT>::E;
  const T* x = (const T*)p;
  T* y = (T*)q;
  if (((uintptr_t)p ^ (uintptr_t)q) & 15) {
    const int nv = n / E, tail = n - nv * E;
#pragma unroll 4
    for (int i = threadIdx.x; i < nv; i += 256) {
      float f[E];
      Vec<DT>::unpack(load_any<T>(x + (int64_t)i * E), f);
#pragma unroll
      for (int e = 0; e < E; e++) f[e] = f[e] * before * factor;
      store_any<T>(y + (int64_t)i * E, Vec<DT>::pack(f));
    }
    if ((int)threadIdx.x < tail) y[nv * E + threadIdx.x] = Elem<DT>::store(Elem<DT>::load(x[nv * E + threadIdx.x]) * before * factor);
    return;
  }
  const int lead = lead_of<DT>(p, n), nv = (n - lead) / E, tail = n - lead - nv * E;
#pragma unroll 4
  for (int i = threadIdx.x; i < nv; i += 256) {
    float f[E];
    Vec<DT>::unpack(__builtin_nontemporal_load((const v4u*)(x + lead) + i), f);
#pragma unroll
    for (int e = 0; e < E; e++) f[e] = f[e] * before * factor;
    __builtin_nontemporal_store(Vec<DT>::pack(f), (v4u*)(y + lead) + i);
  }
  const int i = threadIdx.x;
  if (i < lead + tail) {
    const int at = i < lead ? i : nv * E + i;
    y[at] = Elem<DT>::store(Elem<DT>::load(x[at]) * before * factor);
  }
}

// The partial sums' total is formed by every workgroup for itself, in the same order.
__global__ __launch_bounds__(256) void k_scale(ClipList l, const double* partial, int partials, double max_norm, float* norm,
                                               int first_launch) {
  __shared__ double lds[4];
  double sum = 0;
  for (int i = threadIdx.x; i < partials; i += 256) sum += partial[i];
  const double total = sqrt(sum_of_block(sum, lds));
  if (first_launch && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
  const double ratio = max_norm / total;
  const bool whole = total == 0.0 || ratio >= 1.0 || max_norm == INFINITY;
  // a ratio that fp32 holds with fewer bits is split: half of its exponent, a power of two, is multiplied first, and
  // what that takes below fp32's normal numbers ends as 0; so does every product with 2^-280, which is not split
  // (from 2^-300 on half of the exponent would be none of fp32's powers, and the rest infinite)
  const float before = ratio < 0x1p-100 && ratio > 0x1p-280 ? exp2f((float)(ilogb(ratio) / 2)) : 1.f;
  const float factor = whole ? 1.f : (float)(ratio / before);      // NaN: it stays
  // from the stretch's end, which k_squares read last and which may still be in the cache
  const uint32_t c0 = blockIdx.x * l.each, c1 = min(c0 + l.each, l.chunks);
  int t = c0 < c1 ? tensor_of(l, c1 - 1) : 0;
  for (uint32_t c = c1; c-- > c0;) {
    while (l.first[t] > c) t--;
    if (whole && l.in[t] == l.out[t]) continue;
    const int64_t at = (int64_t)(c - l.first[t]) * CLIP_CHUNK;
    const int n = (int)min(CLIP_CHUNK, l.size[t] - at);
    if (l.dtype[t] == EXTERND_F32) scale_entries<EXTERND_F32>((const float*)l.in[t] + at, (float*)l.out[t] + at, n, before, factor);
    else if (l.dtype[t] == EXTERND_BF16)
      scale_entries<EXTERND_BF16>((const uint16_t*)l.in[t] + at, (uint16_t*)l.out[t] + at, n, before, factor);
    else scale_entries<EXTERND_F16>((const uint16_t*)l.in[t] + at, (uint16_t*)l.out[t] + at, n, before, factor);
  }
}

// Calls `launch(list, workgroups)` for the tensors, CLIP_TENSORS at a time.
template <typename F>
static void each_list(int64_t count, const void* const* tensors, void* const* out, const int64_t* sizes, const int32_t* dtypes, F launch) {
  ClipList l;
  l.count = 0;
  l.chunks = 0;
  auto go = [&] {
    if (!l.count) return;
    const uint32_t blocks = l.chunks < CLIP_BLOCKS ? l.chunks : CLIP_BLOCKS;
    l.each = (l.chunks + blocks - 1) / blocks;
    launch(l, (l.chunks + l.each - 1) / l.each);
    l.count = 0;
    l.chunks = 0;
  };
  for (int64_t i = 0; i < count; i++) {
    if (!sizes[i]) continue;
    const int64_t chunks = (sizes[i] + CLIP_CHUNK - 1) / CLIP_CHUNK;
    if (l.count == CLIP_TENSORS) go();
    l.in[l.count] = tensors[i];
    l.out[l.count] = out ? out[i] : (void*)tensors[i];
    l.size[l.count] = sizes[i];
    l.dtype[l.count] = (uint8_t)dtypes[i];
    l.first[l.count++] = l.chunks;
    l.chunks += (uint32_t)chunks;
  }
  go();
}

}  // namespace externd

using namespace externd;

extern "C" {

size_t externd_clip_gradients_workspace_bytes(int64_t count) {
  if (count < 0 || count > (1 << 20)) return 0;
  return (size_t)((count + CLIP_TENSORS - 1) / CLIP_TENSORS + 1) * CLIP_BLOCKS * sizeof(double);
}

int externd_clip_gradients(int64_t count, const void* const* tensors, void* const* out, const int64_t* sizes,
                           const int32_t* dtypes, double max_norm, float* norm, void* workspace,
                           size_t workspace_bytes, void* stream) {
  if (count < 0 || (count && (!tensors || !sizes || !dtypes)) || !norm || !(max_norm >= 0)) return EXTERND_EINVAL;
  if (count > (1 << 20)) return EXTERND_EUNSUPPORTED;
  int64_t all = 0;
  for (int64_t i = 0; i < count; i++) {
    if (sizes[i] < 0 || !dtype_ok(dtypes[i]) || (sizes[i] && (!tensors[i] || (out && !out[i])))) return EXTERND_EINVAL;
    const uintptr_t odd = (uintptr_t)dtype_bytes(dtypes[i]) - 1;
    if (sizes[i] && (((uintptr_t)tensors[i] & odd) || (out && ((uintptr_t)out[i] & odd)))) return EXTERND_EINVAL;
    // chunks are counted in 31 bits
    if (sizes[i] > (int64_t)INT32_MAX * CLIP_CHUNK || (all += (sizes[i] + CLIP_CHUNK - 1) / CLIP_CHUNK) > INT32_MAX)
      return EXTERND_EUNSUPPORTED;
  }
  if ((uintptr_t)workspace & 255) return EXTERND_EINVAL;
  if (!workspace || workspace_bytes < externd_clip_gradients_workspace_bytes(count)) return EXTERND_EWORKSPACE;
  double* const partial = (double*)workspace;
  const hipStream_t s = (hipStream_t)stream;
  int partials = 0;
  each_list(count, tensors, out, sizes, dtypes, [&](const ClipList& l, uint32_t blocks) {
    k_squares<<<blocks, 256, 0, s>>>(l, partial + partials);
    partials += (int)blocks;
  });
  if (!partials || max_norm == INFINITY) {
    ClipList none;
    none.count = 0;
    none.chunks = none.each = 0;
    k_scale<<<1, 256, 0, s>>>(none, partial, partials, max_norm, norm, 1);
  } else {
    int first = 1;
    each_list(count, tensors, out, sizes, dtypes, [&](const ClipList& l, uint32_t blocks) {
      k_scale<<<blocks, 256, 0, s>>>(l, partial, partials, max_norm, norm, first);
      first = 0;
    });
  }
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
