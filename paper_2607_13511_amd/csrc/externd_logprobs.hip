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

__device__ __forceinline__ float value_of(uint64_t key) {
  int b = (int)((unsigned)(key >> 32) ^ 0x80000000u);
  return __int_as_float(b < 0 ? b ^ 0x7FFFFFFF : b);
}
__device__ __forceinline__ int64_t index_of(uint64_t key) { return (int64_t)(0xFFFFFFFFu - (unsigned)key); }

typedef float f32x4 __attribute__((ext_vector_type(4)));

// A larger of two that is a NaN where one of them is.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Entries of a row before its first 16-byte boundary.
template <int DT>
__device__ __forceinline__ int64_t row_head(const void* p, int64_t n) {
  constexpr int B = DT == EXTERND_F32 ? 4 : 2;
  const int64_t h = (int64_t)((16 - ((uintptr_t)p & 15)) & 15) / B;
  return h < n ? h : n;
}

// The value of lane ^ D, without LDS: DPP within 16 lanes, row swaps beyond.
template <int D>
__device__ __forceinline__ unsigned xor_lane(unsigned v) {
  if constexpr (D == 1) return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true);
  else if constexpr (D == 2) return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true);
  else if constexpr (D == 4) {      // mirrored within 8 lanes (^ 7), then within 4 (^ 3)
    const int m = __builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true);
    return (unsigned)__builtin_amdgcn_update_dpp(0, m, 0x1B, 0xF, 0xF, true);
  } else if constexpr (D == 8) return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, true);
  else if constexpr (D == 16) {
    const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? s[0] : s[1];
  } else {
    const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? s[0] : s[1];
  }
}
template <int D>
__device__ __forceinline__ uint64_t xor_lane64(uint64_t v) {
  return (uint64_t)xor_lane<D>((unsigned)(v >> 32)) << 32 | xor_lane<D>((unsigned)v);
}
// One step of a bitonic network: the lower lane of a pair keeps the smaller key where `up`.
template <int D>
__device__ __forceinline__ uint64_t order_pair(uint64_t k, bool up) {
  const uint64_t o = xor_lane64<D>(k);
  const bool low = !(threadIdx.x & D);
  return (low == up) == (k < o) ? k : o;
}
template <int SIZE, int D>
__device__ __forceinline__ uint64_t order_steps(uint64_t k, bool up) {
  k = order_pair<D>(k, up);
  if constexpr (D > 1) return order_steps<SIZE, D / 2>(k, up);
  else return k;
}
// Rising over the wave.
template <int SIZE = 2>
__device__ __forceinline__ uint64_t sort_rising(uint64_t k) {
  k = order_steps<SIZE, SIZE / 2>(k, SIZE == 64 || !(threadIdx.x & SIZE));
  if constexpr (SIZE < 64) return sort_rising<SIZE * 2>(k);
  else return k;
}
template <int SIZE, int D>
__device__ __forceinline__ unsigned order_steps32(unsigned k, bool up) {
  const unsigned o = xor_lane<D>(k);
  k = (!(threadIdx.x & D) == up) ? min(k, o) : max(k, o);
  if constexpr (D > 1) return order_steps32<SIZE, D / 2>(k, up);
  else return k;
}
template <int SIZE = 2>
__device__ __forceinline__ unsigned sort_rising32(unsigned k) {
  k = order_steps32<SIZE, SIZE / 2>(k, SIZE == 64 || !(threadIdx.x & SIZE));
  if constexpr (SIZE < 64) return sort_rising32<SIZE * 2>(k);
  else return k;
}
// The 64 largest of a falling and a rising list, falling.
__device__ __forceinline__ uint64_t merge_lists(uint64_t falling, uint64_t rising) {
  return order_steps<64, 32>(falling > rising ? falling : rising, false);
}

__device__ __forceinline__ float wave_sum(float v) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// The largest keys that a wave has seen, lane i the i-th, and those not sorted in yet.
constexpr int BEST_WORDS = 128 + 128 + 8;      // 64-bit words of LDS
struct Best {
  uint64_t key;          // 0: none
  uint64_t* waiting;     // LDS, 128 keys
  float* some;           // LDS, 16 lanes' entries, and where each lane's begin
  unsigned* whose;
  int count;             // of them
  int top;
  float bar;             // entries not above it are out; a NaN (nothing compares) while fewer than `top` are known

  __device__ __forceinline__ void init(uint64_t* lds, int k) {
    key = 0;
    waiting = lds;
    some = (float*)(lds + 128);
    whose = (unsigned*)(some + 256);
    count = 0;
    top = k;
    bar = NAN;
  }
  // Sorts the first (at most 64) waiting keys in.
  __device__ __forceinline__ void merge() {
    const int lane = threadIdx.x & 63;
    key = merge_lists(key, sort_rising(lane < count ? waiting[lane] : 0));
    const int left = count - 64;
    if (left > 0 && lane < left) waiting[lane] = waiting[64 + lane];
    count = left > 0 ? left : 0;
    const uint64_t last = (uint64_t)(unsigned)__builtin_amdgcn_readlane((unsigned)(key >> 32), top - 1) << 32 |
                          (unsigned)__builtin_amdgcn_readlane((unsigned)key, top - 1);
    bar = last ? value_of(last) : bar;
  }
  // `in`: this lane's x may be among the largest.
  __device__ __forceinline__ void offer(bool in, float x, unsigned index) {
    const uint64_t mask = __ballot(in);
    if (!mask) return;
    const int lane = threadIdx.x & 63;
    if (in) waiting[count + __popcll(mask & ((1ull << lane) - 1))] = order_key(x, index);
    count += __popcll(mask);
    if (count >= 64) merge();
  }
  // First entries: with `top` lanes or more, the top-th largest of their
  // maxima is a bar already (as many entries are not below it), where sorting
  // in all of them would take eight rounds.  Above 32 it is taken of two maxima a
  // lane: one lets a quarter of the entries pass (8 rows of 65536 in fp32 with 64
  // largest: 42 us, with two 38.5).
  __device__ __forceinline__ void start(float big, float more, bool present, bool two) {
    const int n = __popcll(__ballot(present));
    if (n < top) return;
    unsigned k;
    if (two && top > 32) {
      const unsigned a = sort_rising32(present ? (unsigned)(order_key(big, 0) >> 32) : 0u);
      const unsigned b = ~sort_rising32(present ? ~(unsigned)(order_key(more, 0) >> 32) : ~0u);      // falling
      k = order_steps32<64, 32>(max(a, b), true);      // the 64 largest of both
    } else k = sort_rising32(present ? (unsigned)(order_key(two ? larger(big, more) : big, 0) >> 32) : 0u);
    bar = value_of((uint64_t)(unsigned)__builtin_amdgcn_readlane(k, 64 - top) << 32);
  }
  // The lanes of `may` have one at least.  Sixteen of them at a time put all of
  // theirs side by side, so that 64 are looked at together.
  template <int E, int G>
  __device__ __forceinline__ void search(const float (*x)[E], uint64_t may, unsigned index, float was) {
    constexpr int S = E * G;
    const int lane = threadIdx.x & 63, rank = __popcll(may & ((1ull << lane) - 1)), n = __popcll(may);
    const bool mine = may >> lane & 1;
    for (int r0 = 0; r0 < n; r0 += 16) {
      __builtin_amdgcn_wave_barrier();      // the wave's own LDS, in order
      if (mine && rank >= r0 && rank < r0 + 16) {
        if constexpr (E >= 4) {
#pragma unroll
          for (int g = 0; g < G; g++)
#pragma unroll
            for (int e = 0; e < E; e += 4)
              *(f32x4*)(some + (rank - r0) * S + g * E + e) = f32x4{x[g][e], x[g][e + 1], x[g][e + 2], x[g][e + 3]};
        } else some[rank - r0] = x[0][0];
        whose[rank - r0] = index;
      }
      __builtin_amdgcn_wave_barrier();
      const int m = min(16, n - r0) * S;
      for (int j = lane; j - lane < m; j += 64) {
        const int at = j < m ? j : 0, slot = at % S;
        const float v = some[at];
        const unsigned i = whose[at / S] + (slot / E) * (64 * E) + slot % E;
        offer(j < m && !(v <= was) && !(v < bar), v, i);
      }
    }
  }
};

// Sums of a row (or a part of it) of one lane: with y = (x - ref) scale log2(e),
// s = sum 2^y and t = sum 2^y y.  `ref` is the same in a wave: the largest entry
// of the first ones, and moved only when one is 2^8 larger, so that entries
// need no maximum of their own, and y is one fused multiply-add.
struct Sums {
  float ref, s, t;
  __device__ __forceinline__ void move(float to, float c) {
    const float d = fmaxf((ref - to) * c, -1e9f), f = __builtin_amdgcn_exp2f(d);
    t = s > 0.f ? fmaf(s, d, t) * f : s;      // s is 0 or NaN otherwise
    s *= f;
    ref = to;
  }
};

// Wave-wide: G times E entries of every lane (present: whether the lane has
// any), those of g from index + 64 E g on.
template <int E, int G>
__device__ __forceinline__ void take(const float (*x)[E], bool present, unsigned index, float c, Sums& a, Best& best, bool first) {
  float part[G];
#pragma unroll
  for (int g = 0; g < G; g++) {
    part[g] = x[g][0];
#pragma unroll
    for (int e = 1; e < E; e++) part[g] = larger(part[g], x[g][e]);
  }
  const float big = present ? G > 1 ? larger(part[0], part[G - 1]) : part[0] : -INFINITY;
  if (first) a.ref = fmaxf(wave_max(big), -3.402823466e38f);
  else if (__any((big - a.ref) * c > 8.f)) a.move(wave_max(big), c);
  if (best.top) {
    // earlier entries have lower indices, so what equals their bar is out; what these ones raise it to is not
    const float was = best.bar;
    if (was != was && E * G > 1) best.start(part[0], part[G - 1], present, G > 1);
    const uint64_t may = __ballot(present && !(big <= was) && !(big < best.bar));
    if (may) best.search<E, G>(x, may, index, was);
  }
  float s[4] = {0.f, 0.f, 0.f, 0.f}, t[4] = {0.f, 0.f, 0.f, 0.f};
  const float from = a.ref * c;
  if (fabsf(from) < 1e30f) {
#pragma unroll
    for (int g = 0; g < G; g++)
#pragma unroll
      for (int e = 0; e < E; e++) {
        const float y = larger(fmaf(x[g][e], c, -from), -200.f), w = __builtin_amdgcn_exp2f(y);      // 2^-200 is 0
        s[e & 3] += w;
        t[e & 3] = fmaf(w, y, t[e & 3]);
      }
  } else {                             // the product alone may overflow: the difference first
#pragma unroll
    for (int g = 0; g < G; g++)
#pragma unroll
      for (int e = 0; e < E; e++) {
        const float y = larger((x[g][e] - a.ref) * c, -200.f), w = __builtin_amdgcn_exp2f(y);
        s[e & 3] += w;
        t[e & 3] = fmaf(w, y, t[e & 3]);
      }
  }
  a.s += present ? (s[0] + s[1]) + (s[2] + s[3]) : 0.f;
  a.t += present ? (t[0] + t[1]) + (t[2] + t[3]) : 0.f;
}

// What a row's sums say (lane 0) and the largest logits (lanes below top).
template <int DT>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t r, float ref, float s, float t, uint64_t key) {
  typedef typename Elem<DT>::T T;
  const T* x = (const T*)a.logits + r * a.stride;
  const int lane = threadIdx.x & 63;
  const float ln2 = 0.69314718055994530942f, l2 = log2f(s);
  const bool none = s == 0.f;      // nothing but -infinity
  const float lse = none ? -INFINITY : fmaf(ln2, l2, ref * a.scale);
  if (lane == 0) {
    if (a.lse) a.lse[r] = lse;
    if (a.entropy) a.entropy[r] = none ? 0.f : ln2 * (l2 - t / s);
    if (a.logprob) {
      const int64_t y = a.targets[r];
      const float z = y >= 0 && y < a.vocab ? Elem<DT>::load(x[y]) * a.scale : 0.f;
      a.logprob[r] = y < 0 ? 0.f : y >= a.vocab ? NAN : none ? -INFINITY : z - lse;
    }
  }
  if (lane < a.top) {
    a.top_ids[r * a.top + lane] = index_of(key);
    a.top_logprobs[r * a.top + lane] = none ? -INFINITY : value_of(key) * a.scale - lse;
  }
}

constexpr int MAX_WAVES = 16;

// One workgroup per row: its waves take equal stretches (`each` 16-byte vectors,
// a multiple of 64), in a single pass with four 16-byte loads of every lane in
// flight ahead of those in work, and are joined in LDS.  One exponential and
// one fused multiply-add for y an entry; entries above the bar (the least of
// the wave's largest so far) are rare, so only their lanes go through LDS.
// Bound by memory: 2048 rows of 150001 in bf16, 615 MB, in 129 us (4.8 TB/s) with
// the 20 largest, 113 without (5.4).  8 rows of 65536 in fp32 with the 5 largest in
// 16 us, 10 without: sorting, which so few rows cannot hide.
template <int DT>
__global__ __launch_bounds__(64 * MAX_WAVES) void k_logprobs(LogprobArgs a, int64_t each) {
  typedef typename Elem<DT>::T T;
  constexpr int E = Vec<DT>::E, U = 4;
  extern __shared__ uint64_t waiting[];      // BEST_WORDS a wave, then the pool: 128 a wave
  __shared__ Sums sums[MAX_WAVES];
  __shared__ float bars[MAX_WAVES];
  __shared__ int pooled;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.logits + r * a.stride;
  const int64_t head = row_head<DT>(x, a.vocab), nv = (a.vocab - head) / E, tail = head + nv * E;
  const int64_t v0 = min(wave * each, nv), v1 = wave == waves - 1 ? nv : min(v0 + each, nv);
  const v4u* v = (const v4u*)(x + head);
  const float c = a.scale * 1.44269504088896340736f;
  Sums sum = {-3.402823466e38f, 0.f, 0.f};
  Best best;
  best.init(waiting + wave * BEST_WORDS, a.top);
  bool first = true;
  int64_t i = v0;
  const int64_t blocks = (v1 - v0) / (64 * U);
  v4u A[U], B[U];
  auto load = [&](v4u* d, int64_t at) {
#pragma unroll
    for (int u = 0; u < U; u++) d[u] = v[at + u * 64 + lane];
  };
  auto work = [&](const v4u* d, int64_t at) {
#pragma unroll
    for (int u = 0; u < U; u += 2) {
      float y[2][E];
      Vec<DT>::unpack(d[u], y[0]);
      Vec<DT>::unpack(d[u + 1], y[1]);
      take<E, 2>(y, true, (unsigned)(head + (at + u * 64 + lane) * E), c, sum, best, first);
      first = false;
    }
  };
  if (blocks > 0) load(A, i);
  if (wave == 0 && head) {
    float one[1][1] = {{-INFINITY}};
    if (lane < head) one[0][0] = Elem<DT>::load(x[lane]);
    take<1, 1>(one, lane < head, (unsigned)lane, c, sum, best, first);
    first = false;
  }
  for (int64_t k = 0; k < blocks; k += 2, i += 2 * 64 * U) {
    if (k + 1 < blocks) load(B, i + 64 * U);
    work(A, i);
    if (k + 1 >= blocks) break;
    if (k + 2 < blocks) load(A, i + 2 * 64 * U);
    work(B, i + 64 * U);
  }
  for (i = v0 + blocks * 64 * U; i < v1; i += 64) {
    const bool in = i + lane < v1;
    float y[1][E];
    Vec<DT>::unpack(v[in ? i + lane : v1 - 1], y[0]);
    take<E, 1>(y, in, (unsigned)(head + (i + lane) * E), c, sum, best, first);
    first = false;
  }
  if (wave == waves - 1 && tail < a.vocab) {
    const bool in = tail + lane < a.vocab;
    float one[1][1] = {{-INFINITY}};
    if (in) one[0][0] = Elem<DT>::load(x[tail + lane]);
    take<1, 1>(one, in, (unsigned)(tail + lane), c, sum, best, first);
  }
  sum.s = wave_sum(sum.s);
  sum.t = wave_sum(sum.t);
  if (waves == 1) {
    if (best.count) best.merge();
  } else {
    if (lane == 0) {
      sums[wave] = sum;
      bars[wave] = best.bar;
      if (wave == 0) pooled = 0;
    }
    __syncthreads();
    if (a.top) {
      // what is not below any wave's bar goes into one pool, a little over `top` keys, which wave 0 sorts
      uint64_t* const pool = waiting + waves * BEST_WORDS;
      float bar = -INFINITY;
      for (int w = 0; w < waves; w++) bar = fmaxf(bar, bars[w]);      // passes over NaN: none yet
      const auto give = [&](uint64_t key) {
        if (key && !(value_of(key) < bar)) pool[atomicAdd(&pooled, 1)] = key;
      };
      give(best.key);
      if (lane < best.count) give(best.waiting[lane]);
      __syncthreads();
    }
    if (wave) return;
    Sums one = lane < waves ? sums[lane] : Sums{-3.402823466e38f, 0.f, 0.f};
    const float ref = wave_max(one.s > 0.f ? one.ref : -3.402823466e38f);
    if (one.s != 0.f) one.move(ref, c);
    sum = {ref, wave_sum(one.s), wave_sum(one.s != 0.f ? one.t : 0.f)};
    best.key = 0;
    if (a.top)
      for (int k = 0; k < pooled; k += 64)
        best.key = merge_lists(best.key, sort_rising(k + lane < pooled ? waiting[waves * BEST_WORDS + k + lane] : 0));
  }
  write_row<DT>(a, r, sum.ref, sum.s, sum.t, best.key);
}

struct LogprobGradArgs {
  const void* logits;
  void* grad;
  int64_t rows, vocab, stride, grad_stride;
  const int64_t* targets;
  float scale;
  const float *lse, *entropy, *g_logprob, *g_entropy;
  int64_t first;      // row of the grid's first
};

// One workgroup per row and stretch of it: 16-byte loads and stores where a
// row of both arrays starts at the same place within 16 bytes, else one by one
// (218 us where the other takes 96).  Bound by memory: 2048 rows of 65537 in bf16,
// 537 MB, in 96 us (5.6 TB/s).
template <int DT>
__global__ __launch_bounds__(256) void k_logprobs_grad(LogprobGradArgs a) {
  typedef typename Elem<DT>::T T;
  constexpr int E = Vec<DT>::E, U = 4;
  const int64_t r = a.first + blockIdx.y;
  const T* x = (const T*)a.logits + r * a.stride;
  T* d = (T*)a.grad + r * a.grad_stride;
  const int64_t y = a.targets ? a.targets[r] : -1;
  const float lse = a.lse[r], g = a.g_logprob && y >= 0 ? a.g_logprob[r] : 0.f;
  const float ge = a.g_entropy ? a.g_entropy[r] : 0.f, h = a.g_entropy ? a.entropy[r] : 0.f;
  const float scale = a.scale;
  // grad = scale ([v = y] g - p (g + ge (lp + h))), lp = ln p
  auto entry = [&](float v, int64_t i) -> float {
    const float lp = fmaf(v, scale, -lse), p = __builtin_amdgcn_exp2f(lp * 1.44269504088896340736f);
    float o = p > 0.f ? -p * fmaf(ge, lp + h, g) : p == 0.f || lse == -INFINITY ? 0.f : p;
    if (i == y) o += g;
    return o * scale;
  };
  const int64_t stretch = (int64_t)256 * U * E;
  const int64_t head = row_head<DT>(x, a.vocab), nv = (a.vocab - head) / E, tail = head + nv * E;
  if ((((uintptr_t)x ^ (uintptr_t)d) & 15) != 0) {
    const int64_t end = min((int64_t)(blockIdx.x + 1) * stretch, a.vocab);
    for (int64_t i = (int64_t)blockIdx.x * stretch + threadIdx.x; i < end; i += 256)
      d[i] = Elem<DT>::store(entry(Elem<DT>::load(x[i]), i));
    return;
  }
  const int64_t v0 = (int64_t)blockIdx.x * (256 * U) + threadIdx.x;
  const v4u* from = (const v4u*)(x + head);
  v4u* to = (v4u*)(d + head);
  v4u in[U];
#pragma unroll
  for (int u = 0; u < U; u++)
    if (v0 + u * 256 < nv) in[u] = from[v0 + u * 256];
#pragma unroll
  for (int u = 0; u < U; u++)
    if (v0 + u * 256 < nv) {
      float f[E];
      Vec<DT>::unpack(in[u], f);
      const int64_t i = head + (v0 + u * 256) * E;
#pragma unroll
      for (int e = 0; e < E; e++) f[e] = entry(f[e], i + e);
      to[v0 + u * 256] = Vec<DT>::pack(f);
    }
  if (blockIdx.x == 0) {      // what is off the 16-byte boundaries: fewer than 2 E entries
    const int64_t i = (int64_t)threadIdx.x < head ? threadIdx.x : tail + threadIdx.x - head;
    if (i < a.vocab) d[i] = Elem<DT>::store(entry(Elem<DT>::load(x[i]), i));
  }
}

// Waves of a row: 4096 in all where there is work for them, sixteen a CU, a wave
// not below 2048 entries.  A power of two rounded down: 940 rows of 65536 with
// four waves 35, 42, 62 us (bf16; 5, 20, 64 largest), with eight 41, 53, 88.
static int waves_of(int64_t rows, int64_t vocab) {
  int64_t want = (4096 + rows - 1) / rows;
  const int64_t most = (vocab + 2047) / 2048;
  want = want > most ? most : want;
  int w = 1;
  while (2 * w <= want && w < MAX_WAVES) w *= 2;
  return w;
}

static void launch_logprobs_grad(LogprobGradArgs a, int32_t dtype, int64_t r0, int64_t rows, int64_t stretches, hipStream_t s) {
  a.first = r0;
  const dim3 grid((unsigned)stretches, (unsigned)rows);
  if (dtype == EXTERND_F32) k_logprobs_grad<EXTERND_F32><<<grid, 256, 0, s>>>(a);
  else if (dtype == EXTERND_BF16) k_logprobs_grad<EXTERND_BF16><<<grid, 256, 0, s>>>(a);
  else k_logprobs_grad<EXTERND_F16><<<grid, 256, 0, s>>>(a);
}

template <int DT>
static void launch_logprobs(const LogprobArgs& a, hipStream_t s) {
  const int waves = waves_of(a.rows, a.vocab);
  const int64_t each = ((a.vocab / Vec<DT>::E + waves - 1) / waves + 63) & ~(int64_t)63;
  const size_t lds = a.top ? (size_t)waves * (BEST_WORDS + 128) * sizeof(uint64_t) : 0;
  k_logprobs<DT><<<dim3((unsigned)a.rows), 64 * waves, lds, s>>>(a, each);
}

static bool logprob_sizes_ok(int64_t rows, int64_t vocab, int32_t top) {
  return rows >= 0 && vocab >= 1 && top >= 0 && top <= EXTERND_LOGPROBS_MAX_TOP && top <= vocab;
}

}  // namespace externd

using namespace externd;

extern "C" {

size_t externd_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int32_t top) {
  (void)rows, (void)vocab, (void)top;      // a row is one workgroup's
  return 0;
}

int externd_token_logprobs(const void* logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t row_stride,
                           const int64_t* targets, float scale, int32_t top, float* logprob, float* entropy,
                           float* lse, float* top_logprobs, int64_t* top_ids, void* workspace,
                           size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dtype) || !logprob_sizes_ok(rows, vocab, top) || row_stride < vocab || !(scale > 0) ||
      !std::isfinite(scale) || (top && (!top_logprobs || !top_ids)) || (rows && !logits) || (logprob && rows && !targets))
    return EXTERND_EINVAL;
  if (rows > MAX_THREADS / 64 || vocab > INT32_MAX) return EXTERND_EUNSUPPORTED;      // many rows: one wave each
  (void)workspace, (void)workspace_bytes;
  if (!rows) return EXTERND_OK;
  const LogprobArgs a = {logits, rows, vocab, row_stride, targets, scale, top, logprob, entropy, lse, top_logprobs, top_ids};
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) launch_logprobs<EXTERND_F32>(a, s);
  else if (dtype == EXTERND_BF16) launch_logprobs<EXTERND_BF16>(a, s);
  else launch_logprobs<EXTERND_F16>(a, s);
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
                             g_logprob, g_entropy, 0};
  const hipStream_t s = (hipStream_t)stream;
  const int64_t stretch = 256 * 4 * (dtype == EXTERND_F32 ? 4 : 8);
  for (int64_t r0 = 0; r0 < rows; r0 += 65535) {      // rows are the grid's second dimension
    launch_logprobs_grad(a, dtype, r0, rows - r0 < 65535 ? rows - r0 : 65535, (vocab + stretch - 1) / stretch, s);
  }
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
