// Rows of a table by token, and their gradient: the tokens are sorted, and what
// belongs to one row is summed in a fixed order.
#include <cmath>

#include "externd_decode.hpp"

namespace externd {

// Units of a row: vectors of 16 bytes, the last one short or shifted back.
template <int DT>
__host__ __device__ inline unsigned units_of(int64_t width) {
  return (unsigned)((width + Vec<DT>::E - 1) / Vec<DT>::E);
}

// `base` units before this workgroup's: the row and the unit in it of the first.
__device__ __forceinline__ void split_units(int64_t base, unsigned units, int64_t* row, unsigned* unit) {
  if (base >> 32) {
    *row = base / units;
    *unit = (unsigned)(base - *row * units);
  } else {
    const unsigned r = (unsigned)base / units;
    *row = r;
    *unit = (unsigned)base - r * units;
  }
}

struct EmbedArgs {
  const void* table;
  void* out;
  const int64_t* ids;
  int64_t vocab, width, table_stride, out_stride, tokens;
  float scale;
};

constexpr int EMBED_U = 4;      // units of a thread

// A thread moves four vectors of 16 bytes that are a workgroup's width apart, so
// that the loads of ids, and then of rows, are in flight together.  A row's last
// vector ends with the row: where the width is no multiple, it writes some
// entries a second time, with the same values.
template <int DT>
__global__ __launch_bounds__(256) void k_embedding(EmbedArgs a) {
  typedef typename Elem<DT>::T T;
  constexpr int E = Vec<DT>::E;
  const unsigned units = units_of<DT>(a.width);
  int64_t row;
  unsigned unit;
  split_units((int64_t)blockIdx.x * (256 * EMBED_U), units, &row, &unit);
  int64_t t[EMBED_U], id[EMBED_U];
  int64_t c[EMBED_U];
#pragma unroll
  for (int u = 0; u < EMBED_U; u++) {
    const unsigned at = unit + u * 256 + threadIdx.x, r = at / units;
    t[u] = row + r;
    const int64_t b = (int64_t)(at - r * units) * E;
    c[u] = b + E <= a.width ? b : a.width >= E ? a.width - E : 0;
    id[u] = t[u] < a.tokens ? a.ids[t[u]] : -1;
  }
  if (a.width >= E) {
    v4u v[EMBED_U];
#pragma unroll
    for (int u = 0; u < EMBED_U; u++)
      v[u] = id[u] >= 0 && id[u] < a.vocab ? load_any<T>((const T*)a.table + id[u] * a.table_stride + c[u]) : v4u{0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < EMBED_U; u++) {
      if (t[u] >= a.tokens) continue;
      float x[E];
      Vec<DT>::unpack(v[u], x);
      const bool in = id[u] >= 0 && id[u] < a.vocab;      // a scale of 0 or below must not make -0 of a missing row
#pragma unroll
      for (int e = 0; e < E; e++) x[e] = in ? x[e] * a.scale : 0.f;
      store_any<T>((T*)a.out + t[u] * a.out_stride + c[u], Vec<DT>::pack(x));
    }
    return;
  }
  for (int u = 0; u < EMBED_U; u++) {      // rows of fewer than 16 bytes
    if (t[u] >= a.tokens) continue;
    for (int64_t e = 0; e < a.width; e++)
      ((T*)a.out)[t[u] * a.out_stride + e] =
          Elem<DT>::store(id[u] >= 0 && id[u] < a.vocab ? Elem<DT>::load(((const T*)a.table)[id[u] * a.table_stride + e]) * a.scale : 0.f);
  }
}

// ---------------------------------------------------------------------------
// tokens by id
// ---------------------------------------------------------------------------
constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64;
constexpr int64_t RANK_TOKENS = 16384;      // up to here every token is compared with every other

struct SortArgs {
  const int64_t* ids;
  int64_t tokens, vocab;
  unsigned *keys[2], *places[2];            // sorted so far: the id (vocab where there is none) and the token
  // tokens past RANK_TOKENS: passes over digits of `bits` bits
  int blocks, passes, bits;
  unsigned* counts;                         // blocks x digits of the present pass
  int scanned;                              // counts are those of the blocks before, and one row more of all of them
  // what becomes zero meanwhile: rows zero_from .. zero_to - 1
  void* zero;
  int64_t zero_from, zero_to, zero_width, zero_stride;
};

__device__ __forceinline__ unsigned key_of(const SortArgs& a, int64_t i) {
  const int64_t id = a.ids[i];
  return (unsigned)(id >= 0 && id < a.vocab ? id : a.vocab);
}

// Rows of zeros, by the workgroups behind the sorting ones.
template <int DT>
__device__ void zero_rows(const SortArgs& a, int64_t block, int64_t blocks) {
  typedef typename Elem<DT>::T T;
  constexpr int E = Vec<DT>::E;
  T* const z = (T*)a.zero + a.zero_from * a.zero_stride;
  const int64_t rows = a.zero_to - a.zero_from;
  if (a.zero_stride == a.zero_width) {
    const int64_t n = rows * a.zero_width, lead = min((int64_t)((16 - ((uintptr_t)z & 15)) & 15) / (int64_t)sizeof(T), n);
    const int64_t nv = (n - lead) / E;
    for (int64_t i = block * SORT_THREADS + threadIdx.x; i < nv; i += blocks * SORT_THREADS) ((v4u*)(z + lead))[i] = v4u{0, 0, 0, 0};
    if (block == 0) {
      if ((int64_t)threadIdx.x < lead) z[threadIdx.x] = T(0);
      if (threadIdx.x < n - lead - nv * E) z[lead + nv * E + threadIdx.x] = T(0);
    }
    return;
  }
  const int64_t units = units_of<DT>(a.zero_width);
  for (int64_t i = block * SORT_THREADS + threadIdx.x; i < rows * units; i += blocks * SORT_THREADS) {
    const int64_t r = i / units, c = (i - r * units) * E;
    T* const to = z + r * a.zero_stride + c;
    if (c + E <= a.zero_width) store_any(to, v4u{0, 0, 0, 0});
    else
      for (int64_t e = 0; c + e < a.zero_width; e++) to[e] = T(0);
  }
}

// A token's place is the number of tokens before it in the order of (id, token):
// a workgroup counts for 32 tokens, a lane for one of them over every second key of
// its wave's stretch.  All keys are in LDS; a compare and an add each.  8191
// tokens are 67 million comparisons, 4 us of the card, in one launch, where
// passes over digits are five dependent ones.
template <int DT>
__global__ __launch_bounds__(SORT_THREADS) void k_rank(SortArgs a) {
  extern __shared__ unsigned keys[];        // the tokens rounded up to 128, then the waves' counts
  const int blocks = (int)((a.tokens + 31) / 32), all = (int)((a.tokens + 127) & ~(int64_t)127);
  if (blockIdx.x >= (unsigned)blocks) return zero_rows<DT>(a, blockIdx.x - blocks, gridDim.x - blocks);
  for (int i = threadIdx.x; i < all; i += SORT_THREADS) keys[i] = i < a.tokens ? key_of(a, i) : ~0u;
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, token = blockIdx.x * 32 + (lane & 31);
  const unsigned key = keys[token < all ? token : 0];
  unsigned count = 0;
  // eight keys a step, four in each half of the wave; of equal keys those of earlier tokens count
  for (int i = wave * 8; i < all; i += SORT_WAVES * 8) {
    const int at = i + (lane >> 5) * 4;
    const v4u k = *(const v4u*)(keys + at);
    if (i + 8 <= (int)blockIdx.x * 32) {
#pragma unroll
      for (int e = 0; e < 4; e++) count += k[e] <= key;
    } else if (i >= (int)blockIdx.x * 32 + 32) {
#pragma unroll
      for (int e = 0; e < 4; e++) count += k[e] < key;
    } else
      for (int e = 0; e < 4; e++) count += k[e] < key || (k[e] == key && at + e < token);
  }
  unsigned* const counts = keys + all;
  counts[threadIdx.x] = count;
  __syncthreads();
  if (threadIdx.x < 32 && token < a.tokens) {
    unsigned to = 0;
    for (int w = 0; w < 2 * SORT_WAVES; w++) to += counts[w * 32 + threadIdx.x];
    a.keys[0][to] = key;
    a.places[0][to] = (unsigned)token;
  }
}

// More tokens: stable passes over digits, least significant first.
constexpr int SORT_BITS = 10, SORT_BINS = 1 << SORT_BITS;
constexpr int SORT_ITEMS = 4;               // tokens of a lane
constexpr int64_t SORT_BLOCK = SORT_THREADS * SORT_ITEMS;

template <int DT>
__global__ __launch_bounds__(SORT_THREADS) void k_sort_count(SortArgs a, int pass) {
  __shared__ unsigned n[SORT_BINS];
  if (blockIdx.x >= (unsigned)a.blocks) return zero_rows<DT>(a, blockIdx.x - a.blocks, gridDim.x - a.blocks);
  const int bins = 1 << a.bits, shift = pass * a.bits;
  for (int i = threadIdx.x; i < bins; i += SORT_THREADS) n[i] = 0;
  __syncthreads();
  const int64_t b0 = (int64_t)blockIdx.x * SORT_BLOCK, b1 = min(b0 + SORT_BLOCK, a.tokens);
  unsigned key[SORT_ITEMS];
#pragma unroll
  for (int k = 0; k < SORT_ITEMS; k++) {
    const int64_t i = b0 + k * SORT_THREADS + threadIdx.x;
    key[k] = i >= b1 ? 0 : pass ? a.keys[(pass - 1) & 1][i] : key_of(a, i);
  }
#pragma unroll
  for (int k = 0; k < SORT_ITEMS; k++)
    if (b0 + k * SORT_THREADS + threadIdx.x < b1) {
      const unsigned digit = key[k] >> shift & (bins - 1);
      // those that have the first lane's digit are added at once: frequent tokens would queue at one address
      const bool common = digit == (unsigned)__builtin_amdgcn_readfirstlane(digit);
      const uint64_t m = __ballot(common);
      if (!common) atomicAdd(&n[digit], 1u);
      else if ((threadIdx.x & 63) == __ffsll((unsigned long long)m) - 1) atomicAdd(&n[digit], (unsigned)__popcll(m));
    }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += SORT_THREADS) a.counts[(int64_t)blockIdx.x * bins + i] = n[i];
}

// Counts of each block become those of the blocks before it.
__global__ __launch_bounds__(64) void k_sort_scan(SortArgs a) {
  const int bins = 1 << a.bits, bin = blockIdx.x * 64 + threadIdx.x;
  if (bin >= bins) return;
  unsigned sum = 0;
#pragma unroll 8
  for (int b = 0; b < a.blocks; b++) {
    const unsigned n = a.counts[(int64_t)b * bins + bin];
    a.counts[(int64_t)b * bins + bin] = sum;
    sum += n;
  }
  a.counts[(int64_t)a.blocks * bins + bin] = sum;
}

// Each wave takes a stretch of the workgroup's tokens in order, all of it in
// registers.  Lanes with the same digit find each other by a ballot for each of
// its bits.  Places follow from counts alone, so they do not depend on what runs first.
template <int DT>
__global__ __launch_bounds__(SORT_THREADS) void k_sort_place(SortArgs a, int pass) {
  __shared__ unsigned at[SORT_WAVES][SORT_BINS];       // of each wave: how many of a digit, then where its first one goes
  __shared__ unsigned sums[SORT_WAVES];
  if (blockIdx.x >= (unsigned)a.blocks) return zero_rows<DT>(a, blockIdx.x - a.blocks, gridDim.x - a.blocks);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << a.bits, shift = pass * a.bits;
  const int64_t b0 = (int64_t)blockIdx.x * SORT_BLOCK, b1 = min(b0 + SORT_BLOCK, a.tokens);
  const int64_t w0 = min(b0 + wave * (SORT_BLOCK / SORT_WAVES), b1), w1 = min(w0 + SORT_BLOCK / SORT_WAVES, b1);
  unsigned key[SORT_ITEMS], place[SORT_ITEMS], local[SORT_ITEMS];
#pragma unroll
  for (int k = 0; k < SORT_ITEMS; k++) {
    const int64_t i = w0 + k * 64 + lane;
    key[k] = i >= w1 ? 0 : pass ? a.keys[(pass - 1) & 1][i] : key_of(a, i);
    place[k] = i < w1 && pass ? a.places[(pass - 1) & 1][i] : (unsigned)i;
  }
  for (int i = threadIdx.x; i < SORT_WAVES << a.bits; i += SORT_THREADS) at[i >> a.bits][i & (bins - 1)] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < SORT_ITEMS; k++) {
    const bool in = w0 + k * 64 + lane < w1;
    const unsigned digit = key[k] >> shift & (bins - 1);
    uint64_t same = __ballot(in);
    for (int b = 0; b < a.bits; b++) {
      const uint64_t m = __ballot(digit >> b & 1);
      same &= digit >> b & 1 ? m : ~m;
    }
    const unsigned rank = __popcll(same & ((1ull << lane) - 1)), before = at[wave][digit];
    local[k] = before + rank;
    __builtin_amdgcn_wave_barrier();        // all have read before the next count is written
    if (in && rank == 0) at[wave][digit] = before + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  unsigned total = 0, earlier = 0;
  const int bin = threadIdx.x;
  if (bin < bins) {
    for (int w = 0; w < SORT_WAVES; w++) {
      const unsigned n = at[w][bin];
      at[w][bin] = total;
      total += n;
    }
    if (a.scanned) {
      earlier = a.counts[(int64_t)blockIdx.x * bins + bin];
      total = a.counts[(int64_t)a.blocks * bins + bin];
    } else {
      total = 0;
#pragma unroll 8
      for (int b = 0; b < a.blocks; b++) {
        const unsigned n = a.counts[(int64_t)b * bins + bin];
        if (b < (int)blockIdx.x) earlier += n;
        total += n;
      }
    }
  }
  unsigned upto = total;                    // sum over the digits up to this one
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  unsigned first = upto - total + earlier;
  for (int w = 0; w < wave; w++) first += sums[w];
  if (bin < bins)
    for (int w = 0; w < SORT_WAVES; w++) at[w][bin] += first;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < SORT_ITEMS; k++)
    if (w0 + k * 64 + lane < w1) {
      const unsigned to = at[wave][key[k] >> shift & (bins - 1)] + local[k];
      a.keys[pass & 1][to] = key[k];
      a.places[pass & 1][to] = place[k];
    }
}

// ---------------------------------------------------------------------------
// sums of the tokens of an id
// ---------------------------------------------------------------------------
constexpr int SUM_TOKENS = 16;      // places of a stretch, in the sorted order
constexpr int JOIN_WAVES = 16, JOIN_ALONE = 16;

struct SumArgs {
  const void* grad;
  void* table;
  int64_t tokens, width, grad_stride, table_stride, vocab, stretches;
  const unsigned *keys, *places;
  float* parts;                     // stretches x {begun before, begun here} x padded width
  int64_t part_width;
  float scale;
  int accumulate;
};

// Columns c + skip .. c + n - 1 of a row's gradient, n <= N.
template <int DT, int N>
__device__ __forceinline__ void write_sum(const SumArgs& a, unsigned key, int64_t c, int skip, int n, const float* sum) {
  typedef typename Elem<DT>::T T;
  T* const to = (T*)a.table + (int64_t)key * a.table_stride + c;
  if (n == N && !skip && N == Vec<DT>::E) {
    float x[N];
    if (a.accumulate) Vec<DT>::unpack(load_any<T>(to), x);
#pragma unroll
    for (int e = 0; e < N; e++) x[e] = a.accumulate ? fmaf(sum[e], a.scale, x[e]) : sum[e] * a.scale;
    store_any<T>(to, Vec<DT>::pack(x));
  } else
#pragma unroll
    for (int e = 0; e < N; e++)
      if (e >= skip && e < n) to[e] = Elem<DT>::store(a.accumulate ? fmaf(sum[e], a.scale, Elem<DT>::load(to[e])) : sum[e] * a.scale);
}

// The first place whose key is `key` or above, by a wave, 64 probes at a time.
__device__ __forceinline__ int64_t first_place(const SumArgs& a, unsigned key, int64_t lo, int64_t hi) {
  const int lane = threadIdx.x & 63;      // places before lo are below, those from hi on are not
  while (lo < hi) {
    const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
    const int below = __popcll(__ballot(at < hi && a.keys[at < hi ? at : lo] < key));
    if (!below) return lo;
    hi = min(lo + below * step, hi);
    lo += (below - 1) * step + 1;
  }
  return lo;
}

// A workgroup sums a stretch of sorted places over a part of the width, a
// vector of 16 bytes a thread (the last one shifted back into the row); the
// stretch's keys and places come in one load of a wave's lanes, and all its rows
// are loaded ahead of their sums.  Runs that lie in the stretch are finished
// here, the others leave a part.
template <int DT>
__global__ __launch_bounds__(256) void k_embedding_sum(SumArgs a) {
  typedef typename Elem<DT>::T T;
  constexpr int E = Vec<DT>::E;
  const int lane = threadIdx.x & 63;
  const int64_t s = blockIdx.x, p0 = s * SUM_TOKENS;
  const int count = (int)min((int64_t)SUM_TOKENS, a.tokens - p0);
  // lane 0: the place before the stretch, 1 ..: its places, and the one behind it
  const int64_t mine = p0 + lane - 1;
  const bool there = lane < SUM_TOKENS + 2 && mine >= 0 && mine < a.tokens;
  const unsigned keys = there ? a.keys[mine] : ~0u, places = there ? a.places[mine] : 0;
  const int64_t c0 = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * E, c = a.width < E ? 0 : min(c0, a.width - E);
  const int skip = (int)min(c0 - c, (int64_t)E), n = (int)min((int64_t)E, a.width);      // skip = E: nothing is this thread's
  v4u x[SUM_TOKENS];
#pragma unroll
  for (int i = 0; i < SUM_TOKENS; i++) {
    const unsigned key = __builtin_amdgcn_readlane(keys, i + 1);
    if (i >= count || key >= a.vocab) continue;
    const T* from = (const T*)a.grad + (int64_t)__builtin_amdgcn_readlane(places, i + 1) * a.grad_stride + c;
    if (a.width >= E) x[i] = load_any(from);
    else {
      float y[E];
#pragma unroll
      for (int e = 0; e < E; e++) y[e] = e < n ? Elem<DT>::load(from[e]) : 0.f;
      x[i] = Vec<DT>::pack(y);
    }
  }
  float sum[E] = {};
  bool begun = __builtin_amdgcn_readlane(keys, 1) == __builtin_amdgcn_readlane(keys, 0);      // before this stretch
#pragma unroll
  for (int i = 0; i < SUM_TOKENS; i++) {
    const unsigned key = __builtin_amdgcn_readlane(keys, i + 1), next = __builtin_amdgcn_readlane(keys, i + 2);
    if (i >= count || key >= a.vocab) return;
    float y[E];
    Vec<DT>::unpack(x[i], y);
#pragma unroll
    for (int e = 0; e < E; e++) sum[e] += y[e];
    if (next == key && i + 1 < count) continue;
    if (begun || next == key) {
      float* to = a.parts + (2 * s + (begun ? 0 : 1)) * a.part_width + c;
      if (!skip && n == E) {
#pragma unroll
        for (int e = 0; e < E; e += 4) *(float4*)(to + e) = float4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
      } else
#pragma unroll
        for (int e = 0; e < E; e++)
          if (e >= skip && e < n) to[e] = sum[e];
    } else
      write_sum<DT, E>(a, key, c, skip, n, sum);
#pragma unroll
    for (int e = 0; e < E; e++) sum[e] = 0.f;
    begun = false;
  }
}

// Columns c .. c + 3 of parts q0 .. q1 - 1 of the run that begins in stretch s.
template <int UNROLL>
__device__ __forceinline__ float4 sum_parts(const SumArgs& a, int64_t s, int64_t q0, int64_t q1, int64_t c) {
  float4 sum = {0.f, 0.f, 0.f, 0.f};
  if (c < a.width) {
    for (int64_t q = q0; q < q1; q += UNROLL) {
      float4 x[UNROLL];
#pragma unroll
      for (int i = 0; i < UNROLL; i++) {
        x[i] = float4{0.f, 0.f, 0.f, 0.f};
        if (q + i < q1) x[i] = *(const float4*)(a.parts + (2 * (s + q + i) + (q + i ? 0 : 1)) * a.part_width + c);
      }
#pragma unroll
      for (int i = 0; i < UNROLL; i++)
        sum.x += x[i].x, sum.y += x[i].y, sum.z += x[i].z, sum.w += x[i].w;
    }
  }
  return sum;
}

// The runs that cross a stretch's end: each is joined where it crosses its first
// one.  A workgroup takes 256 columns and looks at as many ends as it has waves:
// a wave joins a run of few parts by itself; to longer ones all waves come
// together, take equal stretches of the parts and are joined in order.
template <int DT>
__global__ __launch_bounds__(64 * JOIN_WAVES) void k_embedding_join(SumArgs a) {
  __shared__ float4 part[JOIN_WAVES][64];
  __shared__ int long_runs[JOIN_WAVES];      // parts, of a run that all waves join
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = ((int64_t)blockIdx.y * 64 + lane) * 4;
  const bool writes = c < a.width;
  const int n = (int)min((int64_t)4, a.width - c);
  const int64_t s = (int64_t)blockIdx.x * JOIN_WAVES + wave + 1, p = s * SUM_TOKENS;      // the run begins in stretch s - 1
  int64_t parts = 0;
  unsigned key = 0;
  if (s < a.stretches) {
    // the keys at this and the next 63 stretches' begins: how many of them are the run's
    const int64_t at = p + (int64_t)lane * SUM_TOKENS;
    const unsigned begin = at < a.tokens ? a.keys[at] : ~0u, last = a.keys[p - 1], before = s > 1 ? a.keys[p - SUM_TOKENS - 1] : ~0u;
    key = __builtin_amdgcn_readfirstlane(begin);
    if (key < a.vocab && last == key && before != key) {
      const int more = __popcll(__ballot(begin == key));
      parts = more < 64 ? more + 1 : (first_place(a, key + 1, p + 63 * SUM_TOKENS, a.tokens) - 1) / SUM_TOKENS - s + 2;
    }
  }
  const bool whole = parts > 0 && parts <= JOIN_ALONE;
  if (whole) {
    const float4 x = sum_parts<4>(a, s - 1, 0, parts, c);
    const float got[4] = {x.x, x.y, x.z, x.w};
    if (writes) write_sum<DT, 4>(a, key, c, 0, n, got);
  }
  if (lane == 0) long_runs[wave] = whole ? 0 : (int)parts;
  __syncthreads();
  for (int i = 0; i < JOIN_WAVES; i++) {
    const int64_t all = long_runs[i];
    if (!all) continue;
    const int64_t from = (int64_t)blockIdx.x * JOIN_WAVES + i, each = (all + JOIN_WAVES - 1) / JOIN_WAVES;
    part[wave][lane] = sum_parts<8>(a, from, min(wave * each, all), min(wave * each + each, all), c);
    __syncthreads();
    if (wave == 0 && writes) {
      float got[4] = {};
      for (int w = 0; w < JOIN_WAVES; w++) {
        const float4 y = part[w][lane];
        got[0] += y.x, got[1] += y.y, got[2] += y.z, got[3] += y.w;
      }
      write_sum<DT, 4>(a, a.keys[(from + 1) * SUM_TOKENS], c, 0, n, got);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
struct EmbedWork {
  size_t keys[2], places[2], counts, parts, bytes;
  int64_t stretches, part_width;
  SortArgs sort;
};

static size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

static bool embed_work(int64_t tokens, int64_t vocab, int64_t width, EmbedWork* w) {
  if (tokens < 0 || tokens > ((int64_t)1 << 26) || vocab < 1 || vocab >= INT32_MAX || width < 1 || width > (1 << 20)) return false;
  *w = EmbedWork{};
  size_t at = 0;
  for (int i = 0; i < 2; i++) {
    w->keys[i] = at, at += round256((size_t)tokens * 4);
    w->places[i] = at, at += round256((size_t)tokens * 4);
  }
  SortArgs& s = w->sort;
  s.tokens = tokens;
  s.vocab = vocab;
  if (tokens > RANK_TOKENS) {
    int need = 1;
    while (vocab >> need) need++;      // the key `vocab` itself is one
    s.passes = (need + SORT_BITS - 1) / SORT_BITS;
    s.bits = (need + s.passes - 1) / s.passes;
    s.blocks = (int)((tokens + SORT_BLOCK - 1) / SORT_BLOCK);
    s.scanned = s.blocks > 16;
    w->counts = at, at += round256((size_t)(s.blocks + 1) * SORT_BINS * 4);
  }
  w->stretches = (tokens + SUM_TOKENS - 1) / SUM_TOKENS;
  w->part_width = (width + 7) & ~(int64_t)7;
  w->parts = at, at += round256((size_t)w->stretches * 2 * w->part_width * 4);
  w->bytes = at;
  return true;
}

// The table's zeros are written beside the sort, which leaves the memory idle:
// 335 MB and the ranks of 8191 tokens in 44 to 58 us, of which the ranks alone take 14.
template <int DT>
static void launch_embedding_backward(SortArgs sort, const SumArgs& sum, hipStream_t s) {
  const int64_t vocab = sort.zero ? sort.vocab : 0;
  auto zeros = [&](int part, int parts) {      // the next share of the rows, and the workgroups for it
    sort.zero_from = vocab * part / parts;
    sort.zero_to = vocab * (part + 1) / parts;
    const int64_t vectors = (sort.zero_to - sort.zero_from) * units_of<DT>(sort.zero_width), want = (vectors + 8 * SORT_THREADS - 1) / (8 * SORT_THREADS);
    return (unsigned)(want > 1024 ? 1024 : want);
  };
  if (!sort.passes) {
    const unsigned blocks = (unsigned)((sort.tokens + 31) / 32) + zeros(0, 1);
    if (blocks) k_rank<DT><<<blocks, SORT_THREADS, (((size_t)sort.tokens + 127 & ~(size_t)127) + SORT_THREADS) * 4, s>>>(sort);
  } else
    for (int pass = 0; pass < sort.passes; pass++) {
      unsigned blocks = sort.blocks + zeros(2 * pass, 2 * sort.passes);
      k_sort_count<DT><<<blocks, SORT_THREADS, 0, s>>>(sort, pass);
      if (sort.scanned) k_sort_scan<<<SORT_BINS / 64, 64, 0, s>>>(sort);
      blocks = sort.blocks + zeros(2 * pass + 1, 2 * sort.passes);
      k_sort_place<DT><<<blocks, SORT_THREADS, 0, s>>>(sort, pass);
    }
  if (!sort.tokens) return;
  const unsigned units = units_of<DT>(sum.width), chunks = (units + 255) / 256;
  const unsigned block = ((units + chunks - 1) / chunks + 63) & ~63u;
  k_embedding_sum<DT><<<dim3((unsigned)sum.stretches, chunks), block, 0, s>>>(sum);
  if (sum.stretches > 1)
    k_embedding_join<DT><<<dim3((unsigned)((sum.stretches - 1 + JOIN_WAVES - 1) / JOIN_WAVES), (unsigned)((sum.width + 255) / 256)),
                           64 * JOIN_WAVES, 0, s>>>(sum);
}

}  // namespace externd

using namespace externd;

extern "C" {

int externd_embedding(const void* table, int32_t dtype, int64_t vocab, int64_t width, int64_t table_stride,
                      const int64_t* ids, int64_t tokens, float scale, void* out, int64_t out_stride, void* stream) {
  if (!dtype_ok(dtype) || vocab < 1 || width < 1 || tokens < 0 || table_stride < width || out_stride < width ||
      !std::isfinite(scale) || (tokens && (!table || !ids || !out)))
    return EXTERND_EINVAL;
  if (vocab > INT32_MAX || width > INT32_MAX || tokens > INT32_MAX) return EXTERND_EUNSUPPORTED;
  if (!tokens) return EXTERND_OK;
  const int64_t units = tokens * (dtype == EXTERND_F32 ? units_of<EXTERND_F32>(width) : units_of<EXTERND_F16>(width));
  const int64_t blocks = (units + 256 * EMBED_U - 1) / (256 * EMBED_U);
  if (blocks * 256 > MAX_THREADS) return EXTERND_EUNSUPPORTED;
  const EmbedArgs a = {table, out, ids, vocab, width, table_stride, out_stride, tokens, scale};
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) k_embedding<EXTERND_F32><<<(unsigned)blocks, 256, 0, s>>>(a);
  else if (dtype == EXTERND_BF16) k_embedding<EXTERND_BF16><<<(unsigned)blocks, 256, 0, s>>>(a);
  else k_embedding<EXTERND_F16><<<(unsigned)blocks, 256, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

size_t externd_embedding_backward_workspace_bytes(int64_t tokens, int64_t vocab, int64_t width) {
  EmbedWork w;
  return embed_work(tokens, vocab, width, &w) ? w.bytes : 0;
}

int externd_embedding_backward(const void* grad, int32_t dtype, int64_t tokens, int64_t width, int64_t grad_stride,
                               const int64_t* ids, int64_t vocab, float scale, int32_t accumulate, void* grad_table,
                               int64_t grad_table_stride, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dtype) || tokens < 0 || width < 1 || vocab < 1 || grad_stride < width || grad_table_stride < width ||
      !std::isfinite(scale) || (accumulate != 0 && accumulate != 1) || !grad_table || (tokens && (!grad || !ids)))
    return EXTERND_EINVAL;
  EmbedWork w;
  if (!embed_work(tokens, vocab, width, &w)) return EXTERND_EUNSUPPORTED;
  if (tokens && ((uintptr_t)workspace & 255)) return EXTERND_EINVAL;
  if (tokens && (!workspace || workspace_bytes < w.bytes)) return EXTERND_EWORKSPACE;
  if (!tokens && accumulate) return EXTERND_OK;
  char* const at = (char*)workspace;
  SortArgs sort = w.sort;
  sort.ids = ids;
  for (int i = 0; i < 2; i++) {
    sort.keys[i] = (unsigned*)(at + w.keys[i]);
    sort.places[i] = (unsigned*)(at + w.places[i]);
  }
  sort.counts = (unsigned*)(at + w.counts);
  sort.zero = accumulate ? nullptr : grad_table;
  sort.zero_width = width;
  sort.zero_stride = grad_table_stride;
  const int last = sort.passes ? (sort.passes - 1) & 1 : 0;
  const SumArgs sum = {grad, grad_table, tokens, width, grad_stride, grad_table_stride, vocab, w.stretches, sort.keys[last],
                       sort.places[last], (float*)(at + w.parts), w.part_width, scale, accumulate};
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) launch_embedding_backward<EXTERND_F32>(sort, sum, s);
  else if (dtype == EXTERND_BF16) launch_embedding_backward<EXTERND_BF16>(sort, sum, s);
  else launch_embedding_backward<EXTERND_F16>(sort, sum, s);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
