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
constexpr int SORT_WAVES = 16, SORT_BITS = 9, SORT_BINS = 1 << SORT_BITS;
constexpr int64_t SORT_BLOCK = 16384;       // tokens of one workgroup; more of them only past 256 workgroups
constexpr int SORT_MOST_BLOCKS = 256;

struct SortArgs {
  const int64_t* ids;
  int64_t tokens, vocab, per_block, per_wave;
  int blocks, passes, bits;                 // bits of a pass's digit
  unsigned *keys[2], *places[2];            // sorted so far: the id (vocab where there is none) and the token
  unsigned* counts;                         // blocks x bins of the present pass
  // what becomes zero meanwhile
  void* zero;
  int64_t zero_rows, zero_width, zero_stride;
};

__device__ __forceinline__ unsigned sort_key(const SortArgs& a, int pass, int64_t i) {
  if (pass) return a.keys[(pass - 1) & 1][i];
  const int64_t id = a.ids[i];
  return (unsigned)(id >= 0 && id < a.vocab ? id : a.vocab);
}

struct SortShared {
  unsigned at[SORT_WAVES][SORT_BINS];       // of each wave: how many of a digit, then where its next one goes
  unsigned sums[SORT_WAVES];
};

// One stable pass over this workgroup's tokens: each wave takes a stretch in
// order.  Places follow from counts alone, so they do not depend on what runs first.
__device__ void sort_pass(const SortArgs& a, int pass, int block, SortShared& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << a.bits, shift = pass * a.bits;
  const int64_t b0 = (int64_t)block * a.per_block, b1 = min(b0 + a.per_block, a.tokens);
  const int64_t w0 = min(b0 + wave * a.per_wave, b1), w1 = min(w0 + a.per_wave, b1);
  for (int i = threadIdx.x; i < SORT_WAVES * SORT_BINS; i += blockDim.x) ((unsigned*)s.at)[i] = 0;
  __syncthreads();
  for (int64_t i = w0 + lane; i < w1; i += 64) atomicAdd(&s.at[wave][sort_key(a, pass, i) >> shift & (bins - 1)], 1u);
  __syncthreads();
  unsigned total = 0, before = 0;
  const int bin = threadIdx.x;
  if (bin < bins) {
    for (int w = 0; w < SORT_WAVES; w++) {
      const unsigned n = s.at[w][bin];
      s.at[w][bin] = total;
      total += n;
    }
    if (a.blocks > 1) {
      total = 0;
      for (int b = 0; b < a.blocks; b++) {
        const unsigned n = a.counts[(int64_t)b * bins + bin];
        if (b < block) before += n;
        total += n;
      }
    }
  }
  unsigned upto = total;                    // sum over the digits up to this one
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 63) s.sums[wave] = upto;
  __syncthreads();
  unsigned first = upto - total + before;
  for (int w = 0; w < wave; w++) first += s.sums[w];
  if (bin < bins)
    for (int w = 0; w < SORT_WAVES; w++) s.at[w][bin] += first;
  __syncthreads();
  unsigned* const keys = a.keys[pass & 1];
  unsigned* const places = a.places[pass & 1];
  for (int64_t i0 = w0; i0 < w1; i0 += 64) {
    const bool in = i0 + lane < w1;
    const unsigned key = in ? sort_key(a, pass, i0 + lane) : 0;
    const unsigned place = !in ? 0 : pass ? a.places[(pass - 1) & 1][i0 + lane] : (unsigned)(i0 + lane);
    const unsigned digit = key >> shift & (bins - 1);
    uint64_t same = __ballot(in);
    for (int b = 0; b < a.bits; b++) {
      const uint64_t m = __ballot(digit >> b & 1);
      same &= digit >> b & 1 ? m : ~m;
    }
    const unsigned rank = __popcll(same & ((1ull << lane) - 1));
    const unsigned to = s.at[wave][digit] + rank;
    __builtin_amdgcn_wave_barrier();        // all have read before the next place is written
    if (in) {
      keys[to] = key;
      places[to] = place;
      if (rank == 0) s.at[wave][digit] = to + __popcll(same);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Rows of zeros, by the workgroups behind the sorting ones.
template <int DT>
__device__ void zero_rows(const SortArgs& a, int64_t block, int64_t blocks) {
  typedef typename Elem<DT>::T T;
  constexpr int E = Vec<DT>::E;
  if (a.zero_stride == a.zero_width) {
    const int64_t n = a.zero_rows * a.zero_width, lead = min((int64_t)((16 - ((uintptr_t)a.zero & 15)) & 15) / (int64_t)sizeof(T), n);
    T* const z = (T*)a.zero;
    const int64_t nv = (n - lead) / E;
    for (int64_t i = block * blockDim.x + threadIdx.x; i < nv; i += blocks * blockDim.x) ((v4u*)(z + lead))[i] = v4u{0, 0, 0, 0};
    if (block == 0) {
      if ((int64_t)threadIdx.x < lead) z[threadIdx.x] = T(0);
      if (threadIdx.x < n - lead - nv * E) z[lead + nv * E + threadIdx.x] = T(0);
    }
    return;
  }
  for (int64_t r = block; r < a.zero_rows; r += blocks) {
    T* const z = (T*)a.zero + r * a.zero_stride;
    for (int64_t c = (int64_t)threadIdx.x * E; c < a.zero_width; c += (int64_t)blockDim.x * E) {
      if (c + E <= a.zero_width) store_any<T>(z + c, v4u{0, 0, 0, 0});
      else
        for (int64_t e = c; e < a.zero_width; e++) z[e] = T(0);
    }
  }
}

// All passes by one workgroup.
template <int DT>
__global__ __launch_bounds__(64 * SORT_WAVES) void k_sort_one(SortArgs a) {
  __shared__ SortShared s;
  if (blockIdx.x >= (unsigned)a.blocks) return zero_rows<DT>(a, blockIdx.x - a.blocks, gridDim.x - a.blocks);
  for (int pass = 0; pass < a.passes; pass++) {
    sort_pass(a, pass, 0, s);
    __threadfence_block();
    __syncthreads();
  }
}

template <int DT>
__global__ __launch_bounds__(64 * SORT_WAVES) void k_sort_count(SortArgs a, int pass) {
  __shared__ unsigned n[SORT_BINS];
  if (blockIdx.x >= (unsigned)a.blocks) return zero_rows<DT>(a, blockIdx.x - a.blocks, gridDim.x - a.blocks);
  const int bins = 1 << a.bits, shift = pass * a.bits;
  for (int i = threadIdx.x; i < bins; i += blockDim.x) n[i] = 0;
  __syncthreads();
  const int64_t b0 = (int64_t)blockIdx.x * a.per_block, b1 = min(b0 + a.per_block, a.tokens);
  for (int64_t i = b0 + threadIdx.x; i < b1; i += blockDim.x) atomicAdd(&n[sort_key(a, pass, i) >> shift & (bins - 1)], 1u);
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += blockDim.x) a.counts[(int64_t)blockIdx.x * bins + i] = n[i];
}

__global__ __launch_bounds__(64 * SORT_WAVES) void k_sort_place(SortArgs a, int pass) {
  __shared__ SortShared s;
  sort_pass(a, pass, blockIdx.x, s);
}

// ---------------------------------------------------------------------------
// sums of the tokens of an id
// ---------------------------------------------------------------------------
constexpr int SUM_TOKENS = 16;      // places of a stretch, in the sorted order
constexpr int JOIN_WAVES = 8, JOIN_BOUNDS = 8;

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

// Entries c .. c + n - 1 of a row's gradient, n <= N.
template <int DT, int N>
__device__ __forceinline__ void write_sum(const SumArgs& a, unsigned key, int64_t c, int n, const float* sum) {
  typedef typename Elem<DT>::T T;
  T* const to = (T*)a.table + (int64_t)key * a.table_stride + c;
  if (n == N && N == Vec<DT>::E) {
    float x[N];
    if (a.accumulate) Vec<DT>::unpack(load_any<T>(to), x);
#pragma unroll
    for (int e = 0; e < N; e++) x[e] = a.accumulate ? fmaf(sum[e], a.scale, x[e]) : sum[e] * a.scale;
    store_any<T>(to, Vec<DT>::pack(x));
  } else
    for (int e = 0; e < N; e++)
      if (e < n) to[e] = Elem<DT>::store(a.accumulate ? fmaf(sum[e], a.scale, Elem<DT>::load(to[e])) : sum[e] * a.scale);
}

// A workgroup sums a stretch of sorted places over a part of the width, a
// vector of 16 bytes a thread; eight rows are loaded ahead of their sums.  Runs
// that lie in the stretch are finished here, the others leave a part.
template <int DT>
__global__ __launch_bounds__(256) void k_embedding_sum(SumArgs a) {
  typedef typename Elem<DT>::T T;
  constexpr int E = Vec<DT>::E, B = 8;
  const int64_t s = blockIdx.x, p0 = s * SUM_TOKENS;
  const int count = (int)min((int64_t)SUM_TOKENS, a.tokens - p0);
  const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * E;
  if (c >= a.width) return;
  const int n = (int)min((int64_t)E, a.width - c);
  const unsigned before = p0 ? a.keys[p0 - 1] : ~0u, after = p0 + count < a.tokens ? a.keys[p0 + count] : ~0u;
  float sum[E] = {};
  bool begun = a.keys[p0] == before;      // the present run began before this stretch
#pragma unroll
  for (int b = 0; b < SUM_TOKENS; b += B) {
    float x[B][E];
#pragma unroll
    for (int i = 0; i < B; i++) {
      const int64_t p = p0 + b + i;
      if (b + i < count && a.keys[p] < a.vocab) {
        const T* from = (const T*)a.grad + (int64_t)a.places[p] * a.grad_stride + c;
        if (n == E) Vec<DT>::unpack(load_any<T>(from), x[i]);
        else
          for (int e = 0; e < E; e++) x[i][e] = e < n ? Elem<DT>::load(from[e]) : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < B; i++) {
      if (b + i >= count) return;
      const unsigned key = a.keys[p0 + b + i], next = b + i + 1 < count ? a.keys[p0 + b + i + 1] : after;
      if (key >= a.vocab) return;
#pragma unroll
      for (int e = 0; e < E; e++) sum[e] += x[i][e];
      const bool last = b + i + 1 == count;
      if (next == key && !last) continue;
      if (begun || next == key) {
        float* to = a.parts + (2 * s + (begun ? 0 : 1)) * a.part_width + c;
#pragma unroll
        for (int e = 0; e < E; e++) to[e] = sum[e];
      } else
        write_sum<DT, E>(a, key, c, n, sum);
#pragma unroll
      for (int e = 0; e < E; e++) sum[e] = 0.f;
      begun = false;
    }
  }
}

// The runs that cross a stretch's end: each is joined where it crosses its first
// one.  A workgroup looks at JOIN_BOUNDS ends and takes 256 columns; its waves take
// equal stretches of a run's parts and are joined in order.
template <int DT>
__global__ __launch_bounds__(64 * JOIN_WAVES) void k_embedding_join(SumArgs a) {
  __shared__ float4 part[JOIN_WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = ((int64_t)blockIdx.y * 64 + lane) * 4;
  for (int i = 0; i < JOIN_BOUNDS; i++) {
    const int64_t s = (int64_t)blockIdx.x * JOIN_BOUNDS + i + 1;      // the run begins in stretch s - 1
    if (s >= a.stretches) return;
    const int64_t p = s * SUM_TOKENS;
    const unsigned key = a.keys[p];
    if (key >= a.vocab) return;
    if (a.keys[p - 1] != key || (s > 1 && a.keys[p - SUM_TOKENS - 1] == key)) continue;
    int64_t lo = p, hi = a.tokens;                                    // the run's end: first place after p with another key
    while (hi - lo > 1) {
      const int64_t mid = (lo + hi) >> 1;
      if (a.keys[mid] == key) lo = mid;
      else hi = mid;
    }
    const int64_t parts = lo / SUM_TOKENS - s + 2;                    // of stretches s - 1 .. that of the last place
    const int64_t each = (parts + JOIN_WAVES - 1) / JOIN_WAVES, q0 = min(wave * each, parts), q1 = min(q0 + each, parts);
    float4 sum = {0.f, 0.f, 0.f, 0.f};
    if (c < a.width) {
#pragma unroll 4
      for (int64_t q = q0; q < q1; q++) {
        const float4 x = *(const float4*)(a.parts + (2 * (s - 1 + q) + (q ? 0 : 1)) * a.part_width + c);
        sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
      }
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < a.width) {
      for (int w = 1; w < JOIN_WAVES; w++) {
        const float4 x = part[w][lane];
        sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
      }
      const float got[4] = {sum.x, sum.y, sum.z, sum.w};
      write_sum<DT, 4>(a, key, c, (int)min((int64_t)4, a.width - c), got);
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
  int need = 1;
  while (vocab >> need) need++;      // the key `vocab` itself is one
  s.passes = (need + SORT_BITS - 1) / SORT_BITS;
  s.bits = (need + s.passes - 1) / s.passes;
  s.per_block = SORT_BLOCK;
  if (tokens > SORT_BLOCK * SORT_MOST_BLOCKS) s.per_block = ((tokens + SORT_MOST_BLOCKS - 1) / SORT_MOST_BLOCKS + 1023) & ~(int64_t)1023;
  s.blocks = tokens ? (int)((tokens + s.per_block - 1) / s.per_block) : 1;
  const int64_t most = s.blocks > 1 ? s.per_block : tokens;
  s.per_wave = ((most + SORT_WAVES - 1) / SORT_WAVES + 63) & ~(int64_t)63;
  w->counts = at, at += s.blocks > 1 ? round256((size_t)s.blocks * SORT_BINS * 4) : 0;
  w->stretches = (tokens + SUM_TOKENS - 1) / SUM_TOKENS;
  w->part_width = (width + 7) & ~(int64_t)7;
  w->parts = at, at += round256((size_t)w->stretches * 2 * w->part_width * 4);
  w->bytes = at;
  return true;
}

template <int DT>
static void launch_embedding_backward(const SortArgs& sort, const SumArgs& sum, hipStream_t s) {
  int zeros = 0;
  if (sort.zero_rows) {      // workgroups of 16 waves with 16 vectors a thread or more
    const int64_t want = (sort.zero_rows * units_of<DT>(sort.zero_width) + 16383) / 16384;
    zeros = (int)(want < 1 ? 1 : want > 1024 ? 1024 : want);
  }
  const int threads = 64 * SORT_WAVES;
  if (sort.blocks == 1) k_sort_one<DT><<<1 + zeros, threads, 0, s>>>(sort);
  else
    for (int pass = 0; pass < sort.passes; pass++) {
      k_sort_count<DT><<<sort.blocks + (pass ? 0 : zeros), threads, 0, s>>>(sort, pass);
      k_sort_place<<<sort.blocks, threads, 0, s>>>(sort, pass);
    }
  if (!sum.tokens) return;
  const unsigned units = units_of<DT>(sum.width), chunks = (units + 255) / 256;
  const unsigned block = ((units + chunks - 1) / chunks + 63) & ~63u;
  k_embedding_sum<DT><<<dim3((unsigned)sum.stretches, chunks), block, 0, s>>>(sum);
  if (sum.stretches > 1)
    k_embedding_join<DT><<<dim3((unsigned)((sum.stretches - 1 + JOIN_BOUNDS - 1) / JOIN_BOUNDS), (unsigned)((sum.width + 255) / 256)),
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
  sort.zero = grad_table;
  sort.zero_rows = accumulate ? 0 : vocab;
  sort.zero_width = width;
  sort.zero_stride = grad_table_stride;
  const int last = (sort.passes - 1) & 1;
  const SumArgs sum = {grad, grad_table, tokens, width, grad_stride, grad_table_stride, vocab, w.stretches, sort.keys[last],
                       sort.places[last], (float*)(at + w.parts), w.part_width, scale, accumulate};
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) launch_embedding_backward<EXTERND_F32>(sort, sum, s);
  else if (dtype == EXTERND_BF16) launch_embedding_backward<EXTERND_BF16>(sort, sum, s);
  else launch_embedding_backward<EXTERND_F16>(sort, sum, s);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
