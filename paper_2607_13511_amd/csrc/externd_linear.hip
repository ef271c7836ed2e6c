// Log probabilities behind a dense head, and the gradients for its input and
// its matrix, without holding the logits.
#include <cmath>

#include "externd_gemm.hpp"

namespace externd {

constexpr int64_t FORWARD_ROWS = 8192;                // of a pass at most (pass_rows)
constexpr int64_t PIECE_ENTRIES = (int64_t)1 << 26;   // of G in a piece of the vocabulary, but eight tiles at least
constexpr int CUS = 256;

struct Part {
  float top, sum, mean, none;      // largest z, sum of e = exp(z - top), sum of e (z - top)
};

// What a row's gradient is made of: with l = log2 p (ln p for fp32), G = p (a l + b)
// and, at the target, g more.  All times `up`, a power of two that brings fp16's G below 2^15.
struct RowInfo {
  float a, b, g, lse, up;          // lse in the units of l; infinite where all p are 0
  int32_t y;                       // -1: no target
  int32_t present, none;
};

struct LinearArgs {
  Operand x, weight;
  int64_t rows, vocab, width;
  const int64_t* targets;
  float scale;
  int row_tiles, vocab_tiles;      // of this launch
  int grad_x_tiles;                // k_grads: before those of grad_weight
  int64_t step;                    // vocabulary of a tile
  int64_t v0, v1;                  // vocabulary of this launch
  // forward
  float *logprob, *entropy, *lse;
  Part* parts;                     // rows x all_parts
  int first_part, all_parts;
  // of 32 rows of fp32 or fewer: x cut into its parts, 3 x 32 x cut_width
  void* cut;
  int64_t cut_width;
  float* at_target;                // z of the target
  // backward
  const float *lse_in, *entropy_in, *g_logprob, *g_entropy;
  RowInfo* info;
  // G enters its products in the type of x and weight: in bf16 and fp16 that is six
  // times as fast as fp32 parts, and the roundings of p in its many entries average
  // out.  The target's entry, which g makes large in every row, does not: its rounding would
  // be in all of the row's grad_x, and of the target's grad_weight, alike.  What it has
  // lost is added to both (2048 rows of 65537, bf16: error of the gradients 2.38e-3 ->
  // 1.66e-3, which the rounding of the result alone makes; 1.3 % of the time).  An
  // entry that p makes large, where a row is sure of another token or of one under an
  // entropy's gradient, keeps its rounding: half a unit of the type, as the result has.
  int32_t* target;                 // of a row that takes part, or -1
  float* rest;
  // fp16: a row's x is packed times x_up / up, so that G^T x is x_up times too large.
  // x_up is the power of two that brings the largest of all rows to 2^14 .. 2^15; the
  // exponents that it follows from are left by ROW_BLOCKS workgroups or fewer.
  float* x_up;
  int32_t* row_exponents;
  int row_blocks;
  void *grad_x, *grad_weight;
  int64_t grad_x_stride, grad_weight_stride, p0, p1;      // this piece of the vocabulary, G's columns
  void *G, *packed;                // rows x G_width; rows x packed_width: x, zero where a row takes no part
  int64_t piece, G_width, packed_width;
  float* dx;                       // splits x rows x dx_width
  int64_t dx_width, split;         // k of a split
  int splits;
};

// Tiles in an order in which those that run together share operands: an XCD
// (workgroups go round robin over the eight) takes a stretch of them, eight
// row tiles of one vocabulary tile after another.
__device__ __forceinline__ void place_tile(int block, int rows, int others, int* row, int* other) {
  const int total = rows * others, xcd = block & 7, per = total >> 3, more = total & 7;
  const int at = xcd * per + min(xcd, more) + (block >> 3);
  const int panel = at / (8 * others), in = at - panel * 8 * others, w = min(8, rows - panel * 8);
  *row = panel * 8 + in % w;
  *other = in / w;
}

__device__ __forceinline__ float propagating_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// A tile on its way to memory: rows of n with BM entries of m, gathered in LDS so
// that whole lines are written (a lane holds four entries of each of its rows; at
// 8 bytes a store lines are written in parts, which with rows at some distances
// cost a fifth of k_logits).  Vectors of 16 bytes are exchanged within a row so
// that neither side meets in the banks.
template <typename P>
struct Gathered {
  typedef typename Elem<P::DT>::T T;
  static constexpr int E = Vec<P::DT>::E, VECTORS = P::BM / E;
  static_assert(P::BN * P::BM * (int)sizeof(T) <= P::LDS, "fits");
  static __device__ __forceinline__ char* at(char* lds, int n, int m) {
    return lds + (n * VECTORS + ((m / E) ^ (n & 31 & (VECTORS - 1)))) * 16 + m % E * (int)sizeof(T);
  }
  // Entries m .. m + 3 of row n.
  static __device__ __forceinline__ void put(char* lds, int n, int m, const float* o) {
    if constexpr (P::DT == EXTERND_F32) *(v4u*)at(lds, n, m) = Vec<P::DT>::pack(o);
    else {
      v2u b;
#pragma unroll
      for (int e = 0; e < 2; e++)
        b[e] = (unsigned)__builtin_bit_cast(uint16_t, Elem<P::DT>::store(o[2 * e])) |
               (unsigned)__builtin_bit_cast(uint16_t, Elem<P::DT>::store(o[2 * e + 1])) << 16;
      *(v2u*)at(lds, n, m) = b;
    }
  }
  // Calls store(n, m, vector) for the vectors of rows below n_count that begin below m_count; all threads.
  template <typename F>
  static __device__ __forceinline__ void write(char* lds, int64_t n_count, int64_t m_count, F store) {
    __syncthreads();
#pragma unroll 4
    for (int i = threadIdx.x; i < P::BN * VECTORS; i += GEMM_THREADS) {
      const int n = i / VECTORS, m = i % VECTORS * E;
      if (n < n_count && m < m_count) store(n, m, *(const v4u*)at(lds, n, m));
    }
  }
};

// e^x for x >= -200 with what the product x log2 e loses: p is within 2 u of itself and
// not within u |x|, which bounded fp32's gradients (517 rows of 8191: 2.8e-6 of them -> 1.9e-6).
__device__ __forceinline__ float exp_whole(float x) {
  const float y = x * LOG2E, rest = fmaf(x, 1.92596299112661746887e-8f, fmaf(x, LOG2E, -y));
  const float p = __builtin_amdgcn_exp2f(y);
  return fmaf(p * rest, LN2, p);
}

__device__ __forceinline__ float finite(float x) { return __builtin_isfinite(x) ? x : 0.f; }

// What x loses when it is stored (nothing, of what has become infinite).
template <int DT>
__device__ __forceinline__ float lost(float x) { return finite(x - Elem<DT>::load(Elem<DT>::store(x))); }

// Logits of a tile: rows of weight along m, rows of x along n, so that a lane
// holds one row's logits and its softmax needs no other lane but at the end.
// BACK: G of the tile; else its part of each row's softmax.
template <typename P, bool BACK>
__global__ __launch_bounds__(GEMM_THREADS, 2) void k_logits(LinearArgs a) {
  constexpr int DT = P::DT, TM = P::TM, TN = P::TN;
  __shared__ __align__(16) char lds[P::LDS];
  int rt, vt;
  place_tile((int)blockIdx.x, a.row_tiles, a.vocab_tiles, &rt, &vt);
  const int64_t m0 = a.v0 + vt * a.step, n0 = (int64_t)rt * P::BN, ms = min(a.step, a.v1 - m0);
  f32x16 acc[TM][TN];
  if constexpr (P::RAW) P::run(a.weight, m0, ms, Operand{a.cut, a.cut_width}, 0, P::BROWS, 0, a.width, (lds_char*)lds, acc);
  else P::run(a.weight, m0, ms, a.x, n0, a.rows - n0, 0, a.width, (lds_char*)lds, acc);
  if constexpr (BACK) {
    typedef typename Elem<DT>::T T;
    const float c = a.scale * LOG2E;
    if (P::holds())
#pragma unroll
    for (int j = 0; j < TN; j++) {
      const int64_t n = n0 + P::col(j);
      RowInfo w = {};
      w.y = -1;
      if (n < a.rows) w = a.info[n];
      if (ms < P::BM) {      // zeros behind the end: G's last vector is whole
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
          for (int r = 0; r < 16; r++)
            if (P::row(i, r) >= ms) acc[i][j][r] = -INFINITY;
      }
      if (__any(!w.present)) {
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
          for (int r = 0; r < 16; r++)
            if (!w.present) acc[i][j][r] = -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
          // p below 2^-200 is 0; the maximum passes a NaN on
          const float l = propagating_max(fmaf(acc[i][j][r], DT == EXTERND_F32 ? a.scale : c, -w.lse), -200.f);
          acc[i][j][r] = (DT == EXTERND_F32 ? exp_whole(l) : __builtin_amdgcn_exp2f(l)) * fmaf(w.a, l, w.b);
        }
      const int64_t y = w.y < 0 ? -1 : w.y - m0;
      if (__any(y >= P::row(0, 0) && y < P::row(0, 0) + TM * 32)) {      // a target among this wave's
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
          for (int r = 0; r < 16; r++)
            if (P::row(i, r) == y && y < ms) {
              acc[i][j][r] += w.g;
              if constexpr (DT != EXTERND_F32) a.rest[n] = lost<DT>(acc[i][j][r]);
            }
      }
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const float o[4] = {acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
          Gathered<P>::put(lds, P::col(j), P::row(i, r), o);
        }
    }
    T* const to = (T*)a.G + n0 * a.G_width + (m0 - a.p0);
    Gathered<P>::write(lds, a.rows - n0, ms, [&](int n, int m, v4u x) { *(v4u*)(to + n * a.G_width + m) = x; });
  } else {
    Part* const shared = (Part*)lds;      // WM x BN
    const float c = a.scale * LOG2E;
    if (P::holds())
#pragma unroll
    for (int j = 0; j < TN; j++) {
      const int64_t n = n0 + P::col(j), y = a.targets && n < a.rows ? a.targets[n] - m0 : -1;
      if (ms < P::BM) {
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
          for (int r = 0; r < 16; r++)
            if (P::row(i, r) >= ms) acc[i][j][r] = -INFINITY;
      }
      if (__any(y >= P::row(0, 0) && y < P::row(0, 0) + TM * 32)) {      // a target among this wave's
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
          for (int r = 0; r < 16; r++)
            if (P::row(i, r) == y && y < ms) a.at_target[n] = acc[i][j][r] * a.scale;      // what lies behind is another tile's
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int r = 0; r < 16; r++) top = fmaxf(top, acc[i][j][r]);
      top = fmaxf(top, __shfl_xor(top, 32));
      const float ref = fmaxf(top, -3.402823466e38f);
      float s[4] = {}, t[4] = {};
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
          // 2^-200 is 0; the maximum passes a NaN on
          const float d = propagating_max((acc[i][j][r] - ref) * c, -200.f), e = __builtin_amdgcn_exp2f(d);
          s[r & 3] += e;
          t[r & 3] = fmaf(e, d, t[r & 3]);
        }
      float sum = (s[0] + s[1]) + (s[2] + s[3]), mean = ((t[0] + t[1]) + (t[2] + t[3]));
      sum += __shfl_xor(sum, 32);
      mean += __shfl_xor(mean, 32);
      top *= a.scale;
      if (!(threadIdx.x & 32)) shared[P::wave() / P::WN * P::BN + P::col(j)] = Part{top, sum, mean * LN2, 0.f};
    }
    __syncthreads();
    const int n = threadIdx.x;
    if (n < P::BN && n0 + n < a.rows) {
      float top = -INFINITY, sum = 0.f, mean = 0.f;
      for (int w = 0; w < P::WM; w++) top = fmaxf(top, shared[w * P::BN + n].top);
      const float ref = fmaxf(top, -3.402823466e38f);
      for (int w = 0; w < P::WM; w++) {
        const Part p = shared[w * P::BN + n];
        const float d = fmaxf(p.top, -3.402823466e38f) - ref, f = __builtin_amdgcn_exp2f(d * LOG2E);
        if (p.sum == 0.f) continue;
        sum += p.sum * f;
        mean += f == 0.f ? 0.f : fmaf(p.sum, d, p.mean) * f;
      }
      a.parts[(n0 + n) * a.all_parts + a.first_part + vt] = Part{top, sum, mean, 0.f};
    }
  }
}

// A workgroup joins a row's parts.
__global__ __launch_bounds__(256) void k_logits_join(LinearArgs a) {
  __shared__ float lds[3][4];
  const int64_t r = blockIdx.x;
  const Part* p = a.parts + r * a.all_parts;
  float top = -3.402823466e38f, sum = 0.f, mean = 0.f;      // of this thread's parts, against the largest so far
  for (int i = threadIdx.x; i < a.all_parts; i += 256) {
    const Part q = p[i];
    if (q.sum == 0.f) continue;
    const float to = fmaxf(top, q.top), f = __builtin_amdgcn_exp2f((top - to) * LOG2E), d = fmaxf(q.top, -3.402823466e38f) - to,
                e = __builtin_amdgcn_exp2f(d * LOG2E);
    mean = (f == 0.f ? 0.f : fmaf(sum, top - to, mean) * f) + (e == 0.f ? 0.f : fmaf(q.sum, d, q.mean) * e);
    sum = sum * f + q.sum * e;
    top = to;
  }
  float all = top;
  for (int d = 32; d; d >>= 1) all = fmaxf(all, __shfl_xor(all, d));
  if ((threadIdx.x & 63) == 0) lds[0][threadIdx.x >> 6] = all;
  __syncthreads();
  all = fmaxf(fmaxf(lds[0][0], lds[0][1]), fmaxf(lds[0][2], lds[0][3]));
  const float d = top - all, f = __builtin_amdgcn_exp2f(d * LOG2E);
  mean = sum == 0.f || f == 0.f ? 0.f : fmaf(sum, d, mean) * f;
  sum = sum == 0.f ? 0.f : sum * f;
  for (int x = 32; x; x >>= 1) {
    sum += __shfl_xor(sum, x);
    mean += __shfl_xor(mean, x);
  }
  if ((threadIdx.x & 63) == 0) {
    lds[1][threadIdx.x >> 6] = sum;
    lds[2][threadIdx.x >> 6] = mean;
  }
  __syncthreads();
  if (threadIdx.x) return;
  sum = (lds[1][0] + lds[1][1]) + (lds[1][2] + lds[1][3]);
  mean = (lds[2][0] + lds[2][1]) + (lds[2][2] + lds[2][3]);
  const bool none = sum == 0.f;
  const float l = LN2 * log2f(sum), lse = none ? -INFINITY : all + l;
  if (a.lse) a.lse[r] = lse;
  if (a.entropy) a.entropy[r] = none ? 0.f : l - mean / sum;
  if (a.logprob) {
    const int64_t y = a.targets[r];
    a.logprob[r] = y < 0 ? 0.f : y >= a.vocab ? NAN : none ? -INFINITY : a.at_target[r] - lse;
  }
}

// What row r's gradient is made of.
__device__ __forceinline__ RowInfo row_info(const LinearArgs& a, int64_t r, bool fp16, bool fp32) {
  const int64_t y = a.targets ? a.targets[r] : -1;
  const bool asked = y >= 0 && y < a.vocab;
  RowInfo w = {};
  w.y = asked ? (int32_t)y : -1;
  const float g = a.g_logprob && asked ? a.g_logprob[r] : 0.f, ge = a.g_entropy ? a.g_entropy[r] : 0.f;
  const float h = ge == 0.f ? 0.f : a.entropy_in[r], lse = a.lse_in[r];
  w.present = g != 0.f || ge != 0.f;
  w.lse = !w.present || lse == -INFINITY ? INFINITY : fp32 ? lse : lse * LOG2E;
  w.up = 1.f;
  if (fp16 && w.present) {
    // |G| <= |g| + |ge| (p |ln p| + p H) < |g| + |ge| (1 + H)
    const float most = fabsf(g) + (ge == 0.f ? 0.f : fabsf(ge) * (1.f + fabsf(h)));
    const int k = most <= 3.402823466e38f ? 14 - ilogbf(most) : 0;
    w.up = ldexpf(1.f, k > 120 ? 120 : k < -120 ? -120 : k);
  }
  // -p (g + ge (ln p + H))
  w.g = g * w.up;
  w.a = -ge * w.up * (fp32 ? 1.f : LN2);
  w.b = -fmaf(ge, h, g) * w.up;
  return w;
}
__device__ __forceinline__ void put_row(const LinearArgs& a, int64_t r, const RowInfo& w) {
  a.info[r] = w;
  a.target[r] = w.present ? w.y : -1;
  a.rest[r] = 0.f;
}

// Of all rows, where k_pack does not do it.
__global__ __launch_bounds__(1024) void k_rows(LinearArgs a, int fp16, int fp32) {
  const int64_t r = (int64_t)blockIdx.x * 1024 + threadIdx.x;
  if (r < a.rows) put_row(a, r, row_info(a, r, fp16, fp32));
}

// The same before fp16's k_pack, a wave a row, which also looks for the largest
// finite entry of x: its exponent without that of `up`, the largest of a workgroup's rows.
constexpr int ROW_BLOCKS = 1024, NO_EXPONENT = -1000;
__global__ __launch_bounds__(256) void k_rows_of_x(LinearArgs a) {
  __shared__ int most[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int exponent = NO_EXPONENT;
  for (int64_t r = (int64_t)blockIdx.x * 4 + wave; r < a.rows; r += (int64_t)gridDim.x * 4) {
    const RowInfo w = row_info(a, r, true, false);
    if (lane == 0) put_row(a, r, w);
    if (!w.present) continue;
    const _Float16* x = (const _Float16*)a.x.p + r * a.x.stride;
    unsigned largest = 0;      // magnitudes order as whole numbers do
    auto look = [&](unsigned bits) { largest = max(largest, (bits & 0x7FFFu) < 0x7C00u ? bits & 0x7FFFu : 0u); };
    const int64_t whole = a.width & ~(int64_t)7;
#pragma unroll 4
    for (int64_t c = lane * 8; c < whole; c += 512) {
      const v4u v = load_any(x + c);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        look(v[i]);
        look(v[i] >> 16);
      }
    }
    if (whole + lane < a.width) look(__builtin_bit_cast(uint16_t, x[whole + lane]));
    for (int d = 32; d; d >>= 1) largest = max(largest, (unsigned)__shfl_xor((int)largest, d));
    if (largest) exponent = max(exponent, ilogbf((float)__builtin_bit_cast(_Float16, (uint16_t)largest)) - ilogbf(w.up));
  }
  if (lane == 0) most[wave] = exponent;
  __syncthreads();
  if (threadIdx.x == 0) a.row_exponents[blockIdx.x] = max(max(most[0], most[1]), max(most[2], most[3]));
}

// x for its product with G: rows that take no part are zeros whatever they hold.
// In fp16 G is up by a power of two for each row, and x is down by as much, all of it
// up by x_up: a product is exact but for entries that this takes below 2^-14, which
// are rounded by 2^-25, some 2^-39 of the largest.  (Down by the rows' own powers alone, with the
// largest row's x as it is, 2^-25 of x: of rows 2^10 below the largest no more than seven bits
// were left of small entries, and none of rows 2^24 below it.)  In the other types a row's
// first thread also writes what k_rows would, a launch less (58 fp32 rows of 3607: 41 -> 39.5 us).
template <int DT>
__global__ __launch_bounds__(256) void k_pack(LinearArgs a) {
  typedef typename Elem<DT>::T T;
  constexpr int E = Vec<DT>::E;
  int up = 0;
  if constexpr (DT == EXTERND_F16) {
    __shared__ int most[4];
    int exponent = NO_EXPONENT;
    for (int i = threadIdx.x; i < a.row_blocks; i += 256) exponent = max(exponent, a.row_exponents[i]);
    for (int d = 32; d; d >>= 1) exponent = max(exponent, __shfl_xor(exponent, d));
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = exponent;
    __syncthreads();
    // at least 14 - (15 + 120); at most so that its reciprocal is a normal number
    up = min(14 - max(max(most[0], most[1]), max(most[2], most[3])), 126);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.x_up = ldexpf(1.f, up);
  }
  const int64_t units = a.packed_width / E, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= units * a.rows) return;
  const int64_t r = i / units, c = (i - r * units) * E;
  const RowInfo w = DT == EXTERND_F16 ? a.info[r] : row_info(a, r, false, DT == EXTERND_F32);
  if (DT != EXTERND_F16 && c == 0) {
    put_row(a, r, w);
    if (r == 0) *a.x_up = 1.f;
  }
  const T* from = (const T*)a.x.p + r * a.x.stride + c;
  float x[E] = {};
  if (w.present) {
    if (c + E <= a.width) Vec<DT>::unpack(load_any(from), x);
    else
      for (int e = 0; e < E; e++) x[e] = c + e < a.width ? Elem<DT>::load(from[e]) : 0.f;
    if constexpr (DT == EXTERND_F16) {
      const int d = up - ilogbf(w.up);
#pragma unroll
      for (int e = 0; e < E; e++) x[e] = ldexpf(x[e], d);
    }
  }
  *(v4u*)((T*)a.packed + r * a.packed_width + c) = Vec<DT>::pack(x);
}

// At most 32 rows of x cut into their parts, with zeros behind rows and columns.
__global__ __launch_bounds__(256) void k_cut(LinearArgs a) {
  const int64_t units = a.cut_width / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= 32 * units) return;
  const int64_t r = i / units, c = (i - r * units) * 8;
  const float* x = (const float*)a.x.p + r * a.x.stride + c;
  v4u held[2], part[3];
#pragma unroll
  for (int e = 0; e < 8; e++) held[e / 4][e % 4] = r < a.rows && c + e < a.width ? __float_as_uint(x[e]) : 0u;
  cut(held, part);
#pragma unroll
  for (int p = 0; p < 3; p++) *(v4u*)((uint16_t*)a.cut + (p * 32 + r) * a.cut_width + c) = part[p];
}

// G weight of this piece (columns of weight along m, rows of G along n), added to
// the split's sums so far.
template <typename P>
__device__ __forceinline__ void grad_x_tile(const LinearArgs& a, int block, char* lds) {
  const int cols = (int)((a.width + P::BM - 1) / P::BM);
  int rt, other;
  place_tile(block, a.row_tiles, cols * a.splits, &rt, &other);
  const int s = other / cols;
  const int64_t m0 = (int64_t)(other - s * cols) * P::BM, n0 = (int64_t)rt * P::BN, k0 = s * a.split, K = min(a.split, a.p1 - a.p0 - k0);
  f32x16 acc[P::TM][P::TN];
  const Operand G = {a.G, a.G_width};
  P::run(a.weight, m0, a.width - m0, G, n0, a.rows - n0, a.p0 + k0, K > 0 ? K : 0, (lds_char*)lds, acc, -a.p0);
#pragma unroll
  for (int j = 0; j < P::TN; j++) {
    const int64_t n = n0 + P::col(j);
    if (n >= a.rows) continue;
    float* const to = a.dx + (s * a.rows + n) * a.dx_width + m0;
#pragma unroll
    for (int i = 0; i < P::TM; i++)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int c = P::row(i, r);
        if (m0 + c >= a.dx_width) continue;
        float4 x = {acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
        if (a.p0) {
          const float4 b = *(const float4*)(to + c);
          x = float4{x.x + b.x, x.y + b.y, x.z + b.z, x.w + b.w};
        }
        *(float4*)(to + c) = x;
      }
  }
}

// The splits' sums joined in order, scaled and rounded.  A thread has four
// columns; GROUPS of them share many splits (few rows, whose loads would otherwise
// wait for each other) and are joined in LDS.
template <int DT, int GROUPS>
__global__ __launch_bounds__(256) void k_grad_x_join(LinearArgs a) {
  typedef typename Elem<DT>::T T;
  constexpr int UNITS = 256 / GROUPS;
  __shared__ float4 part[GROUPS][UNITS];
  const int64_t units = a.dx_width / 4, i = (int64_t)blockIdx.x * UNITS + threadIdx.x % UNITS;
  const int group = threadIdx.x / UNITS;
  const bool in = i < units * a.rows;
  const int64_t r = in ? i / units : 0, c = in ? (i - r * units) * 4 : 0;
  const RowInfo w = a.info[r];
  float x[4] = {};
  if (in && w.present) {
    const int each = (a.splits + GROUPS - 1) / GROUPS, s1 = min((group + 1) * each, a.splits);
    const float* p = a.dx + r * a.dx_width + c;
#pragma unroll 8
    for (int s = group * each; s < s1; s++) {
      const float4 b = *(const float4*)(p + s * a.rows * a.dx_width);
      x[0] += b.x, x[1] += b.y, x[2] += b.z, x[3] += b.w;
    }
  }
  if constexpr (GROUPS > 1) {
    part[group][threadIdx.x % UNITS] = float4{x[0], x[1], x[2], x[3]};
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int g = 1; g < GROUPS; g++) {
      const float4 b = part[g][threadIdx.x];
      x[0] += b.x, x[1] += b.y, x[2] += b.z, x[3] += b.w;
    }
  }
  if (!in) return;
  if (DT != EXTERND_F32 && a.target[r] >= 0) {
    const float rest = a.rest[r];
    const T* y = (const T*)a.weight.p + a.target[r] * a.weight.stride + c;
#pragma unroll
    for (int e = 0; e < 4; e++)
      if (c + e < a.width) x[e] += finite(rest * Elem<DT>::load(y[e]));
  }
  const float f = a.scale, down = 1.f / w.up;
  T* const to = (T*)a.grad_x + r * a.grad_x_stride + c;
#pragma unroll
  for (int e = 0; e < 4; e++)
    if (c + e < a.width) to[e] = Elem<DT>::store(x[e] * f * down);
}

// Adds what the targets' entries of G have lost, for the rows whose target is one of
// this tile's columns: steps of up to 64 such rows, of their rows of x and of a tile
// with one entry for each.  All threads, none of which reads `lds` before.
template <typename P>
__device__ __forceinline__ void add_rests(const LinearArgs& a, f32x16 (*acc)[P::TN], int64_t m0, int64_t n0, char* lds) {
  typedef typename Elem<P::DT>::T T;
  constexpr int WAVES = GEMM_THREADS / 64, U = 4, ROWS = U * GEMM_THREADS;
  static_assert(P::BK == 64 && P::STAGES >= 2 && P::STAGE >= 4 * (ROWS + U * WAVES), "the list is in the second stage");
  int* const list = (int*)(lds + P::STAGE);
  int* const counts = list + ROWS;
  char* const b = lds + P::TA::BYTES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t first = a.v0 + n0;
  const int last = (int)min((int64_t)P::BN, a.v1 - first);
  for (int64_t r0 = 0; r0 < a.rows; r0 += ROWS) {
    uint64_t mine[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int64_t r = r0 + u * GEMM_THREADS + threadIdx.x;
      const int64_t c = (r < a.rows ? a.target[r] : -1) - first;
      mine[u] = __ballot(c >= 0 && c < last);
      if (lane == 0) counts[u * WAVES + wave] = __popcll(mine[u]);
    }
    __syncthreads();
    int have = 0;
#pragma unroll
    for (int u = 0; u < U; u++)
      for (int w = 0; w < WAVES; w++) {
        if (w == wave && (mine[u] >> lane & 1)) list[have + __popcll(mine[u] & ((1ull << lane) - 1))] = (int)(r0 + u * GEMM_THREADS + threadIdx.x);
        have += counts[u * WAVES + w];
      }
    __syncthreads();
    for (int from = 0; from < have; from += 64) {
      const int n = min(64, have - from);
#pragma unroll 1
      for (int i = threadIdx.x; i < P::TA::VECTORS; i += GEMM_THREADS) {
        int k, v;
        P::TA::place(i, &k, &v);
        v4u x = {0, 0, 0, 0};
        if (k < n && m0 + v * 8 < a.packed_width) x = *(const v4u*)((const T*)a.packed + list[from + k] * a.packed_width + m0 + v * 8);
        *(v4u*)(lds + i * 16) = x;
      }
#pragma unroll 1
      for (int i = threadIdx.x; i < P::TB::VECTORS; i += GEMM_THREADS) *(v4u*)(b + i * 16) = v4u{0, 0, 0, 0};
      __syncthreads();
      if ((int)threadIdx.x < n) {
        const int k = threadIdx.x, r = list[from + k], c = (int)(a.target[r] - first);
        *(T*)(b + (k * P::TB::CH + ((c >> 4 ^ P::TB::spread(k)) << 1 | (c >> 3 & 1))) * 16 + (c & 7) * 2) = Elem<P::DT>::store(a.rest[r]);
      }
      __syncthreads();
      P::step((const lds_char*)lds, acc);
      __syncthreads();
    }
  }
}

// G^T x of this piece: columns of x along m, of G (the vocabulary) along n.
template <typename P>
__device__ __forceinline__ void grad_weight_tile(const LinearArgs& a, int block, char* lds) {
  typedef typename Elem<P::DT>::T T;
  int ct, vt;
  place_tile(block, (int)((a.width + P::BM - 1) / P::BM), a.vocab_tiles, &ct, &vt);
  const int64_t m0 = (int64_t)ct * P::BM, n0 = (int64_t)vt * P::BN, ns = a.v1 - a.v0;
  f32x16 acc[P::TM][P::TN];
  const Operand x = {a.packed, a.packed_width}, G = {(T*)a.G + (a.v0 - a.p0), a.G_width};
  P::run(x, m0, a.packed_width - m0, G, n0, (ns - n0 + 7) & ~(int64_t)7, 0, a.rows, (lds_char*)lds, acc);      // whole vectors: G's rows have room
  if constexpr (P::DT != EXTERND_F32) add_rests<P>(a, acc, m0, n0, lds);
  const float f = a.scale, down = 1.f / *a.x_up;
#pragma unroll
  for (int j = 0; j < P::TN; j++)
#pragma unroll
    for (int i = 0; i < P::TM; i++)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] = acc[i][j][r + e] * f * down;
        Gathered<P>::put(lds, P::col(j), P::row(i, r), o);
      }
  T* const to = (T*)a.grad_weight + (a.v0 + n0) * a.grad_weight_stride + m0;
  const int64_t width = a.width - m0;
  Gathered<P>::write(lds, ns - n0, width, [&](int n, int m, v4u x) {
    T* const at = to + n * a.grad_weight_stride + m;
    if (m + Vec<P::DT>::E <= width) store_any(at, x);
    else {
      float y[Vec<P::DT>::E];
      Vec<P::DT>::unpack(x, y);
#pragma unroll
      for (int e = 0; e < Vec<P::DT>::E; e++)
        if (m + e < width) at[e] = Elem<P::DT>::store(y[e]);      // exact: of its type
    }
  });
}

template <typename P>
__global__ __launch_bounds__(GEMM_THREADS, 2) void k_grad_x(LinearArgs a) {
  __shared__ __align__(16) char lds[P::LDS];
  grad_x_tile<P>(a, (int)blockIdx.x, lds);
}
template <typename P>
__global__ __launch_bounds__(GEMM_THREADS, 2) void k_grad_weight(LinearArgs a) {
  __shared__ __align__(16) char lds[P::LDS];
  grad_weight_tile<P>(a, (int)blockIdx.x, lds);
}
// Both, where the CUs hold the tiles of both at once.
template <typename X, typename W>
__global__ __launch_bounds__(GEMM_THREADS, 2) void k_grads(LinearArgs a) {
  __shared__ __align__(16) char lds[X::LDS > W::LDS ? X::LDS : W::LDS];
  if ((int)blockIdx.x < a.grad_x_tiles) grad_x_tile<X>(a, (int)blockIdx.x, lds);
  else grad_weight_tile<W>(a, (int)blockIdx.x - a.grad_x_tiles, lds);
}

// grad_weight without rows.
template <int DT>
__global__ __launch_bounds__(256) void k_zero_rows(LinearArgs a) {
  typedef typename Elem<DT>::T T;
  for (int64_t r = blockIdx.x; r < a.vocab; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < a.width; c += 256) ((T*)a.grad_weight)[r * a.grad_weight_stride + c] = T(0);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of a launch, of 512 threads each, and vectors of x are counted in 32 bits.
static bool linear_sizes(int64_t rows, int64_t vocab, int64_t width) {
  return rows <= (1 << 22) && vocab <= (1 << 25) && width <= (1 << 20) && rows * width <= (int64_t)1 << 33 && vocab * width <= (int64_t)1 << 37;
}

// Rows of a tile, as sizes are planned.  16-bit operands that go through registers have tiles of 128 rows
// where this says 256 (which would not leave enough of them): twice the tiles that the plan counts, and
// with a step of 128 columns half of each tile of 256 lies behind its end, masked.
static int tile_rows(int32_t dtype, int64_t rows) {
  if (rows <= 32) return 32;
  return dtype == EXTERND_F32 || rows <= 128 ? 128 : 256;
}

// Few large tiles leave CUs without work: small ones then, 64 columns by 32
// rows, whose eight waves share the k of a step.  A large tile takes as long as
// about four small ones (121 fp32 rows of 2556, width 4026: 316 -> 46 us).
static bool small_tiles(int32_t dtype, int64_t rows, int64_t vocab) {
  const int64_t small = ceil_div(vocab, 64) * ceil_div(rows, 32);
  return ceil_div(vocab, 256) * ceil_div(rows, tile_rows(dtype, rows)) < CUS && small <= CUS * (rows <= 32 ? 1 : 4);
}

// Rows of a pass of the forward call, so that the parts stay small and the tiles of
// a launch, of 128 rows at the least here, have fewer than 2^32 threads.
static int64_t pass_rows(int64_t rows, int64_t vocab) {
  int64_t most = FORWARD_ROWS;
  while (most / 128 * ceil_div(vocab, 256) * GEMM_THREADS > MAX_THREADS) most /= 2;
  return rows < most ? rows : most;
}

// Vocabulary of a tile of logits: 64 for small tiles; 128 where tiles of 256 are
// so few that half as large ones still take one round (452 fp32 rows of 7232, 116
// tiles or 228: the gradients take 630 -> 546 us); else 256.  One row tile of the
// forward call reads weight once, so there the card's CUs take equally many tiles of
// equal length: 65537 columns are 512 tiles of 136 and not 256 of 256 and one of 1.
static int64_t tile_step(int32_t dtype, int64_t rows, int64_t vocab, bool back) {
  if (small_tiles(dtype, rows, vocab)) return 64;
  const int64_t n = tile_rows(dtype, rows);
  if (n >= 128 && 2 * ceil_div(vocab, 256) * ceil_div(rows, n) <= CUS && (dtype == EXTERND_F32 || n == 256)) return 128;
  if (back || rows > n || vocab <= 256 * CUS / 8) return 256;
  const int64_t tiles = ceil_div(ceil_div(vocab, 256), CUS) * CUS;
  return ceil_div(ceil_div(vocab, tiles), 8) * 8;
}

struct LinearWork {
  size_t cut, parts, at_target, info, target, rest, x_up, row_exponents, packed, G, dx, bytes;
  int64_t tiles, step, piece, G_width, packed_width, dx_width, cut_width, split;
  int splits;
};

// Room for the parts of x; its width is whole vectors of 8.
static size_t cut_bytes(int32_t dtype, int64_t rows, int64_t width, LinearWork* w) {
  w->cut_width = ceil_div(width, 8) * 8;
  return dtype == EXTERND_F32 && rows <= 32 ? round256((size_t)(3 * 32 * w->cut_width) * 2) : 0;
}

static LinearWork forward_work(int32_t dtype, int64_t rows, int64_t vocab, int64_t width) {
  LinearWork w = {};
  const int64_t r = pass_rows(rows, vocab);
  w.step = tile_step(dtype, r, vocab, false);
  w.tiles = ceil_div(vocab, w.step);
  w.parts = cut_bytes(dtype, r, width, &w);
  w.at_target = w.parts + round256((size_t)(r * w.tiles) * sizeof(Part));
  w.bytes = w.at_target + round256((size_t)r * 4);
  return w;
}

// Vocabulary of a piece, of which the last takes up to 255 more: G of a piece
// stays below PIECE_ENTRIES or is eight tiles of 256, whichever is more (2^22 rows: 2048
// columns and the rest, 19 GB of bf16), and among such pieces the one is taken whose tiles leave the fewest rounds of the CUs partly empty (a round of
// logits costs width, one of grad_weight rows).  2048 rows, 65537 x 2560: two of 32768,
// 4 and 5 whole rounds, where three equal ones are 3 and 4 each: 2127 -> 2070 us.
static int64_t choose_piece(int64_t rows, int64_t vocab, int64_t width, int64_t row_tiles, int64_t weight_tiles) {
  const int64_t tiles = vocab / 256, most = PIECE_ENTRIES / rows / 256, least = ceil_div(tiles, most < 8 ? 8 : most);
  if (tiles <= 1) return 256;
  int64_t best = 0, best_cost = 0;
  for (int64_t pieces = least; pieces <= least + 4 && pieces <= tiles; pieces++) {
    const int64_t each = ceil_div(tiles, pieces), last = tiles - (ceil_div(tiles, each) - 1) * each;
    auto cost = [&](int64_t n) { return ceil_div(n * row_tiles, CUS) * width + ceil_div(n * weight_tiles, CUS) * rows; };
    const int64_t all = (ceil_div(tiles, each) - 1) * cost(each) + cost(last);
    if (!best || all < best_cost) {
      best = each;
      best_cost = all;
    }
  }
  return best * 256;
}

static LinearWork backward_work(int32_t dtype, int64_t rows, int64_t vocab, int64_t width, bool need_x, bool need_weight) {
  LinearWork w = {};
  const int64_t row_tiles = ceil_div(rows, tile_rows(dtype, rows)), cols = ceil_div(width, 256);
  w.piece = choose_piece(rows, vocab, width, row_tiles, need_weight ? cols * (dtype == EXTERND_F32 ? 2 : 1) : 0);
  // rows an odd number of 512 bytes apart: at a power of two they share the caches' sets (4095 rows 16384 entries apart: 738 us for 607)
  w.G_width = (ceil_div(vocab < w.piece + 256 ? vocab : w.piece + 256, 256) | 1) * 256;
  const int vec = 16 / dtype_bytes(dtype);
  w.packed_width = ceil_div(width, vec) * vec;
  w.dx_width = ceil_div(width, 4) * 4;
  int64_t splits = CUS / (cols * row_tiles);
  const int64_t max_splits = ceil_div(w.G_width, 128);
  splits = splits < 1 ? 1 : splits > max_splits ? max_splits : splits;
  // fewer, if grad_weight's tiles then run beside them and not after: the longer of both sums for one after the other
  const int64_t weight_tiles = cols * ceil_div(vocab < w.piece + 255 ? vocab : w.piece + 255, dtype == EXTERND_F32 ? 128 : 256);
  const int64_t beside = (CUS - weight_tiles) / (cols * row_tiles), sum = beside > 0 ? ceil_div(w.G_width, beside) : 0;
  if (need_x && need_weight && beside > 0 && beside < splits && (sum > rows ? sum : rows) < rows + ceil_div(w.G_width, splits)) splits = beside;
  w.split = ceil_div(ceil_div(w.G_width, splits), 64) * 64;
  w.splits = (int)ceil_div(w.G_width, w.split);
  size_t at = cut_bytes(dtype, rows, width, &w);
  w.info = at, at += round256((size_t)rows * sizeof(RowInfo));
  w.target = at, at += round256((size_t)rows * 4);
  w.rest = at, at += round256((size_t)rows * 4);
  w.x_up = at, at += 256;
  w.row_exponents = at, at += dtype == EXTERND_F16 && need_weight ? ROW_BLOCKS * 4 : 0;
  w.packed = at, at += need_weight ? round256((size_t)(rows * w.packed_width) * dtype_bytes(dtype)) : 0;
  w.G = at, at += round256((size_t)(rows * w.G_width) * dtype_bytes(dtype));
  w.dx = at, at += need_x ? round256((size_t)(w.splits * rows * w.dx_width) * 4) : 0;
  w.bytes = at;
  return w;
}

// Whether rows are whole vectors of 16 bytes at multiples of 16.
static bool direct_rows(const Operand& o, int64_t width, int32_t dtype) {
  const int vec = 16 / dtype_bytes(dtype);
  return !((uintptr_t)o.p & 15) && o.stride % vec == 0 && width % vec == 0;
}

template <typename P, bool BACK>
static void launch_logits(LinearArgs a, hipStream_t s) {
  a.row_tiles = (int)ceil_div(a.rows, P::BN);
  a.vocab_tiles = (int)ceil_div(a.v1 - a.v0, a.step);
  k_logits<P, BACK><<<(unsigned)(a.row_tiles * a.vocab_tiles), GEMM_THREADS, 0, s>>>(a);
}

// Calls `large` for a launch's vocabulary, or for its tiles of 256 and then
// `small` for the last few columns, where those alone would begin one more round of
// the CUs: a small tile waits for memory as often as a large one, and takes 70 us of a
// round's 85 (2048 rows, 65537 columns); in tiles of 32 rows it takes 25
// (of grad_weight 21 for 70; both together 2081 -> 2032 us).
template <typename L, typename S>
static void with_tail(LinearArgs a, int64_t other_tiles, L large, S small) {
  const int64_t tiles = (a.v1 - a.v0) / 256, rest = (a.v1 - a.v0) % 256;
  if (a.step != 256 || !tiles || !rest || ceil_div((tiles + 1) * other_tiles, CUS) == ceil_div(tiles * other_tiles, CUS)) return large(a);
  LinearArgs b = a;
  a.v1 = b.v0 = a.v0 + tiles * 256;
  b.first_part += (int)tiles;
  large(a);
  small(b);
}

template <typename P>
static void launch_grad_weight(LinearArgs a, hipStream_t s) {
  a.vocab_tiles = (int)ceil_div(a.v1 - a.v0, P::BN);
  k_grad_weight<P><<<(unsigned)(ceil_div(a.width, P::BM) * a.vocab_tiles), GEMM_THREADS, 0, s>>>(a);
}

template <int DT, bool DIRECT, bool BACK>
static void choose_logits(const LinearArgs& a, hipStream_t s) {
  const int n = tile_rows(DT, a.rows);
  if (a.step == 64) return launch_logits<Product<DT, DIRECT && DT != EXTERND_F32, false, false, 64, 32, 1, DIRECT && DT != EXTERND_F32 ? 3 : 2, 8>, BACK>(a, s);
  if constexpr (DT == EXTERND_F32) {
    // small tiles leave room for more of them on their way: 8 rows of 65537, tiles of 136, 166 -> 155 us
    if (DIRECT && !BACK && n == 32 && a.step <= 160) launch_logits<Product<DT, true, false, false, 256, 32, 8, 6, 1, 160>, false>(a, s);
    else if (n == 32) launch_logits<Product<DT, DIRECT, false, false, 256, 32, 8, DIRECT ? 4 : 2>, BACK>(a, s);
    else if (a.step == 128) launch_logits<Product<DT, false, false, false, 128, 128, 2, 2>, BACK>(a, s);
    else launch_logits<Product<DT, false, false, false, 256, 128, 4, 2>, BACK>(a, s);
  } else {
    typedef Product<DT, DIRECT, false, false, 256, 32, 8, DIRECT ? 4 : 2> Small;
    if (n == 32) launch_logits<Small, BACK>(a, s);
    else if (n == 128 || !DIRECT) launch_logits<Product<DT, DIRECT, false, false, 256, 128, 4, DIRECT ? 3 : 2>, BACK>(a, s);
    else if (a.step == 128) launch_logits<Product<DT, true, false, false, 128, 256, 2, 3>, BACK>(a, s);
    else if constexpr (DIRECT)
      with_tail(a, ceil_div(a.rows, 256), [&](const LinearArgs& b) { launch_logits<Product<DT, true, false, false, 256, 256, 2, 2>, BACK>(b, s); },
                [&](const LinearArgs& b) { launch_logits<Small, BACK>(b, s); });
  }
}
// grad_x of this piece, and grad_weight in the same launch if the tiles of both are no
// more than CUs (58 fp32 rows of 3607, width 521: 52 -> 41 us; 1000 bf16 rows of 5000,
// width 1024, of which fewer splits make room: 104 -> 83).  Returns whether it was.
template <typename X, typename W>
static bool launch_grad_x(LinearArgs a, hipStream_t s) {
  a.row_tiles = (int)ceil_div(a.rows, X::BN);
  const int64_t cols = ceil_div(a.width, X::BM), tiles = a.row_tiles * cols * a.splits;
  a.vocab_tiles = (int)ceil_div(a.v1 - a.v0, W::BN);
  const bool both = a.grad_weight && tiles + ceil_div(a.width, W::BM) * a.vocab_tiles <= CUS;
  if (both) {
    a.grad_x_tiles = (int)tiles;
    k_grads<X, W><<<(unsigned)(tiles + ceil_div(a.width, W::BM) * a.vocab_tiles), GEMM_THREADS, 0, s>>>(a);
  } else k_grad_x<X><<<(unsigned)tiles, GEMM_THREADS, 0, s>>>(a);
  return both;
}
template <int DT, bool DIRECT, typename W>
static bool choose_grad_x(const LinearArgs& a, hipStream_t s) {
  const int n = tile_rows(DT, a.rows);
  if constexpr (DT == EXTERND_F32) {
    if (n == 32) return launch_grad_x<Product<DT, false, true, false, 256, 32, 8, 2>, W>(a, s);
    return launch_grad_x<Product<DT, false, true, false, 256, 128, 4, 2>, W>(a, s);
  } else {
    if (n == 32) return launch_grad_x<Product<DT, DIRECT, true, false, 256, 32, 8, DIRECT ? 4 : 2>, W>(a, s);
    if constexpr (DIRECT)
      if (n == 256) return launch_grad_x<Product<DT, true, true, false, 256, 256, 2, 2>, W>(a, s);
    return launch_grad_x<Product<DT, DIRECT, true, false, 256, 128, 4, DIRECT ? 3 : 2>, W>(a, s);
  }
}

template <int DT>
static void launch_cut(const LinearArgs& a, hipStream_t s) {
  if (DT == EXTERND_F32 && a.step != 64 && tile_rows(DT, a.rows) == 32) k_cut<<<(unsigned)ceil_div(32 * (a.cut_width / 8), 256), 256, 0, s>>>(a);
}

template <int DT>
static void launch_forward(LinearArgs a, bool direct, hipStream_t s) {
  if (direct && (DT != EXTERND_F32 || a.cut || tile_rows(DT, a.rows) > 32)) {
    launch_cut<DT>(a, s);
    choose_logits<DT, true, false>(a, s);
  } else choose_logits<DT, false, false>(a, s);
  k_logits_join<<<(unsigned)a.rows, 256, 0, s>>>(a);
}

template <int DT>
static void launch_backward(LinearArgs a, bool direct, hipStream_t s) {
  if (!a.rows) {
    k_zero_rows<DT><<<(unsigned)(a.vocab < 4096 ? a.vocab : 4096), 256, 0, s>>>(a);
    return;
  }
  if (!a.grad_weight) k_rows<<<(unsigned)ceil_div(a.rows, 1024), 1024, 0, s>>>(a, DT == EXTERND_F16, DT == EXTERND_F32);
  else if (DT == EXTERND_F16) k_rows_of_x<<<a.row_blocks, 256, 0, s>>>(a);
  if (direct) launch_cut<DT>(a, s);
  if (a.grad_weight) k_pack<DT><<<(unsigned)ceil_div(a.rows * (a.packed_width / Vec<DT>::E), 256), 256, 0, s>>>(a);
  for (a.p0 = 0; a.p0 < a.vocab; a.p0 = a.p1) {
    a.p1 = a.p0 + a.piece + 256 > a.vocab ? a.vocab : a.p0 + a.piece;
    a.v0 = a.p0;
    a.v1 = a.p1;
    if (direct) choose_logits<DT, true, true>(a, s);
    else choose_logits<DT, false, true>(a, s);
    typedef std::conditional_t<DT == EXTERND_F32, Product<DT, false, true, true, 256, 128, 4, 2>, Product<DT, DT != EXTERND_F32, true, true, 256, 256, 2, 2>> W;
    bool both = false;
    if (a.grad_x) both = DT != EXTERND_F32 && direct ? choose_grad_x<DT, DT != EXTERND_F32, W>(a, s) : choose_grad_x<DT, false, W>(a, s);
    if (a.grad_weight && !both) {
      if constexpr (DT == EXTERND_F32) launch_grad_weight<W>(a, s);
      else
        with_tail(a, ceil_div(a.width, 256), [&](const LinearArgs& b) { launch_grad_weight<W>(b, s); },
                  [&](const LinearArgs& b) { launch_grad_weight<Product<DT, true, true, true, 256, 32, 8, 4>>(b, s); });
    }
  }
  if (a.grad_x) {
    const int64_t units = a.rows * (a.dx_width / 4);
    if (a.splits >= 8) k_grad_x_join<DT, 8><<<(unsigned)ceil_div(units, 32), 256, 0, s>>>(a);
    else k_grad_x_join<DT, 1><<<(unsigned)ceil_div(units, 256), 256, 0, s>>>(a);
  }
}

}  // namespace externd

using namespace externd;

extern "C" {

size_t externd_linear_logprobs_workspace_bytes(int32_t dtype, int64_t rows, int64_t vocab, int64_t width) {
  if (!dtype_ok(dtype) || rows < 0 || vocab < 1 || width < 1 || !linear_sizes(rows, vocab, width)) return 0;
  return forward_work(dtype, rows ? rows : 1, vocab, width).bytes;
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
  const LinearWork w = forward_work(dtype, rows, vocab, width);
  if (!workspace || workspace_bytes < w.bytes) return EXTERND_EWORKSPACE;
  const hipStream_t s = (hipStream_t)stream;
  const int64_t pass = pass_rows(rows, vocab);
  for (int64_t r = 0; r < rows; r += pass) {
    LinearArgs a = {};
    a.x = {(const char*)x + r * x_stride * dtype_bytes(dtype), x_stride};
    a.weight = {weight, weight_stride};
    a.rows = rows - r < pass ? rows - r : pass;
    a.vocab = a.v1 = vocab;
    a.all_parts = (int)w.tiles;
    a.width = width;
    a.targets = logprob ? targets + r : nullptr;
    a.scale = scale;
    a.logprob = logprob ? logprob + r : nullptr;
    a.entropy = entropy ? entropy + r : nullptr;
    a.lse = lse ? lse + r : nullptr;
    a.cut = w.parts ? workspace : nullptr;      // there only if all rows are few, not if those of the last pass are
    a.cut_width = w.cut_width;
    a.parts = (Part*)((char*)workspace + w.parts);
    a.at_target = (float*)((char*)workspace + w.at_target);
    a.step = w.step;
    const bool direct = direct_rows(a.x, width, dtype) && direct_rows(a.weight, width, dtype);
    if (dtype == EXTERND_F32) launch_forward<EXTERND_F32>(a, direct, s);
    else if (dtype == EXTERND_BF16) launch_forward<EXTERND_BF16>(a, direct, s);
    else launch_forward<EXTERND_F16>(a, direct, s);
  }
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

size_t externd_linear_logprobs_backward_workspace_bytes(int32_t dtype, int64_t rows, int64_t vocab, int64_t width,
                                                        int32_t need_x, int32_t need_weight) {
  if (!dtype_ok(dtype) || rows < 0 || vocab < 1 || width < 1 || !linear_sizes(rows, vocab, width)) return 0;
  return backward_work(dtype, rows ? rows : 1, vocab, width, need_x, need_weight).bytes;
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
  const LinearWork w = backward_work(dtype, rows ? rows : 1, vocab, width, grad_x, grad_weight);
  if (!workspace || workspace_bytes < w.bytes) return EXTERND_EWORKSPACE;
  LinearArgs a = {};
  a.x = {x, x_stride};
  a.weight = {weight, weight_stride};
  a.rows = rows;
  a.vocab = vocab;
  a.width = width;
  a.targets = targets;
  a.scale = scale;
  a.step = tile_step(dtype, rows, vocab, true);
  a.lse_in = lse;
  a.entropy_in = entropy;
  a.g_logprob = g_logprob;
  a.g_entropy = g_entropy;
  a.grad_x = grad_x;
  a.grad_weight = grad_weight;
  a.grad_x_stride = grad_x_stride;
  a.grad_weight_stride = grad_weight_stride;
  char* const at = (char*)workspace;
  a.cut = at;
  a.cut_width = w.cut_width;
  a.info = (RowInfo*)(at + w.info);
  a.target = (int32_t*)(at + w.target);
  a.rest = (float*)(at + w.rest);
  a.x_up = (float*)(at + w.x_up);
  a.row_exponents = (int32_t*)(at + w.row_exponents);
  a.row_blocks = (int)(rows < 4 * ROW_BLOCKS ? ceil_div(rows, 4) : ROW_BLOCKS);
  a.packed = at + w.packed;
  a.G = at + w.G;
  a.dx = (float*)(at + w.dx);
  a.piece = w.piece;
  a.G_width = w.G_width;
  a.packed_width = w.packed_width;
  a.dx_width = w.dx_width;
  a.split = w.split;
  a.splits = w.splits;
  const bool direct = direct_rows(a.x, width, dtype) && direct_rows(a.weight, width, dtype);
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) launch_backward<EXTERND_F32>(a, direct, s);
  else if (dtype == EXTERND_BF16) launch_backward<EXTERND_BF16>(a, direct, s);
  else launch_backward<EXTERND_F16>(a, direct, s);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
