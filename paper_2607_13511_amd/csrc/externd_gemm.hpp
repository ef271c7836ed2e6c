// Matrix products on the matrix cores for the operators behind a dense head:
// C(m, n) = sum over k of A(m, k) B(n, k) by tiles of a workgroup.
//
// Either operand lies in memory as rows of k ("by rows") or as rows of m or n,
// one for each k ("by columns"); both reach the same fragments, eight
// consecutive k of one m in a lane, the latter through LDS reads that transpose
// 4 x 16 entries.  A tile's LDS holds vectors of 16 bytes in an order that keeps
// the reads of a fragment apart in the banks; as loads write LDS in lane order,
// each lane picks its vector of global memory accordingly.
#pragma once

#include <type_traits>

#include "externd_decode.hpp"

namespace externd {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int GEMM_THREADS = 512;

// An operand of a product: `count` of m (or n) and K of k, with rows `stride` entries apart.
struct Operand {
  const void* p;
  int64_t stride;
};

// What a product of type DT takes: fp32 operands become three bf16 parts of 8
// bits each, x = x1 + x2 + x3 exactly (cut, not rounded), of which the six
// products not below 2^-24 are summed.
template <int DT> struct Kind {
  static constexpr int PLANES = DT == EXTERND_F32 ? 3 : 1;
  static constexpr int BK = DT == EXTERND_F32 ? 32 : 64;      // k of a step
};

template <int DT>
__device__ __forceinline__ f32x16 mfma(v4u a, v4u b, f32x16 c) {
  if constexpr (DT == EXTERND_F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The LDS tile of one operand: X of m (or n) by BK of k, EV entries in 16 bytes.
template <bool COL, int X, int BK, int EV = 8>
struct Tile {
  static constexpr int VECTORS = X * BK / EV;                 // of 16 bytes, in each plane
  static constexpr int BYTES = VECTORS * 16;
  static constexpr int LOADS = VECTORS / GEMM_THREADS;        // of a thread
  static_assert(VECTORS % GEMM_THREADS == 0 || VECTORS < GEMM_THREADS, "whole loads");
  static constexpr int CH = COL ? X / EV : BK / EV;            // vectors of a row in memory
  // Where in the operand the vector at place `i` of the tile is: its row in memory and its vector there.
  static __host__ __device__ __forceinline__ void place(int i, int* row, int* vec) {
    *row = i / CH;
    const int v = i % CH;
    if constexpr (COL) *vec = ((v >> 1) ^ spread(*row)) << 1 | (v & 1);
    else *vec = v ^ swap(*row);
  }
  // By rows: the sixteen rows that are read together go to different banks (256 bytes of them).
  static __host__ __device__ __forceinline__ int swap(int row) { return CH >= 16 ? row & 15 : (row / (16 / (CH < 16 ? CH : 16))) & (CH - 1); }
  // By columns: pairs of vectors (16 columns) of four rows of k go to different banks.
  static __host__ __device__ __forceinline__ int spread(int k) { return (2 * (k & 3)) & (X / 16 - 1); }
  // The byte at which a lane reads its fragment of 32 columns from x0 on, without what depends on x0 and on the step of 16 k.
  static __device__ __forceinline__ v4u fragment(const lds_char* t, int x0, int ks) {
    const int lane = threadIdx.x & 63;
    if constexpr (COL) {
      const int k = ks * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2), q = (x0 >> 4) + ((lane >> 4) & 1);
      const lds_char* at = t + k * (X * 2) + ((q ^ spread(k)) << 5) + (lane & 3) * 8;
      typedef __attribute__((address_space(3))) s16x4* four;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((four)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((four)(at + 4 * (X * 2)));
      const v2u a = __builtin_bit_cast(v2u, lo), b = __builtin_bit_cast(v2u, hi);
      return v4u{a[0], a[1], b[0], b[1]};
    } else {
      const int row = x0 + (lane & 31), v = (ks * 2 + (lane >> 5)) ^ swap(row);
      return *(const __attribute__((address_space(3))) v4u*)(t + (row * CH + v) * 16);
    }
  }
  // The same of a tile of fp32 entries by rows: the fragment's eight in two vectors.
  static __device__ __forceinline__ void fragment_f32(const lds_char* t, int x0, int ks, v4u* x) {
    const int lane = threadIdx.x & 63, row = x0 + (lane & 31);
#pragma unroll
    for (int i = 0; i < 2; i++)
      x[i] = *(const __attribute__((address_space(3))) v4u*)(t + (row * CH + ((ks * 4 + (lane >> 5) * 2 + i) ^ swap(row))) * 16);
  }
};

// Eight fp32 entries as three vectors of bf16: x = x1 + x2 + x3 exactly, 8 bits each,
// cut and not rounded.  An infinity or a NaN becomes NaN in one of them.
__device__ __forceinline__ void cut(const v4u* x, v4u* part) {
#pragma unroll
  for (int w = 0; w < 4; w++) {
    unsigned p[3][2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const unsigned v = x[w >> 1][(w & 1) * 2 + h], y = v & 0xFFFF0000u;
      const float r = __uint_as_float(v) - __uint_as_float(y);
      const unsigned z = __float_as_uint(r) & 0xFFFF0000u;
      p[0][h] = y;
      p[1][h] = z;
      p[2][h] = __float_as_uint(r - __uint_as_float(z));
    }
#pragma unroll
    for (int i = 0; i < 3; i++) part[i][w] = __builtin_amdgcn_perm(p[i][1], p[i][0], 0x07060302u);      // the upper halves
  }
}

// The six products of two operands' parts that are not below 2^-24.  The smaller
// five are summed by themselves first: c would round each of them at its own size
// (8 rows of 65537: the error of lse is 1.2e-8 to 1.0e-7 of itself, and 7e-8 to
// 2.4e-7 with all six summed into c; 5 % of the time).  Few rows hold the smaller
// ones' sum over all of K beside c (2.5e-8 to 7.5e-8); many have no registers for it.
__device__ __forceinline__ f32x16 mfma_cut(const v4u* a, const v4u* b, f32x16 c) {
  f32x16 small = {};
  small = mfma<EXTERND_BF16>(a[1], b[1], small);
  small = mfma<EXTERND_BF16>(a[0], b[2], small);
  small = mfma<EXTERND_BF16>(a[2], b[0], small);
  small = mfma<EXTERND_BF16>(a[0], b[1], small);
  small = mfma<EXTERND_BF16>(a[1], b[0], small);
  c = mfma<EXTERND_BF16>(a[0], b[0], c);
#pragma unroll
  for (int r = 0; r < 16; r++) c[r] += small[r];
  return c;
}

// Loads of operands whose rows begin at multiples of 16 bytes and are whole
// vectors, straight into LDS.  (Part of a vector would come as zeros where the operand
// ends.  K is rounded up to whole vectors by rows: zeros in memory.)  The buffer's base moves on with the
// steps, and what lies past its end becomes zeros.  HELD: rows that are loaded at all.
template <bool COL, int X, int BK, int EV = 8, int HELD = X>
struct Direct {
  typedef Tile<COL, X, BK, EV> T;
  static constexpr int B = 16 / EV;                           // bytes of an entry
  static constexpr int VECTORS = COL ? T::VECTORS : HELD * T::CH;
  static constexpr int LOADS = (VECTORS + GEMM_THREADS - 1) / GEMM_THREADS;      // of a wave, or one less
  static_assert(VECTORS % 64 == 0, "a wave has all of a load or none");
  static constexpr unsigned NONE = 0xFFFFFFFFu;
  const char* base;
  int64_t left, k_left;      // bytes from the base to the operand's end; k's from the next step on
  int64_t step;              // bytes: 64 rows of 2^24 entries of G (a piece of few rows) are past 31 bits
  unsigned offset[LOADS];

  // count of m (or n) from x0 on, K of k from k0 on.
  __host__ __device__ __forceinline__ void init(const Operand& o, int64_t x0, int64_t count, int64_t k0, int64_t K, int thread) {
    const int64_t row = o.stride * B, cols = count < X ? count : X;
    if (!COL) K = (K + EV - 1) & ~(int64_t)(EV - 1);
    const int64_t rows = COL ? K : cols, width = (COL ? cols : K) * B;
    base = (const char*)o.p + (COL ? k0 * row + x0 * B : x0 * row + k0 * B);
    left = rows > 0 ? (rows - 1) * row + width : 0;
    k_left = K;
    step = COL ? BK * row : BK * B;
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      int r, v;
      T::place(i * GEMM_THREADS + thread, &r, &v);
      const bool in = i * GEMM_THREADS + thread < VECTORS && (COL ? v * 16 < width : r < rows);
      offset[i] = in ? (unsigned)(r * row + v * 16) : NONE;
    }
  }
  // Bytes behind the base that are the operand's, as the buffer's size.
  __host__ __device__ __forceinline__ unsigned room() const { return left <= 0 ? 0u : left < (int64_t)0xFFFFFFF0 ? (unsigned)left : 0xFFFFFFF0u; }
  __host__ __device__ __forceinline__ void next() {
    base += step;
    left -= step;
    k_left -= BK;
  }
  static __device__ __forceinline__ bool has(int i) {      // whether this wave has a load i
    return (i + 1) * GEMM_THREADS <= VECTORS || i * GEMM_THREADS + (int)(threadIdx.x & ~63u) < VECTORS;
  }
  // The vectors of the next step, to the tile at `lds`.
  __device__ __forceinline__ void issue(lds_char* lds) {
    const unsigned to = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)lds + (threadIdx.x >> 6) * 1024);
    const i32x4 resource = {__builtin_amdgcn_readfirstlane((int)(uintptr_t)base), __builtin_amdgcn_readfirstlane((int)((uintptr_t)base >> 32)),
                            __builtin_amdgcn_readfirstlane((int)room()), 0x00020000};
    if (COL || k_left >= BK) {
#pragma unroll
      for (int i = 0; i < LOADS; i++)
        if (has(i)) load(to + i * (GEMM_THREADS * 16), offset[i], resource);
    } else {                 // by rows, the last step: the next row's entries are none of this one's
#pragma unroll
      for (int i = 0; i < LOADS; i++) {
        int r, v;
        T::place(i * GEMM_THREADS + (int)threadIdx.x, &r, &v);
        if (has(i)) load(to + i * (GEMM_THREADS * 16), v * EV < k_left ? offset[i] : NONE, resource);
      }
    }
    next();
  }
  // LDS is written behind the compiler's back: whoever reads it waits for it (wait_loads).
  static __device__ __forceinline__ void load(unsigned to, unsigned from, i32x4 resource) {
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(from), "s"(resource) : "memory");
  }
};

// At most N of this wave's loads are under way, and its LDS reads are done.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Moves the eight entries of a vector down by s, 0 .. 7, with zeros behind.
template <int DT, int WORDS>
__device__ __forceinline__ void shift_down(v4u* x, int s) {
  unsigned w[4 * WORDS + 4] = {};
#pragma unroll
  for (int i = 0; i < 4 * WORDS; i++) w[i] = x[i / 4][i % 4];
  const int words = DT == EXTERND_F32 ? s : s >> 1;
#pragma unroll
  for (int d = 4; d; d >>= 1)
#pragma unroll
    for (int i = 0; i < 4 * WORDS; i++) w[i] = words & d ? (i + d < 4 * WORDS ? w[i + d] : 0u) : w[i];
  if (DT != EXTERND_F32 && (s & 1)) {
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = w[i] >> 16 | w[i + 1] << 16;
  }
#pragma unroll
  for (int i = 0; i < 4 * WORDS; i++) x[i / 4][i % 4] = w[i];
}

// Loads of any operand through registers: rows that begin anywhere and end within
// a vector, and fp32 operands, cut into their parts.  DEPTH steps are under way at
// a time, and no load stands behind a branch that waits: a vector that is only
// partly there is read so that it ends where its row does, and moved into place
// on its way to LDS.
template <int DT, bool COL, int X, int BK, int DEPTH>
struct Staged {
  typedef typename Elem<DT>::T E;
  typedef Tile<COL, X, BK> T;
  static constexpr int LOADS = T::LOADS ? T::LOADS : 1, WORDS = DT == EXTERND_F32 ? 2 : 1;
  const E *at[LOADS], *safe, *begin;      // safe: eight entries that are there; begin: of the step, for put_tiny
  v4u held[DEPTH][LOADS][WORDS];
  int64_t stride, k_left;
  int cols, over, tail;         // of m (or n); by columns, entries that the last vector lacks; k of the last step, if fewer than BK
  bool tiny;                    // rows of fewer than eight entries: put_tiny

  __device__ __forceinline__ bool none(int i) const { return i * GEMM_THREADS + (int)threadIdx.x >= T::VECTORS; }
  __device__ __forceinline__ bool short_column(int v) const { return v * 8 < cols && cols < v * 8 + 8; }

  __device__ __forceinline__ void init(const Operand& o, int64_t x0, int64_t count, int64_t k0, int64_t K) {
    stride = o.stride;
    cols = (int)min(count, (int64_t)X);
    over = COL && cols & 7 ? 8 - (cols & 7) : 0;
    tail = (int)(K % BK);
    k_left = K;
    tiny = (COL ? x0 + cols : k0 + K) < 8;
    const E* base = (const E*)o.p + (COL ? k0 * stride + x0 : x0 * stride + k0);
    begin = base;
    safe = (const E*)o.p + (COL ? k0 * stride + x0 + cols - 8 : x0 * stride);
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      int r, v;
      T::place(i * GEMM_THREADS + (int)threadIdx.x, &r, &v);
      // past the last m (or n) any entries do, as what becomes of them is not used: the first ones
      if (COL ? v * 8 >= cols : r >= cols) COL ? v = 0 : r = 0;
      at[i] = base + r * stride + v * 8 - (!tiny && COL && short_column(v) ? over : 0);
    }
  }
  // The next step's vectors, into set `set`.  It always loads, so that waits can count the loads behind their own.
  __device__ __forceinline__ void fetch(int set) {
    const int n = (int)max((int64_t)0, min(k_left, (int64_t)BK));
    k_left -= BK;
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const E* from = at[i];
      if (n < BK) {      // the last step, or none: in the place of what is not there, entries that are
        int r, v;
        T::place(i * GEMM_THREADS + (int)threadIdx.x, &r, &v);
        if (n == 0) from = safe;
        else if (COL) from -= r < n ? 0 : r * stride;
        else from -= n - v * 8 >= 8 ? 0 : v * 8 + 8 - n;
      }
#pragma unroll
      for (int w = 0; w < WORDS; w++) held[set][i][w] = load_any(from + w * Vec<DT>::E);
      at[i] += COL ? BK * stride : BK;
    }
  }
  static __device__ __forceinline__ void write(lds_char* to, int plane, const v4u* x) {
    typedef __attribute__((address_space(3))) v4u* vec;
    if constexpr (DT != EXTERND_F32) *(vec)to = x[0];
    else {
      v4u part[3];
      cut(x, part);
#pragma unroll
      for (int p = 0; p < 3; p++) *(vec)(to + p * plane) = part[p];
    }
  }
  // Set `set`, to the tile at `lds`; planes lie `plane` bytes apart.  LAST: a step of `tail` k.
  template <bool LAST>
  __device__ __forceinline__ void put(int set, lds_char* lds, int plane) {
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      if (none(i)) return;
      int r, v;
      T::place(i * GEMM_THREADS + (int)threadIdx.x, &r, &v);
      v4u x[WORDS];
#pragma unroll
      for (int w = 0; w < WORDS; w++) x[w] = held[set][i][w];
      if (COL && over) {
        if (short_column(v)) shift_down<DT, WORDS>(x, over);
      }
      if constexpr (LAST) {
        if (!COL && tail - v * 8 > 0 && tail - v * 8 < 8) shift_down<DT, WORDS>(x, 8 - (tail & 7));
        if (COL ? r >= tail : v * 8 >= tail) {
#pragma unroll
          for (int w = 0; w < WORDS; w++) x[w] = v4u{0, 0, 0, 0};
        }
      }
      write(lds + (i * GEMM_THREADS + (int)threadIdx.x) * 16, plane, x);
    }
  }
  // A step of an operand with short rows, entry by entry.
  __device__ __forceinline__ void put_tiny(lds_char* lds, int plane) {
    const int n = (int)max((int64_t)0, min(k_left, (int64_t)BK));
#pragma unroll 1
    for (int i = threadIdx.x; i < T::VECTORS; i += GEMM_THREADS) {
      int r, v;
      T::place(i, &r, &v);
      const bool first = COL ? v * 8 >= cols : r >= cols;      // in the place of a column or row that is not there
      const E* from = begin + (int64_t)(!COL && first ? 0 : r) * stride + (COL && first ? 0 : v * 8);
      const int there = COL ? r >= n ? 0 : first ? min(cols, 8) : min(cols - v * 8, 8) : min(n - v * 8, 8);
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; e++) y[e] = e < there ? Elem<DT>::load(from[e]) : 0.f;
      v4u x[WORDS];
#pragma unroll
      for (int w = 0; w < WORDS; w++) x[w] = Vec<DT>::pack(y + w * Vec<DT>::E);
      write(lds + i * 16, plane, x);
    }
    k_left -= BK;
    begin += COL ? BK * stride : BK;
  }
};

// How a workgroup of eight waves divides a tile of BM x BN: WM x WN of them over
// the tile, and KW over the k of a step (for small tiles, which need many k in
// flight to keep a CU busy): those are summed at the end, and the first WM x WN
// waves hold the result.
// HELD: rows of A that there are at most, where their room in LDS is for more stages.
template <int DT_, bool DIRECT_, bool ACOL_, bool BCOL_, int BM_, int BN_, int WM_, int STAGES_, int KW_ = 1, int HELD_ = BM_>
struct Product {
  static constexpr int DT = DT_, BM = BM_, BN = BN_, WM = WM_, KW = KW_, WN = 8 / WM_ / KW_, STAGES = STAGES_, HELD = HELD_;
  static constexpr bool DIRECT = DIRECT_, ACOL = ACOL_, BCOL = BCOL_;
  // fp32 by rows: A's entries in LDS, cut as they are read; B comes as its three
  // parts, cut ahead, each BN rows of bf16 behind the other.
  static constexpr bool RAW = DIRECT && DT == EXTERND_F32;
  static constexpr int BK = Kind<DT>::BK * (KW > 1 ? 4 : 1), PLANES = RAW ? 1 : Kind<DT>::PLANES, EV = RAW ? 4 : 8, BROWS = RAW ? 3 * BN : BN;
  static constexpr int NK = BK / 16 / KW;                     // of a wave, 16 k each
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  typedef Tile<ACOL, BM, BK, EV> TA;
  typedef Tile<BCOL, BROWS, BK, 8> TB;
  // steps in registers ahead, where loads go through them: small tiles wait for memory
  static constexpr int DEPTH = BN > 32 ? 1 : DT == EXTERND_F32 || KW > 1 ? 2 : 4;
  static constexpr int A_BYTES = TA::BYTES / BM * HELD;
  static constexpr int STAGE = (A_BYTES + TB::BYTES) * PLANES, LOOP_LDS = STAGE * STAGES, JOIN_LDS = KW > 1 ? KW * BM * BN * 4 : 0;
  static constexpr int LDS = LOOP_LDS > JOIN_LDS ? LOOP_LDS : JOIN_LDS;
  static_assert(LDS <= 160 * 1024 && TM >= 1 && TN >= 1 && !(RAW && (ACOL || BCOL || TM > 1 || TN > 1)), "fits");

  static __device__ __forceinline__ int wave() { return (threadIdx.x >> 6) % (WM * WN); }
  static __device__ __forceinline__ int k_wave() { return (threadIdx.x >> 6) / (WM * WN); }
  static __device__ __forceinline__ bool holds() { return KW == 1 || k_wave() == 0; }
  // Entry `r` (0 .. 15) of acc[i][j] is C(m0 + row(i, r), n0 + col(j)).
  static __device__ __forceinline__ int row(int i, int r) {
    return (wave() / WN * TM + i) * 32 + 8 * (r >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (r & 3);
  }
  static __device__ __forceinline__ int col(int j) { return (wave() % WN * TN + j) * 32 + (threadIdx.x & 31); }

  // One step's products, from the tiles at `s`.
  static __device__ __forceinline__ void step(const lds_char* s, f32x16 (*acc)[TN]) {
    const lds_char *a = s, *b = s + TA::BYTES * PLANES;
    const int ma = wave() / WN * TM * 32, nb = wave() % WN * TN * 32;
#pragma unroll
    for (int k = 0; k < NK; k++) {
      const int ks = k_wave() * NK + k;
      v4u fa[PLANES][TM], fb[PLANES][TN];
#pragma unroll
      for (int p = 0; p < PLANES; p++) {
#pragma unroll
        for (int j = 0; j < TN; j++) fb[p][j] = TB::fragment(b + p * TB::BYTES, nb + j * 32, ks);
#pragma unroll
        for (int i = 0; i < TM; i++) fa[p][i] = TA::fragment(a + p * TA::BYTES, ma + i * 32, ks);
      }
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) {
          if constexpr (PLANES == 3) {
            const v4u x[3] = {fa[0][i], fa[1][i], fa[2][i]}, y[3] = {fb[0][j], fb[1][j], fb[2][j]};
            acc[i][j] = mfma_cut(x, y, acc[i][j]);
          } else acc[i][j] = mfma<DT>(fa[0][i], fb[0][j], acc[i][j]);
        }
    }
  }

  // acc = the products over K k's from k0 of A and k0 + b_k of B on; all threads of the workgroup, which has `lds` to itself.
  static __device__ __forceinline__ void run(const Operand& A, int64_t m0, int64_t m_count, const Operand& B, int64_t n0, int64_t n_count,
                                             int64_t k0, int64_t K, lds_char* lds, f32x16 (*acc)[TN], int64_t b_k = 0) {
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
      for (int j = 0; j < TN; j++)
#pragma unroll
        for (int r = 0; r < 16; r++) acc[i][j][r] = 0.f;
    if (K <= 0) return;      // before any load: row k0 need not exist
    const int64_t steps = (K + BK - 1) / BK;
    if constexpr (DIRECT) {
      typedef Direct<ACOL, BM, BK, EV, HELD> DA;
      typedef Direct<BCOL, BROWS, BK, 8> DB;
      static_assert(HELD == BM || !ACOL, "rows of A");
      DA la;
      DB lb;
      la.init(A, m0, m_count, k0, K, (int)threadIdx.x);
      lb.init(B, n0, n_count, k0 + b_k, K, (int)threadIdx.x);
      const int absent = !DA::has(DA::LOADS - 1) + !DB::has(DB::LOADS - 1);      // of a step's loads, in this wave
      auto issue = [&](int stage) {
        la.issue(lds + stage * STAGE);
        lb.issue(lds + stage * STAGE + A_BYTES);
      };
      auto wait = [&](auto stages) {
        constexpr int N = decltype(stages)::value, EACH = DA::LOADS + DB::LOADS;
        if (absent == 0) wait_loads<EACH * N>();
        else if (absent == 1) wait_loads<(EACH - 1) * N>();
        else wait_loads<(EACH - 2) * N>();
        barrier();
      };
      // fp32 by rows is bound by its cuts: of five or six pieces of 32 rows the last
      // ones are shared by two waves, 16 k of a step each, as their SIMDs have one
      // of the first four already (8 rows of 65537, tiles of 136: 181 -> 167 us)
      const int pieces = (int)min((m_count + 31) / 32, (int64_t)8), helped = RAW && (pieces == 5 || pieces == 6) ? pieces - 4 : 0;
      int turn = -1;                                   // which 16 k of a step are this wave's; -1: all, NK or more: none
      static_assert(!RAW || (NK == 2 && WM == 8), "two waves and their two halves");
      // Fragments are read 16 k ahead of their products, those of the next step
      // as well: the barrier and the loads of a step stand in front of products
      // whose operands are in registers.
      static_assert(NK % 2 == 0, "two sets of fragments in turn");
      int ma = wave() / WN * TM * 32;
      const int nb = wave() % WN * TN * 32, k0s = k_wave() * NK;
      if (RAW && helped && wave() >= 4) {
        ma = (4 + (wave() - 4) % helped) * 32;
        turn = (wave() - 4) / helped;
      }
      // of this wave's 32 x 32 products, how many lie in the operands
      const int tm = turn < NK ? (int)max((int64_t)0, min((m_count - ma + 31) / 32, (int64_t)TM)) : 0, tn = (int)max((int64_t)0, min((n_count - nb + 31) / 32, (int64_t)TN));
      for (int s = 0; s < STAGES; s++) issue(s);      // past the last step: zeros, which nothing reads
      wait(std::integral_constant<int, STAGES - 1>());
      auto loop = [&](auto partial) {
        v4u fa[2][TM], fb[2][TN];
        auto read = [&](int set, const lds_char* s, int ks) {
#pragma unroll
          for (int j = 0; j < TN; j++)
            if (!partial || j < tn) fb[set][j] = TB::fragment(s + A_BYTES, nb + j * 32, k0s + ks);
#pragma unroll
          for (int i = 0; i < TM; i++)
            if (!partial || i < tm) fa[set][i] = TA::fragment(s, ma + i * 32, k0s + ks);
        };
        read(0, lds, 0);
        int stage = 0;
        for (int64_t t = 0; t < steps; t++) {
          const int next = stage + 1 == STAGES ? 0 : stage + 1;
#pragma unroll
          for (int ks = 0; ks < NK; ks++) {
            if (ks < NK - 1) read((ks + 1) & 1, lds + stage * STAGE, ks + 1);
            else if (t + 1 < steps) {
              wait(std::integral_constant<int, STAGES - 2>());
              issue(stage);
              read(0, lds + next * STAGE, 0);
            }
#pragma unroll
            for (int i = 0; i < TM; i++)
#pragma unroll
              for (int j = 0; j < TN; j++)
                if (!partial || (i < tm && j < tn)) acc[i][j] = mfma<DT>(fa[ks & 1][i], fb[ks & 1][j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
          }
          stage = next;
        }
      };
      // The same of fp32 by rows.  The cut of the next 16 k goes between the
      // products of these, which wait for one another.
      auto loop_raw = [&](auto partial) {
        v4u raw[2], part[2][3], fb[2][3];
        f32x16 small = {};
        auto mine = [&](int ks) { return !partial || (tm && tn && (turn < 0 || turn == ks)); };
        auto read = [&](int set, const lds_char* s, int ks) {
          if (!mine(ks)) return;
          TA::fragment_f32(s, ma, ks, raw);
#pragma unroll
          for (int p = 0; p < 3; p++) fb[set][p] = TB::fragment(s + A_BYTES, p * BN, ks);
        };
        read(0, lds, 0);
        if (mine(0)) cut(raw, part[0]);
        int stage = 0;
        for (int64_t t = 0; t < steps; t++) {
          const int next = stage + 1 == STAGES ? 0 : stage + 1;
#pragma unroll
          for (int ks = 0; ks < 2; ks++) {
            if (ks == 0) read(1, lds + stage * STAGE, 1);
            else if (t + 1 < steps) {
              wait(std::integral_constant<int, STAGES - 2>());
              issue(stage);
              read(0, lds + next * STAGE, 0);
            }
            const v4u *a = part[ks], *b = fb[ks];
            if (mine(ks)) {
              small = mfma<EXTERND_BF16>(a[1], b[1], small);
              small = mfma<EXTERND_BF16>(a[0], b[2], small);
              small = mfma<EXTERND_BF16>(a[2], b[0], small);
              acc[0][0] = mfma<EXTERND_BF16>(a[0], b[0], acc[0][0]);
              small = mfma<EXTERND_BF16>(a[0], b[1], small);
              small = mfma<EXTERND_BF16>(a[1], b[0], small);
            }
            if (mine(ks ^ 1)) cut(raw, part[ks ^ 1]);      // behind the last step: of what was read before
            if (!partial) {
#pragma unroll
              for (int i = 0; i < 6; i++) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);      // a product,
                __builtin_amdgcn_sched_group_barrier(0x2, 8, 0);      // vector instructions
              }
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          stage = next;
        }
#pragma unroll
        for (int r = 0; r < 16; r++) acc[0][0][r] += small[r];
      };
      // a tile at the operands' ends costs what it holds: 65537 columns are 256 tiles and a small one
      if constexpr (RAW) {
        if (tm < TM || tn < TN || turn >= 0) loop_raw(std::true_type());
        else loop_raw(std::false_type());
      } else if (tm < TM || tn < TN) loop(std::true_type());
      else loop(std::false_type());
      wait_loads<0>();
      barrier();
      if (RAW && helped) {
        typedef __attribute__((address_space(3))) float* floats;
        floats part = (floats)lds + (ma / 32 - 4) * 16 * 64 + (threadIdx.x & 63);
        if (turn == 1) {
#pragma unroll
          for (int r = 0; r < 16; r++) part[r * 64] = acc[0][0][r];
        }
        wait_loads<63>();
        barrier();
        if (turn == 0) {
#pragma unroll
          for (int r = 0; r < 16; r++) acc[0][0][r] += part[r * 64];
        }
        wait_loads<63>();
        barrier();
      }
    } else {
      static_assert(DIRECT || STAGES == 2, "two buffers");
      Staged<DT, ACOL, BM, BK, DEPTH> la;
      Staged<DT, BCOL, BN, BK, DEPTH> lb;
      la.init(A, m0, m_count, k0, K);
      lb.init(B, n0, n_count, k0 + b_k, K);
      auto stage = [&](int u, auto last, bool more) {
        lds_char* const s = lds + (u & 1) * STAGE;
        la.template put<decltype(last)::value>(u % DEPTH, s, TA::BYTES);
        lb.template put<decltype(last)::value>(u % DEPTH, s + TA::BYTES * PLANES, TB::BYTES);
        wait_loads<63>();
        barrier();
        if (more) {
          la.fetch(u % DEPTH);
          lb.fetch(u % DEPTH);
          __builtin_amdgcn_sched_barrier(0);      // the loads go out before the products, not among them
        }
        step(s, acc);
      };
      if (la.tiny || lb.tiny) {
        for (int64_t t = 0; t < steps; t++) {
          la.put_tiny(lds, TA::BYTES);
          lb.put_tiny(lds + TA::BYTES * PLANES, TB::BYTES);
          wait_loads<63>();
          barrier();
          step(lds, acc);
          wait_loads<63>();
          barrier();
        }
      } else {
#pragma unroll
        for (int d = 0; d < DEPTH; d++) {
          la.fetch(d);
          lb.fetch(d);
        }
        constexpr int UNROLL = DEPTH > 1 ? DEPTH : 2;
        const int64_t whole = K / BK;
        int64_t t = 0;
        for (; t + UNROLL <= whole; t += UNROLL) {
#pragma unroll
          for (int u = 0; u < UNROLL; u++) stage(u, std::false_type(), true);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
          if (t + u < whole) stage(u, std::false_type(), DEPTH == 1);
          else if (t + u == whole && whole < steps) stage(u, std::true_type(), false);
        }
      }
      wait_loads<0>();
      barrier();
    }
    if constexpr (KW > 1) {
      // the waves' sums over their k, [wave][entry][lane]: each wave adds up its share, the first reads it all
      typedef __attribute__((address_space(3))) float* floats;
      constexpr int EACH = TM * TN * 16;
      static_assert(WM * WN == 1 && EACH % KW == 0, "one wave holds the tile");
      floats all = (floats)lds + (threadIdx.x & 63);
#pragma unroll
      for (int e = 0; e < EACH; e++) all[(k_wave() * EACH + e) * 64] = acc[e / 16 / TN][e / 16 % TN][e % 16];
      wait_loads<63>();
      barrier();
#pragma unroll
      for (int i = 0; i < EACH / KW; i++) {
        const int e = k_wave() * (EACH / KW) + i;
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < KW; w++) x += all[(w * EACH + e) * 64];
        all[e * 64] = x;
      }
      wait_loads<63>();
      barrier();
      if (holds()) {
#pragma unroll
        for (int e = 0; e < EACH; e++) acc[e / 16 / TN][e / 16 % TN][e % 16] = all[e * 64];
      }
      wait_loads<63>();
      barrier();
    }
  }
};

}  // namespace externd
