// Attention over the cache in 4 bits.
#include <limits.h>
#include <math.h>

#include "externd_decode.hpp"

namespace externd {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef v2u v2u_any __attribute__((aligned(2)));      // 8 bytes at any entry of a 16-bit type (one store all the same)

// A row block that a workgroup begins and others go on with.
struct AttnShare {
  int64_t t0;             // RowBlock's
  int rows, r0, h, count; // cache head; workgroups (below 2: none to join)
};

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
  int window, dtype;
  int q_vec;              // every query starts at a multiple of 16 bytes
  int whole;              // a workgroup per row block and cache head, nothing to join
  int blocks;             // numbers of row blocks (below)
  float* part;            // per workgroup two row blocks' parts; a row: DIM sums, the maximum and the sum of weights, two unused
  AttnShare* shares;      // per workgroup
};

__device__ __forceinline__ float load_any(const void* p, int64_t i, int dtype) {
  if (dtype == EXTERND_F32) return ((const float*)p)[i];
  if (dtype == EXTERND_F16) return (float)((const _Float16*)p)[i];
  return __uint_as_float((unsigned)((const uint16_t*)p)[i] << 16);
}
__device__ __forceinline__ void store_any(void* p, int64_t i, float v, int dtype) {
  if (dtype == EXTERND_F32) ((float*)p)[i] = v;
  else if (dtype == EXTERND_F16) ((_Float16*)p)[i] = (_Float16)v;
  else ((__bf16*)p)[i] = (__bf16)v;
}

// The first position that a query at `pos` sees.  Positions below 0 see none
// either way: counted as 0, so that no window leaves 32 bits.
__device__ __forceinline__ int least_position(const AttnArgs& a, int pos) {
  return a.window > 0 ? max(max(pos, 0) - a.window + 1, 0) : 0;
}

// The queries of one sequence and cache head are rows: row r is new token
// r / each, query head r % each of the cache head.  A row block (ROWS rows)
// sees the tokens lo .. hi - 1 among it, in tiles of 64.
struct RowBlock {
  int64_t t0;          // first new token of the sequence
  int rows, first;     // rows of the sequence; position of its first new token
  int r0;              // the block's first row
  int lo, hi, tiles;
};
template <int ROWS>
__device__ __forceinline__ RowBlock row_block(const AttnArgs& a, int b, int rb) {
  RowBlock r;
  int64_t t0 = a.s.starts ? a.s.starts[b] : b, t1 = a.s.starts ? a.s.starts[b + 1] : b + 1;
  t0 = t0 < 0 ? 0 : t0 > a.s.tokens ? a.s.tokens : t0;
  t1 = t1 < t0 ? t0 : t1 > a.s.tokens ? a.s.tokens : t1;
  r.t0 = t0;
  r.rows = (int)(t1 - t0) * a.each;
  const int len = max(a.s.lens[b], 0);      // below 0 as 0: no position either way
  r.first = len - (int)(t1 - t0);
  const int64_t room = a.s.table_pages << a.c.page_log2;
  const int held = len > room ? (int)room : len;
  r.r0 = rb * ROWS;
  const int r1 = min(r.rows, r.r0 + ROWS) - 1;
  r.hi = min(held, r.first + (r1 < 0 ? 0 : r1 / a.each) + 1);
  r.lo = least_position(a, r.first + min(r.r0, max(r.rows - 1, 0)) / a.each) & ~63;
  r.tiles = ((max(0, r.hi - r.lo) - 1) >> 6) + 1;      // lengths up to 2^31 - 1
  return r;
}

// Row blocks are numbered through the call: those of sequence b from
// starts[b] each / ROWS + b on (some numbers name no block), or evenly with one
// token each.  A workgroup's share is a stretch of the list of all tiles, block
// by block and cache head by cache head, as long as every other's, so lengths
// need not be alike; the first and the last row block of a stretch may be
// shared with neighbours, whose parts are joined by k_attention_join.  A row
// block and head counts as its tiles (one, where it sees nothing) and a few
// units before them, for what a workgroup does besides tiles; a stretch that
// would end or begin in those does so at their start.  (With 1, 4, 8, 12 units,
// 4 rows a block: 128 users of 2000 61, 57, 55, 54 us, 8 of 4000 28, 27, 22, 28.
// With 1, 4, 6, 10, 256 rows: one prompt of 2048 136, 100, 100, 102 us.)
template <int ROWS>
struct Begin {
  static constexpr int UNITS = ROWS == 256 ? 6 : 8;
};
template <int ROWS>
__device__ __forceinline__ int units_of(const RowBlock& r) {
  return max(r.tiles, 1) + Begin<ROWS>::UNITS;
}
template <int ROWS>
__device__ __forceinline__ int64_t first_number(const AttnArgs& a, int b) {
  return (int64_t)max(a.s.starts[b], 0) * a.each / ROWS + b;
}
template <int ROWS>
__device__ __forceinline__ bool numbered_block(const AttnArgs& a, int number, RowBlock* r, int* b) {
  int rb;
  if (!a.s.starts) {
    const int per = (a.each + ROWS - 1) / ROWS;
    *b = number / per;
    rb = number - *b * per;
  } else {
    int lo = 0, hi = a.s.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first_number<ROWS>(a, mid) <= number) lo = mid; else hi = mid - 1;
    }
    *b = lo;
    rb = number - (int)first_number<ROWS>(a, lo);
  }
  if (rb < 0) return false;
  *r = row_block<ROWS>(a, *b, rb);
  return r->r0 < r->rows;
}

struct Walk {
  int64_t at, end, base, total;      // this workgroup's stretch, where the current row block's units begin, all units
  int number, b, groups;
  RowBlock R;
};
__device__ __forceinline__ int64_t uniform64(int64_t v) {
  return (int64_t)((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
                   (unsigned)__builtin_amdgcn_readfirstlane((int)v));
}
// In scalar registers: the same for all threads.
__device__ __forceinline__ void walk_uniform(Walk& w) {
  w.b = __builtin_amdgcn_readfirstlane(w.b);
  w.R.t0 = uniform64(w.R.t0);
  w.R.rows = __builtin_amdgcn_readfirstlane(w.R.rows);
  w.R.first = __builtin_amdgcn_readfirstlane(w.R.first);
  w.R.r0 = __builtin_amdgcn_readfirstlane(w.R.r0);
  w.R.lo = __builtin_amdgcn_readfirstlane(w.R.lo);
  w.R.hi = __builtin_amdgcn_readfirstlane(w.R.hi);
  w.R.tiles = __builtin_amdgcn_readfirstlane(w.R.tiles);
}
// The next row block that is one, from `number` on.
template <int ROWS>
__device__ __forceinline__ void walk_to(const AttnArgs& a, Walk& w, int number) {
  while (!numbered_block<ROWS>(a, number, &w.R, &w.b) && number < a.blocks - 1) number++;
  w.number = number;
  walk_uniform(w);
}
template <int ROWS, int NT>
__device__ __forceinline__ bool walk_begin(const AttnArgs& a, Walk& w) {
  __shared__ int64_t sums[NT / 64 + 1], found_base;
  __shared__ int found;
  const int tid = threadIdx.x;
  if (a.whole) {
    if (!numbered_block<ROWS>(a, blockIdx.x / a.c.heads, &w.R, &w.b)) return false;
    walk_uniform(w);
    const int n = units_of<ROWS>(w.R);
    w.base = 0;
    w.at = (int64_t)(blockIdx.x % a.c.heads) * n;
    w.end = w.at + n;
    return true;
  }
  if (tid == 0) a.shares[blockIdx.x].count = 0;      // until walk_turn finds one
  const int each = (a.blocks + NT - 1) / NT, n0 = min(tid * each, a.blocks), n1 = min(n0 + each, a.blocks);
  int64_t mine = 0;
  RowBlock r;
  int b;
  for (int n = n0; n < n1; n++)
    if (numbered_block<ROWS>(a, n, &r, &b)) mine += (int64_t)units_of<ROWS>(r) * a.c.heads;
  int64_t to = mine;      // inclusive sum
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up(to, d);
    if ((tid & 63) >= d) to += o;
  }
  if ((tid & 63) == 63) sums[tid >> 6] = to;
  __syncthreads();
  int64_t before = 0, total = 0;
  for (int i = 0; i < NT / 64; i++) {
    if (i < tid >> 6) before += sums[i];
    total += sums[i];
  }
  to += before;
  w.total = uniform64(total);
  w.groups = (int)min((int64_t)gridDim.x, w.total);
  if ((int)blockIdx.x >= w.groups) return false;
  w.at = w.total * blockIdx.x / w.groups;
  w.end = w.total * (blockIdx.x + 1) / w.groups;
  if (to - mine <= w.at && w.at < to) {      // one thread: its own row blocks again
    int64_t base = to - mine;
    for (int n = n0; n < n1; n++)
      if (numbered_block<ROWS>(a, n, &r, &b)) {
        const int64_t size = (int64_t)units_of<ROWS>(r) * a.c.heads;
        if (w.at < base + size) {
          found = n;
          found_base = base;
          break;
        }
        base += size;
      }
  }
  __syncthreads();
  w.base = uniform64(found_base);
  walk_to<ROWS>(a, w, __builtin_amdgcn_readfirstlane(found));
  const int n = units_of<ROWS>(w.R), off = (int)((w.at - w.base) % n);
  if (off > Begin<ROWS>::UNITS) return true;
  w.at -= off;
  return w.end - w.at > Begin<ROWS>::UNITS;
}
// The row block's tiles of this turn: cache head, first and last tile, and where its part goes (null: it is whole).
struct Turn {
  int h, tile0, tile1;
  float* part;
};
template <int ROWS, int DIM>
__device__ __forceinline__ Turn walk_turn(const AttnArgs& a, const Walk& w) {
  Turn u;
  const int n = units_of<ROWS>(w.R), off = (int)(w.at - w.base), tiles = n - Begin<ROWS>::UNITS;
  u.h = off / n;
  const int from = off - u.h * n;
  u.tile0 = from ? from - Begin<ROWS>::UNITS : 0;
  u.tile1 = (int)min((int64_t)tiles, from + (w.end - w.at) - Begin<ROWS>::UNITS);
  const bool whole = u.tile0 == 0 && u.tile1 == tiles;
  u.part = whole ? nullptr : a.part + ((int64_t)(2 * blockIdx.x + (u.tile0 == 0)) * ROWS) * (DIM + 4);
  if (!whole && u.tile0 == 0 && threadIdx.x == 0) {
    const int64_t last = w.base + (int64_t)u.h * n + n - 1;
    const int count = (int)(((last + 1) * w.groups - 1) / w.total) - (int)blockIdx.x + 1;
    a.shares[blockIdx.x] = {w.R.t0, w.R.rows, w.R.r0, u.h, count};
  }
  return u;
}
// To the next turn; false at the stretch's end.
template <int ROWS>
__device__ __forceinline__ bool walk_on(const AttnArgs& a, Walk& w, const Turn& u) {
  const int n = units_of<ROWS>(w.R);
  w.at = w.base + (int64_t)(u.h + 1) * n;
  if (w.end - w.at <= Begin<ROWS>::UNITS) return false;
  if (u.h + 1 == a.c.heads) {
    w.base = w.at;
    walk_to<ROWS>(a, w, w.number + 1);
  }
  return true;
}

template <int CTRL>
__device__ __forceinline__ float dppf(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ unsigned dppu(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
// Over the 16 lanes of a row (rotations by 8, 4, 2, 1): every lane has the result.
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, dppf<0x128>(v));
  v = fmaxf(v, dppf<0x124>(v));
  v = fmaxf(v, dppf<0x122>(v));
  return fmaxf(v, dppf<0x121>(v));
}
__device__ __forceinline__ float row_sum(float v) {
  v += dppf<0x128>(v);
  v += dppf<0x124>(v);
  v += dppf<0x122>(v);
  return v + dppf<0x121>(v);
}

// ln of 2^ref sum.  The kernel of 256 rows has its weights up by 2^7 and its
// reference down by as much: out of that first, so that the logarithm is of
// the sum as the definition has it (lse 4.9e-8 of itself, 7.5e-8 otherwise).
constexpr float WEIGHTS_UP = 7.f;
template <int ROWS>
__device__ __forceinline__ float lse_of(float ref, float sum) {
  const float up = ROWS == 256 ? WEIGHTS_UP : 0.f, down = ROWS == 256 ? 1.f / 128 : 1.f;
  return (ref + up + log2f(sum * down)) * 0.69314718055994530942f;
}

__device__ __forceinline__ float scale_of(unsigned word) {
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(word & 0xFFF0u));
}

// Four signed base-256 digits of a whole number below 2^31 - 2^23, lowest first.
__device__ __forceinline__ unsigned digits_of(int u) { return ((unsigned)u + 0x00808080u) ^ 0x00808080u; }

// Attention of up to four rows over one part of a sequence, by integer matrix
// products.  The codes are whole numbers already; a query row enters as 31-bit
// whole numbers (of its largest entry) in four base-256 digits, and so do the
// softmax weights times the values' scales, 64 tokens at a time.  So
//   scores:  A = digits of 4 rows (16 x 64 channels), B = codes of 16 tokens,
//   values:  A = digits of 4 rows' weights (16 x 64 tokens), B = codes of 16 channels
// on v_mfma_i32_16x16x64_i8, whose result leaves a row's four digits in one
// lane: they are put together there, exactly.  The zero points enter as whole
// numbers too (a multiple of the query's digit sum; an accumulator that starts
// at minus the weighted zero points), so codes equal to the zero point add
// nothing at all.  A code becomes a matrix operand by one mask (3 operations for
// 8 codes), where conversion to floating point would take 8 or more; this is
// what the memory-bound case needs (14 TB/s of codes in instructions).
//
// Roundings: a query to 31 bits of its row's largest entry; a weight times a
// scale to 30 bits of the tile's largest (to its own 24 and less with FINE, for
// fp32 results); sums and the running maximum are fp32.
//
// Four waves share a part; each takes every fourth tile of 64 tokens with its
// own running maximum, and they are joined at the end.  Four rows always: with
// 8 or 16 rows a workgroup the codes are taken apart less often, but the
// registers leave half the waves (20 rows over 4001 tokens 50 us, now 33; 8 rows of
// 256 channels over 13848 50 us, now 36).  Bound by memory: 32 users' 363 MB in
// 75 us (4.9 TB/s), 143 MB of one of 131071 tokens in 32 us (4.5), where a
// start of about 8 us (lengths, table, first tiles, one after another) is what
// is left above the 6.3 TB/s that plain loads reach.
template <int DIM, bool FINE>
__global__ __launch_bounds__(256, DIM <= 128 ? 3 : 2) void k_attention_split(AttnArgs a) {
  constexpr int NG = DIM / KV4_GROUP, HALF = DIM / 2, ROWS = 4;
  constexpr int NU = DIM == 256 ? 2 : 1;     // 16-byte K loads of a lane and token
  constexpr int NC = DIM / 32;               // 16-byte V loads of a lane: 16 byte columns each
  constexpr int QROW = 80, PROW = 80;        // bytes of a digit row of 64 in LDS (padded against bank conflicts)
  constexpr int ACC = DIM + 4;               // floats of a row when waves join
  constexpr int SHARED_Q = NG * 16 * QROW, SHARED_P = 4 * NG * (16 * PROW + 64), SHARED_O = 4 * ROWS * ACC * 4;
  constexpr int SHARED = SHARED_Q + SHARED_P > SHARED_O ? SHARED_Q + SHARED_P : SHARED_O;
  __shared__ __align__(16) uint8_t lds[SHARED];
  __shared__ float row_factor[ROWS];
  __shared__ int row_sums[ROWS][NG][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, seg = lane >> 4;
  const int P = 1 << a.c.page_log2;
  Walk W;
  if (!walk_begin<ROWS, 256>(a, W)) return;

  while (true) {
    const RowBlock& R = W.R;
    const Turn turn = walk_turn<ROWS, DIM>(a, W);
    const int b = W.b, h = turn.h;
    if (R.tiles == 0) {      // rows that see nothing
      for (int i = threadIdx.x; i < ROWS * DIM; i += 256) {
        const int r = R.r0 + i / DIM;
        if (r >= R.rows) break;
        const int64_t o = (R.t0 + r / a.each) * a.heads_q + h * a.each + r % a.each;
        store_any(a.out, o * DIM + i % DIM, 0.f, a.dtype);
        if (a.lse && i % DIM == 0) a.lse[o] = -INFINITY;
      }
      if (!walk_on<ROWS>(a, W, turn)) return;
      continue;
    }
    const int c0 = R.lo + 64 * turn.tile0, c1 = (int)min((int64_t)R.hi, (int64_t)R.lo + 64 * (int64_t)turn.tile1);
    const int ntiles = turn.tile1 - turn.tile0;
    uint8_t* const pbuf = lds + SHARED_Q + wave * (NG * (16 * PROW + 64));
    uint8_t* const zbuf = pbuf + NG * 16 * PROW;
    constexpr int NW = NG == 1 ? 1 : NG / 2;    // 32-bit loads of a token's K words (V's likewise; one for both at 64)
    v4u kr[4][NU], vr[NC];
    unsigned kw[4][NW], vw[4][NW];
    uint64_t ok = 0;        // bit 16 t: block t of the tile has a page (as lanes say)
    // table entry of this lane's block (seg) of a tile; only read here, so that nothing waits for it yet
    auto entry = [&](int tile) -> int {
      const unsigned tok = min((unsigned)c0 + (unsigned)tile * 64 + seg * 16, (unsigned)(c1 - 1));
      return a.s.table[(int64_t)b * a.s.table_pages + (tok >> a.c.page_log2)];
    };
    // its page's place in the cache; `has`: whether there is one (a page for no tokens reads page 0)
    auto place = [&](int tile, int page, bool* has) -> uint64_t {
      *has = (unsigned)c0 + (unsigned)tile * 64 + seg * 16 < (unsigned)c1 && page >= 0 && page < a.c.num_pages;
      return (uint64_t)((int64_t)(*has ? page : 0) * a.c.heads + h) * (uint64_t)a.c.head_bytes;
    };
    auto base_of = [&](uint64_t off, int t) -> const uint8_t* {
      const unsigned lo = __builtin_amdgcn_readlane((unsigned)off, 16 * t);
      const unsigned hi = __builtin_amdgcn_readlane((unsigned)(off >> 32), 16 * t);
      return a.cache + ((uint64_t)hi << 32 | lo);
    };
    auto load_k = [&](int tile, uint64_t off) {
#pragma unroll
      for (int t = 0; t < 4; t++) {
        const uint8_t* base = base_of(off, t);
        const unsigned o = (((unsigned)c0 + (unsigned)tile * 64 + 16 * t) & (P - 1)) + l16;
        const uint8_t* kp = base + o * HALF + seg * (DIM == 64 ? 8 : 16);
        if constexpr (DIM == 64) {
          const v2u x = *(const v2u*)kp;
          kr[t][0] = v4u{x[0], x[1], 0, 0};
        } else {
#pragma unroll
          for (int u = 0; u < NU; u++) kr[t][u] = *(const v4u*)(kp + 64 * u);
        }
        const unsigned* wp = (const unsigned*)(base + (unsigned)P * DIM + o * (4 * NG));
#pragma unroll
        for (int g = 0; g < NW; g++) kw[t][g] = wp[g];
      }
    };
    auto load_v = [&](int tile, uint64_t off) {
      const unsigned tok = (unsigned)c0 + (unsigned)tile * 64;
#pragma unroll
      for (int t = 0; t < 4; t++) {
        if constexpr (NG > 1) {
          const unsigned o = ((tok + 16 * t) & (P - 1)) + l16;
          const unsigned* wp = (const unsigned*)(base_of(off, t) + (unsigned)P * DIM + o * (4 * NG)) + NW;
#pragma unroll
          for (int g = 0; g < NW; g++) vw[t][g] = wp[g];
        }
      }
      const uint8_t* vp = a.cache + off + (unsigned)P * HALF + (((tok + 16 * seg) & (P - 1)) >> 4) * (HALF * 16) + l16 * 16;
#pragma unroll
      for (int c = 0; c < NC; c++) vr[c] = *(const v4u*)(vp + c * 256);
    };
    auto k_word = [&](int t, int g) -> unsigned { return g & 1 ? kw[t][g / 2] >> 16 : kw[t][g / 2] & 0xFFFFu; };
    auto v_word = [&](int t, int g) -> unsigned {
      if (NG == 1) return vw[t][0] >> 16;
      return g & 1 ? vw[t][g / 2] >> 16 : vw[t][g / 2] & 0xFFFFu;
    };

    // the first tile's loads are in flight while the queries are taken apart
    const int here = entry(wave);
    int ahead = entry(wave + 4);
    {
      bool has = false;
      const uint64_t off = place(wave, here, &has);
      ok = __ballot(has);
      load_k(wave, off);
      load_v(wave, off);
    }

    // ---- the rows' digits, one wave per row ----
    {
      const int r = wave, row = R.r0 + r;
      float x[NG], top = 0.f;
      bool bad = false;
#pragma unroll
      for (int g = 0; g < NG; g++) {
        x[g] = 0.f;
        if (row < R.rows) {
          const int64_t at = (R.t0 + row / a.each) * a.q_ts + (h * a.each + row % a.each) * a.q_hs;
          x[g] = load_any(a.q, at + g * 64 + lane, a.dtype);
        }
        bad |= !__builtin_isfinite(x[g]);
        top = fmaxf(top, fabsf(x[g]));
      }
      bad = __any(bad);
      for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
      int e = 0;
      frexpf(top, &e);                  // top < 2^e
#pragma unroll
      for (int g = 0; g < NG; g++) {
        const int u = bad ? 0 : (int)rintf(ldexpf(x[g], 30 - e));
        const unsigned dg = digits_of(u);
        // channel 64 g + lane: its group's slot (the byte's place in a lane's K load)
        const int slot = DIM == 64 ? ((lane & 31) >> 3) * 16 + (lane >> 5) * 8 + (lane & 7) : lane;
        uint8_t* to = lds + (g * 16 + r * 4) * QROW + slot;
        int hi = 0, lo = 0;
#pragma unroll
        for (int d = 0; d < 4; d++) {
          const int v = (int8_t)(dg >> (8 * d));
          to[d * QROW] = (uint8_t)v;
          (d >= 2 ? hi : lo) += v << (8 * (d & 1));
        }
        for (int d = 32; d; d >>= 1) {
          hi += __shfl_xor(hi, d);
          lo += __shfl_xor(lo, d);
        }
        if (lane == 0) {
          row_sums[r][g][0] = hi;
          row_sums[r][g][1] = lo;
        }
      }
      // scores in powers of two: x log2(e)
      if (lane == 0) row_factor[r] = bad ? NAN : ldexpf(a.scale * 1.44269504088896340736f, e - 30);
    }
    __syncthreads();
    v4i Q[NG];
    int qhi[NG], qlo[NG];
    float O[2 * NC], poison[NG];
#pragma unroll
    for (int g = 0; g < NG; g++) {
      Q[g] = *(const v4i*)(lds + (g * 16 + l16) * QROW + seg * 16);
      qhi[g] = -row_sums[seg][g][0];
      qlo[g] = -row_sums[seg][g][1];
      poison[g] = 0.f;
    }
    const float factor = row_factor[seg];
    float m = -INFINITY, l = 0.f;
    const int row = R.r0 + seg, pos = R.first + min(row, R.rows - 1) / a.each;
    const int last = row < R.rows ? min(pos, c1 - 1) : -1;
    const int least = least_position(a, pos);
#pragma unroll
    for (int i = 0; i < 2 * NC; i++) O[i] = 0.f;
    // One tile: K's registers are free once the scores are there and take the
    // next tile's K then; V's likewise at the end.
    auto compute = [&](int tile, int next_entry) {
      const int tok = c0 + tile * 64 + l16;
      const v4i zero = {0, 0, 0, 0};
      float x[4];
      // ---- scores ----
#pragma unroll
      for (int t = 0; t < 4; t++) {
        v4i kop[NG];
        if constexpr (DIM == 64) {
          kop[0] = v4i{(int)(kr[t][0][0] & 0x0F0F0F0Fu), (int)(kr[t][0][1] & 0x0F0F0F0Fu),
                       (int)((kr[t][0][0] >> 4) & 0x0F0F0F0Fu), (int)((kr[t][0][1] >> 4) & 0x0F0F0F0Fu)};
        } else {
#pragma unroll
          for (int u = 0; u < NU; u++) {
            kop[u] = (v4i)(kr[t][u] & 0x0F0F0F0Fu);
            kop[NU + u] = (v4i)((kr[t][u] >> 4) & 0x0F0F0F0Fu);
          }
        }
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < NG; g++) {
          const unsigned word = k_word(t, g);
          const v4i r = __builtin_amdgcn_mfma_i32_16x16x64_i8(Q[g], kop[g], zero, 0, 0, 0);
          const int z = (int)(word & 15);
          const int hi = __mul24(z, qhi[g]) + ((r[3] << 8) + r[2]);
          const int lo = __mul24(z, qlo[g]) + ((r[1] << 8) + r[0]);
          sum = fmaf(scale_of(word), fmaf((float)hi, 65536.f, (float)lo), sum);
        }
        x[t] = sum * factor;
        if constexpr (NG >= 4) __builtin_amdgcn_sched_barrier(0);      // one block's registers at a time
      }
      if constexpr (NG == 1) {
#pragma unroll
        for (int t = 0; t < 4; t++) vw[t][0] = kw[t][0];
      }
      // always loaded, so that the number of loads in flight is known where they are waited for: past the part's end
      // a few lines of page 0, the same for all
      bool has = false;
      const uint64_t next = place(tile + 4, next_entry, &has);
      const uint64_t next_ok = __ballot(has);
      __builtin_amdgcn_sched_barrier(0);
      load_k(tile + 4, next);
      // ---- zero points of the values, negated, for the accumulators' start ----
#pragma unroll
      for (int t = 0; t < 4; t++)
#pragma unroll
        for (int g = 0; g < NG; g++)
          zbuf[g * 64 + 16 * t + l16] = (uint8_t)(0u - (v_word(t, g) & 15));
      // ---- softmax weights of this lane's row and tokens ----
      bool seen[4];
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; t++) {
        const int pos = tok + 16 * t;
        seen[t] = (bool)(ok >> (16 * t) & 1) & (pos <= last) & (pos >= least);
        x[t] = seen[t] ? x[t] : -INFINITY;
        top = fmaxf(top, x[t]);
      }
      const float mn = fmaxf(m, row_max(top)), at = mn == -INFINITY ? 0.f : mn;
      const float keep = __builtin_amdgcn_exp2f(m - at);
      m = mn;
      float w[4];
      l *= keep;
#pragma unroll
      for (int t = 0; t < 4; t++) {
        w[t] = __builtin_amdgcn_exp2f(x[t] - at);
        l += w[t];
      }
      // ---- times the values' scales, as whole numbers of the tile's largest, four digits ----
      float ws[NG][4];
#pragma unroll
      for (int g = 0; g < NG; g++)
#pragma unroll
        for (int t = 0; t < 4; t++) {
          ws[g][t] = seen[t] ? w[t] * scale_of(v_word(t, g)) : 0.f;
          poison[g] = fmaf(ws[g][t], 0.f, poison[g]);
        }
#pragma unroll
      for (int c = 0; c < 2 * NC; c++) O[c] *= keep;
      for (int round = 0; round < 8; round++) {
        float back[NG], left = 0.f;
#pragma unroll
        for (int g = 0; g < NG; g++) {
          const float big = row_max(fmaxf(fmaxf(ws[g][0], ws[g][1]), fmaxf(ws[g][2], ws[g][3])));
          // big < 2^(e - 126): whole numbers below 2^30
          const unsigned e = max(__float_as_uint(big) >> 23, 30u);
          const float up = __uint_as_float((283u - e) << 23);
          back[g] = __uint_as_float((e - 29u) << 23);
#pragma unroll
          for (int t = 0; t < 4; t++) {
            const int u = (int)(ws[g][t] * up);
            ws[g][t] = fmaf(-(float)u, back[g], ws[g][t]);      // what the whole numbers leave, exactly
            left = fmaxf(left, ws[g][t]);
            const unsigned d0 = digits_of(u);
            // 4 x 4 bytes among neighbouring lanes: lane i of four gets digit i of the four tokens
            const unsigned d1 = __builtin_amdgcn_perm(dppu<0xB1>(d0), d0, lane & 1 ? 0x03070105u : 0x06020400u);
            const unsigned d2 = __builtin_amdgcn_perm(dppu<0x4E>(d1), d1, lane & 2 ? 0x03020706u : 0x05040100u);
            *(unsigned*)(pbuf + (g * 16 + seg * 4 + (lane & 3)) * PROW + 16 * t + (l16 & 12)) = d2;
          }
        }
        // ---- weighted sums ----
        v4i A[NG], start[NG];
#pragma unroll
        for (int g = 0; g < NG; g++) {
          A[g] = *(const v4i*)(pbuf + (g * 16 + l16) * PROW + seg * 16);
          const v4i zb = *(const v4i*)(zbuf + g * 64 + seg * 16);
          start[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(A[g], zb, zero, 0, 0, 0);
        }
#pragma unroll
        for (int c = 0; c < NC; c++) {
          const v4i vlo = (v4i)(vr[c] & 0x0F0F0F0Fu), vhi = (v4i)((vr[c] >> 4) & 0x0F0F0F0Fu);
          const int glo = c / 4, ghi = DIM == 64 ? 0 : NG / 2 + c / 4;
          const v4i r0 = __builtin_amdgcn_mfma_i32_16x16x64_i8(A[glo], vlo, start[glo], 0, 0, 0);
          const v4i r1 = __builtin_amdgcn_mfma_i32_16x16x64_i8(A[ghi], vhi, start[ghi], 0, 0, 0);
          const float f0 = fmaf((float)((r0[3] << 8) + r0[2]), 65536.f, (float)((r0[1] << 8) + r0[0]));
          const float f1 = fmaf((float)((r1[3] << 8) + r1[2]), 65536.f, (float)((r1[1] << 8) + r1[0]));
          O[c] = fmaf(f0, back[glo], O[c]);
          O[NC + c] = fmaf(f1, back[ghi], O[NC + c]);
        }
        // 16-bit results end here: what is left is below 2^-30 of the tile's largest weight.  fp32 results keep
        // every weight's own 24 bits: again with what is left (twice in all where no weight is below 2^-37), until
        // that is below the smallest normal number.  A round leaves less than 2^-29 of the largest weight, or
        // less than 2^-126: weights are at most 4352, so six rounds at most.
        // masks anew each time: kept, they cost 32 registers
        if (FINE)
#pragma unroll
          for (int c = 0; c < NC; c++) asm volatile("" : "+v"(vr[c]));
        if (!FINE || !__any(left >= 1.17549435e-38f)) break;
      }
      __builtin_amdgcn_sched_barrier(0);      // into the registers that this tile's have left
      load_v(tile + 4, next);
      ok = next_ok;
    };

    // by two, so that no register is copied (and its load waited for) at the loop's end
    for (int tile = wave; tile < ntiles; tile += 8) {
      const int after = entry(tile + 8);
      compute(tile, ahead);
      if (tile + 4 >= ntiles) break;
      ahead = entry(tile + 12);
      compute(tile + 4, after);
    }

    // ---- join the four waves: lane (row, channel) sums of each, then by the row's maximum ----
    __syncthreads();
    float* const acc = (float*)lds;
    float* o = acc + (wave * ROWS + seg) * ACC;
    const float sum = row_sum(l);
#pragma unroll
    for (int c = 0; c < NC; c++) {
      const int glo = c / 4, ghi = DIM == 64 ? 0 : NG / 2 + c / 4;
      o[16 * c + l16] = O[c] + row_sum(poison[glo]);
      o[HALF + 16 * c + l16] = O[NC + c] + row_sum(poison[ghi]);
    }
    if (l16 == 0) {
      o[DIM] = m;
      o[DIM + 1] = sum;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < ROWS * DIM; i += 256) {
      const int r = i / DIM, d = i % DIM, row = R.r0 + r;
      if (row >= R.rows) break;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < 4; w++) top = fmaxf(top, acc[(w * ROWS + r) * ACC + DIM]);
      const float at = top == -INFINITY ? 0.f : top;
      float o = 0.f, sum = 0.f;
#pragma unroll
      for (int w = 0; w < 4; w++) {
        const float* from = acc + (w * ROWS + r) * ACC;
        const float f = __builtin_amdgcn_exp2f(from[DIM] - at);
        o = fmaf(from[d], f, o);
        sum = fmaf(from[DIM + 1], f, sum);
      }
      const int64_t to = (R.t0 + row / a.each) * a.heads_q + h * a.each + row % a.each;
      if (!turn.part) {
        const bool none = sum == 0.f;
        store_any(a.out, to * DIM + d, none ? 0.f : o / sum, a.dtype);
        if (a.lse && d == 0) a.lse[to] = none ? -INFINITY : lse_of<ROWS>(top, sum);
      } else {
        float* part = turn.part + r * (DIM + 4);
        part[d] = o;
        if (d == 0) {
          part[DIM] = top;
          part[DIM + 1] = sum;
        }
      }
    }
    if (!walk_on<ROWS>(a, W, turn)) return;
    __syncthreads();
  }
}

// Attention of 256 rows over one part of a sequence, for 16-bit queries: the
// codes become fp16 values in LDS, shared by eight waves of 32 rows each, and
//   S^T = K Q^T  and  O^T += V^T P^T  on v_mfma_f32_32x32x16_f16.
// Every value s (code - z) is exactly an fp16 number and a query row enters as
// fp16 with its largest entry near 2^15 (exact for bf16 entries within 2^-29
// of it), so the scores are fp32 sums of exact products; only the softmax weights are
// rounded, to fp16 for the second product (their sum takes them as they are),
// as the values take the other operand's 11 bits whole and a second part of the
// weights would be half as many products again.  Relative error against 64 bits
// (1 K tokens over 6 K), with that rounding and without: bf16 results 1.668e-3
// and 1.656e-3, fp16 results 2.91e-4 and 2.07e-4.  S^T leaves a row's scores in two
// lanes, whose registers, rounded, are the second product's operand as they
// are: token order within 16 is free, so V is stored in the order that S^T has.
//
// A tile of TT tokens is converted once (4 operations for 2 codes: mask to
// 1024 + code, subtract 1024 + z, times s) while the tiles before are in work.
// The weights are taken against a running reference, 2^-7 of the row's maximum
// when it is set, that moves only when a weight passes 2^15, so O is rarely
// rescaled and a weight below 2^8 times the maximum of then fits fp16 (65504).
// So weights have 11 bits down to 2^-21 of that maximum and are 0 only below
// 2^-32 of it: many weak keys beside a strong one whose value is small are the
// result.  (Moving at 2^4 times, 2^-25 and 2^-36: 256 channels 1.5 % slower.)
//
// Bound by the vector instructions between the products, and by the clock that
// falls to 1.8 GHz under both: a wave's step of 64 tokens at 128 channels has 32
// products of 32 cycles and 328 vector instructions (32 exponentials of 16
// cycles among them), so a SIMD's two waves have 2048 and 3400 cycles of the
// 4560 that a step takes.  3.5 K tokens of 32 heads over 12 K with the join in
// 570 to 605 us as the clock allows, 855 to 907 TFLOP/s.  All waves in one phase:
// 700 us; conversion among the products: 754; rows padded to an odd number of
// units instead of permuted (48 instructions fewer): 619 against 614.  Registers:
// at 128 channels what is spilled is used outside the tile loop only; at 256 a
// step reads 24 spilled words back.
template <int DIM, int DT>
__global__ __launch_bounds__(512, 2) void k_attention_chunk(AttnArgs a) {
  typedef typename Elem<DT>::T T;
  constexpr int NG = DIM / KV4_GROUP, HALF = DIM / 2, ROWS = 256;
  constexpr int TT = DIM == 256 ? 32 : 64;          // tokens of a tile
  constexpr int NS = TT / 32, KS = DIM / 16, PS = TT / 16, CT = DIM / 32;
  constexpr int KU = DIM / 8, VU = TT / 8;          // 16-byte units of a row of K (a token) and of V (a channel)
  constexpr int WB = 8 / PS;                        // waves of a 16-token block
  constexpr int AHEAD = 4;
  constexpr float UP = WEIGHTS_UP, TOP = 15.f;      // powers of two of the weights (above)
  constexpr float BAD = 5.87747175e-39f;            // 2^-127
  __shared__ __align__(16) _Float16 kt[3][TT * DIM], vt[3][DIM * TT];
  __shared__ __align__(8) uint8_t flags[3][8];      // of each wave's 8 values' tokens: 1 there, 3 some NaN among them
  __shared__ uint16_t nans[3][8][NG];               // which of the block's tokens
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
  const int P = 1 << a.c.page_log2;
  const int block = wave / WB;                      // the 16-token block of a tile that this wave converts
  const int vhalf = WB == 2 ? wave & 1 : (wave >> 1) & 1;      // of it, tokens 4 vhalf + {0..3, 8..11}
  const int vcol = WB == 2 ? lane : (wave & 1) * 64 + lane;    // byte column of V
  const bool vin = DIM > 64 || lane < 32;
  const int ktok = DIM == 256 ? wave * 4 + (lane >> 4) : DIM == 128 ? wave * 8 + (lane >> 3) : wave * 8 + ((lane & 31) >> 2);
  const int kunit = DIM == 256 ? lane & 15 : DIM == 128 ? lane & 7 : lane & 3;
  // 16-byte units are permuted within a row so that 16 rows' same unit spans all banks
  auto kat = [](int tok, int u) { return (tok * KU + (DIM == 64 ? u ^ ((tok >> 1) & 7) : u ^ (tok & 15))) * 8; };
  auto vat = [](int ch, int u) { return (ch * VU + (TT == 64 ? u ^ ((ch >> 1) & 7) : u ^ ((ch >> 2) & 3))) * 8; };

  Walk W;
  if (!walk_begin<ROWS, 512>(a, W)) return;
  while (true) {
    const RowBlock& R = W.R;
    const Turn turn = walk_turn<ROWS, DIM>(a, W);
    const int b = W.b, h = turn.h;
    const int row = R.r0 + wave * 32 + l32;
    const int64_t to = (R.t0 + row / a.each) * a.heads_q + h * a.each + row % a.each;
    if (R.tiles == 0) {      // rows that see nothing
      if (row < R.rows) {
        for (int d = half; d < DIM; d += 2) ((T*)a.out)[to * DIM + d] = Elem<DT>::store(0.f);
        if (a.lse && !half) a.lse[to] = -INFINITY;
      }
      if (!walk_on<ROWS>(a, W, turn)) return;
      continue;
    }
    const int c0 = R.lo + 64 * turn.tile0, c1 = (int)min((int64_t)R.hi, (int64_t)R.lo + 64 * (int64_t)turn.tile1);

    // ---- this lane's half of its row's query, as fp16 ----
    f16x8 Q[KS];
    float factor;
    {
      v4u raw[KS];
      const T* q = (const T*)a.q + (R.t0 + min(row, R.rows - 1) / a.each) * a.q_ts + (h * a.each + row % a.each) * a.q_hs + half * 8;
#pragma unroll
      for (int k = 0; k < KS; k++) {
        if (a.q_vec) raw[k] = *(const v4u*)(q + k * 16);
        else {
          const uint16_t* u = (const uint16_t*)(q + k * 16);
#pragma unroll
          for (int i = 0; i < 4; i++) raw[k][i] = (unsigned)u[2 * i] | (unsigned)u[2 * i + 1] << 16;
        }
      }
      float top = 0.f;
      bool bad = false;
#pragma unroll
      for (int k = 0; k < KS; k++) {
        float x[8];
        Vec<DT>::unpack(raw[k], x);
#pragma unroll
        for (int j = 0; j < 8; j++) {
          bad |= !__builtin_isfinite(x[j]);
          top = fmaxf(top, fabsf(x[j]));
        }
      }
      top = fmaxf(top, __shfl_xor(top, 32));
      bad |= __shfl_xor((int)bad, 32) != 0;
      int e = 0;
      frexpf(top, &e);                  // top < 2^e
      const float sign = a.scale < 0.f ? -1.f : 1.f;
#pragma unroll
      for (int k = 0; k < KS; k++) {
        constexpr int order[8] = {0, 2, 1, 3, 4, 6, 5, 7};      // as two codes come out of one mask
        float x[8];
        Vec<DT>::unpack(raw[k], x);
#pragma unroll
        for (int j = 0; j < 8; j++) Q[k][j] = (_Float16)(bad ? 0.f : ldexpf(sign * x[order[j]], 15 - e));
      }
      // above 0, so that a masked score of -infinity stays one; below the least of other rows marks a row that is NaN
      factor = bad ? BAD : fmaxf(ldexpf(fabsf(a.scale) * 1.44269504088896340736f, e - 15), 1.17549435e-38f);
    }
    const int pos = R.first + min(row, R.rows - 1) / a.each;
    const int last = row < R.rows ? max(min(pos, c1 - 1), -1) : -1;
    const int least = least_position(a, pos);
    // over the wave: where every row sees every token
    int all_from = row < R.rows ? least : INT_MIN, all_to = row < R.rows ? last : INT_MAX;
    for (int d = 16; d; d >>= 1) {
      all_from = max(all_from, __shfl_xor(all_from, d));
      all_to = min(all_to, __shfl_xor(all_to, d));
    }
    all_from = __builtin_amdgcn_readfirstlane(all_from);
    all_to = __builtin_amdgcn_readfirstlane(all_to);

    f32x16 O[CT];
#pragma unroll
    for (int c = 0; c < CT; c++)
#pragma unroll
      for (int i = 0; i < 16; i++) O[c][i] = 0.f;
    float ref = -INFINITY, l = 0.f, poison[NG];
#pragma unroll
    for (int g = 0; g < NG; g++) poison[g] = 0.f;

    const int ntiles = (c1 - c0 - 1) / TT + 1;
    struct KRaw {
      v2u codes;
      unsigned words[(NG + 1) / 2];
    };
    struct VRaw {
      unsigned codes[2], words[(NG + 1) / 2];      // words: of the token that lane % 8 stands for
    };
    const int vtok = 4 * vhalf + (lane & 3) + (lane & 4) * 2;
    // this wave's block of a tile; may be past the part's end, and 2^31
    auto tile_at = [&](int tile) -> unsigned { return (unsigned)c0 + (unsigned)tile * TT + block * 16; };
    // its table entry; only read here, so that nothing waits for it yet
    auto entry = [&](int tile) -> int {
      const unsigned tok = min(tile_at(tile), (unsigned)(c1 - 1));
      return a.s.table[(int64_t)b * a.s.table_pages + (tok >> a.c.page_log2)];
    };
    // where the block is; no page (past the part's end as well): page 0, so that all loads are always issued and their
    // number in flight is known where they are waited for
    struct Place {
      const uint8_t* base;
      bool there;
    };
    const int64_t page_bytes = a.c.heads * a.c.head_bytes;
    const uint8_t* const head_base = a.cache + h * a.c.head_bytes;
    auto place_at = [&](int tile, int page) -> Place {
      page = __builtin_amdgcn_readfirstlane(page);
      const bool there = tile_at(tile) < (unsigned)c1 && (unsigned)page < (unsigned)a.c.num_pages;
      return {head_base + (there ? page : 0) * page_bytes, there};
    };
    auto load_k = [&](KRaw& r, int tile, const Place& pl) {
      const uint8_t* base = pl.base;
      const int t = (int)(tile_at(tile) & (P - 1)) + (ktok & 15);
      r.codes = *(const v2u*)(base + t * HALF + kunit * 8);
#pragma unroll
      for (int g = 0; g < (NG + 1) / 2; g++) r.words[g] = ((const unsigned*)(base + (unsigned)P * DIM + t * (4 * NG)))[g];
    };
    auto load_v = [&](VRaw& r, int tile, const Place& pl) {
      const uint8_t* base = pl.base;
      const int o = (int)(tile_at(tile) & (P - 1));
      const unsigned* vp = (const unsigned*)(base + (unsigned)P * HALF + (o >> 4) * (HALF * 16) + (vin ? vcol : 0) * 16);
      r.codes[0] = vp[vhalf];
      r.codes[1] = vp[2 + vhalf];
      const unsigned* w = (const unsigned*)(base + (unsigned)P * DIM + (o + vtok) * (4 * NG));
#pragma unroll
      for (int g = 0; g < (NG + 1) / 2; g++) r.words[g] = NG == 1 ? w[0] >> 16 : w[NG / 2 + g];
    };
    // one dword of codes to four pairs of values: bytes (0, 2), (1, 3) of the low nibbles, then of the high ones
    unsigned magic = 0x64006400u;      // in a register: mask and magic are one operation then
    asm("" : "+v"(magic));
    auto pair = [&](unsigned w, unsigned minus, unsigned scale) -> unsigned {
      const f16x2 c = __builtin_bit_cast(f16x2, (w & 0x000F000Fu) | magic);
      return __builtin_bit_cast(unsigned, (c + __builtin_bit_cast(f16x2, minus)) * __builtin_bit_cast(f16x2, scale));
    };
    auto convert_k = [&](int buf, const KRaw& raw) {
        // K: the low nibbles are unit kunit, the high ones unit kunit + KU / 2
        unsigned out[2][4];
#pragma unroll
        for (int s = 0; s < 2; s++) {
          // groups of byte column 8 kunit: below D / 2, and D / 2 further
          const int g = DIM == 256 ? 2 * s : DIM == 128 ? s : 0;
          unsigned w = DIM == 256 ? raw.words[s] : raw.words[0];
          w = DIM == 256 ? (kunit >= 8 ? w >> 16 : w & 0xFFFFu) : g & 1 ? w >> 16 : w & 0xFFFFu;
          w |= w << 16;
          const unsigned scale = w & 0xFFF0FFF0u, minus = (w & 0x000F000Fu) | 0xE400E400u;
#pragma unroll
          for (int j = 0; j < 2; j++) {
            out[s][2 * j] = pair(raw.codes[j] >> (4 * s), minus, scale);
            out[s][2 * j + 1] = pair(raw.codes[j] >> (4 * s + 8), minus, scale);
          }
        }
        if (vin) {
          *(v4u*)&kt[buf][kat(ktok, kunit)] = v4u{out[0][0], out[0][1], out[0][2], out[0][3]};
          *(v4u*)&kt[buf][kat(ktok, kunit + KU / 2)] = v4u{out[1][0], out[1][1], out[1][2], out[1][3]};
        }
    };
    auto convert_v = [&](int buf, int tile, bool there, const VRaw& raw) {
        // V: words of tokens that are not there count as 0, NaN ones too (kept as bits)
        const bool in = there && tile_at(tile) + vtok < (unsigned)c1;
        unsigned flag = there, bad[(NG + 1) / 2], scale[NG][4], minus[NG][4];
#pragma unroll
        for (int g = 0; g < (NG + 1) / 2; g++) {
          unsigned w = in ? raw.words[g] : 0u;
          const bool lo = (w & 0x7C00u) == 0x7C00u, hi = NG > 1 && (w & 0x7C000000u) == 0x7C000000u;
          bad[g] = 0;
          if (__any(lo || hi)) {
            bad[g] = (unsigned)(__ballot(lo) & 0xFF) | (unsigned)(__ballot(hi) & 0xFF) << 8;
            w &= (lo ? 0xFFFF0000u : ~0u) & (hi ? 0xFFFFu : ~0u);
            flag = 3;
          }
          // tokens j and j + 2 side by side, one word per group, in the lanes of j = 0, 1, 4, 5
          const unsigned w2 = dppu<0xEE>(w);
          const unsigned p0 = __builtin_amdgcn_perm(w2, w, 0x05040100u), p1 = __builtin_amdgcn_perm(w2, w, 0x07060302u);
          const unsigned s0 = p0 & 0xFFF0FFF0u, s1 = p1 & 0xFFF0FFF0u;
          const unsigned m0 = (p0 & 0x000F000Fu) | 0xE400E400u, m1 = (p1 & 0x000F000Fu) | 0xE400E400u;
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const int at = (j >> 1) * 4 + (j & 1);
            scale[2 * g][j] = __builtin_amdgcn_readlane(s0, at);
            minus[2 * g][j] = __builtin_amdgcn_readlane(m0, at);
            if (NG > 1) {
              scale[NG > 1 ? 2 * g + 1 : 0][j] = __builtin_amdgcn_readlane(s1, at);
              minus[NG > 1 ? 2 * g + 1 : 0][j] = __builtin_amdgcn_readlane(m1, at);
            }
          }
        }
        unsigned out[2][4];
#pragma unroll
        for (int s = 0; s < 2; s++) {
          // the column's group: below D / 2, and D / 2 further
          const int g0 = DIM == 256 ? 2 * s : DIM == 128 ? s : 0, g1 = DIM == 256 ? 2 * s + 1 : g0;
#pragma unroll
          for (int j = 0; j < 2; j++)
#pragma unroll
            for (int q = 0; q < 2; q++) {
              const unsigned sc = DIM == 256 && (wave & 1) ? scale[g1][2 * j + q] : scale[g0][2 * j + q];
              const unsigned mi = DIM == 256 && (wave & 1) ? minus[g1][2 * j + q] : minus[g0][2 * j + q];
              out[s][2 * j + q] = pair(raw.codes[j] >> (4 * s + 8 * q), mi, sc);
            }
        }
        const int u = block * 2 + vhalf;
        if (vin) {
          *(v4u*)&vt[buf][vat(vcol, u)] = v4u{out[0][0], out[0][1], out[0][2], out[0][3]};
          *(v4u*)&vt[buf][vat(HALF + vcol, u)] = v4u{out[1][0], out[1][1], out[1][2], out[1][3]};
        }
        if (lane == 0) flags[buf][wave] = (uint8_t)flag;
        if (flag & 2 && lane < NG) {
          unsigned m = bad[0];
#pragma unroll
          for (int g = 1; g < (NG + 1) / 2; g++) m = lane >> 1 == g ? bad[g] : m;
          m = m >> (8 * (lane & 1)) & 0xFF;
          nans[buf][wave][lane] = (uint16_t)((m & 15) << (4 * vhalf) | (m >> 4) << (8 + 4 * vhalf));
        }
    };

    f32x16 S[NS];
    f16x8 B[PS];
    // The matrix products of a step: the last tile's weights times its values, and this tile's scores.
    auto values = [&](const _Float16* vb) {
#pragma unroll
      for (int k = 0; k < PS; k++)
#pragma unroll
        for (int c = 0; c < CT; c++) {
          const f16x8 A = *(const f16x8*)&vb[vat(c * 32 + l32, 2 * k + half)];
          O[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(A, B[k], O[c], 0, 0, 0);
        }
    };
    auto scores = [&](const _Float16* kb) {
#pragma unroll
      for (int s = 0; s < NS; s++) {
        const f32x16 zero = {};
#pragma unroll
        for (int k = 0; k < KS; k++) {
          const f16x8 A = *(const f16x8*)&kb[kat(s * 32 + l32, 2 * k + half)];
          S[s] = __builtin_amdgcn_mfma_f32_32x32x16_f16(A, Q[k], k ? S[s] : zero, 0, 0, 0);
        }
      }
    };
    // This tile's scores to weights.
    auto weights = [&](int buf, int tile) {
      const int tok0 = c0 + tile * TT;
      const v2u fl = *(const v2u*)flags[buf];
      const unsigned f0 = __builtin_amdgcn_readfirstlane(fl[0]), f1 = __builtin_amdgcn_readfirstlane(fl[1]);
      if (f0 != 0x01010101u || f1 != 0x01010101u || tok0 < all_from || tok0 + TT - 1 > all_to) {
        // the tile's tokens that this lane's row sees, a bit each
        const int from = max(least - tok0, 0), to = min(last - tok0, TT - 1);
        uint64_t there = 0;      // blocks that have a page
#pragma unroll
        for (int k = 0; k < PS; k++)
          if ((k * WB < 4 ? f0 >> (8 * k * WB) : f1 >> (8 * (k * WB - 4))) & 1) there |= 0xFFFFull << (16 * k);
        const uint64_t see = to < from ? 0 : there & (~0ull >> (63 - to)) & (~0ull << from);
        if ((f0 | f1) & 0x02020202u)      // a NaN among the values: for the rows that see it, in its group
          for (int g = 0; g < NG; g++) {
            uint64_t nan = 0;
            for (int w = 0; w < 8; w++)
              if ((w < 4 ? f0 >> (8 * w) : f1 >> (8 * (w - 4))) & 2) nan |= (uint64_t)nans[buf][w][g] << (16 * (w / WB));
            if (nan & see)
#pragma unroll
              for (int i = 0; i < NG; i++) poison[i] = i == g ? NAN : poison[i];
          }
#pragma unroll
        for (int s = 0; s < NS; s++) {
          const unsigned bits = (unsigned)(see >> (32 * s)) >> (4 * half);
#pragma unroll
          for (int i = 0; i < 16; i++) {
            const int m = (int)(bits << (31 - (8 * (i / 4) + i % 4))) >> 31;
            S[s][i] = __int_as_float((__float_as_int(S[s][i]) & m) | ((int)0xFF800000 & ~m));
          }
        }
      }
      float top = S[0][0];
#pragma unroll
      for (int s = 0; s < NS; s++)
#pragma unroll
        for (int i = 0; i < 16; i++) top = fmaxf(top, S[s][i]);
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * factor;
      if (__any(top > ref + TOP)) {
        const float to = fmaxf(ref, top - UP), keep = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - to);
        ref = to;
        l *= keep;
#pragma unroll
        for (int c = 0; c < CT; c++)
#pragma unroll
          for (int i = 0; i < 16; i++) O[c][i] *= keep;
      }
      const float at = ref == -INFINITY ? 0.f : ref;
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; s++)
#pragma unroll
        for (int i = 0; i < 16; i++) S[s][i] = fmaf(S[s][i], factor, -at);
#pragma unroll
      for (int k = 0; k < PS; k++) {
        const int s = k / 2, i0 = (k & 1) * 8;
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const int i = i0 + (j >> 1) * 4 + (j & 1);
          const float p0 = __builtin_amdgcn_exp2f(S[s][i]), p1 = __builtin_amdgcn_exp2f(S[s][i + 2]);
          sum[0] += p0;
          sum[1] += p1;
          B[k][2 * j] = (_Float16)p0;
          B[k][2 * j + 1] = (_Float16)p1;
        }
      }
      l += sum[0] + sum[1];
      __builtin_amdgcn_sched_barrier(0);      // the sums here, not beside the products: their registers
    };

    // Two groups of four waves, one of each on a SIMD.  Between two barriers the first turns its scores of tile n
    // into weights, converts its share of later tiles (K's n + 2, V's n + 1) and then runs the products of tile n; the
    // second first runs the products of tile n - 1 and then does the same for its scores of tile n.  So one group's
    // products run beside the other's vector work, and what is written between two barriers (K n + 2, V n + 1) is read
    // after the second one at the earliest, what is read (K n and n + 1, V n - 1 and n) is in the other two of three
    // buffers each.  With a second barrier between the halves 631 us for 607, 316 for 242 at 64 channels.
    KRaw kr;
    VRaw vr;
    int e1 = entry(1), e2 = entry(2), e = entry(0);
    const Place first = place_at(0, e);
    load_k(kr, 0, first);
    load_v(vr, 0, first);
    e = entry(3);
    Place vplace = place_at(1, e1), kplace = place_at(2, e2);
    {
      KRaw k1;
      load_k(k1, 1, vplace);
      convert_k(0, kr);
      convert_v(0, 0, first.there, vr);
      load_v(vr, 1, vplace);
      load_k(kr, 2, kplace);
      convert_k(1, k1);
    }
    __syncthreads();
    if (wave >= 4) __syncthreads();
    int b0 = 0, b1 = 1, b2 = 2;      // buffers of tiles n, n + 1, n + 2 (and n - 1)
    scores(kt[0]);
    for (int n = 0;; n++) {
      __builtin_amdgcn_s_setprio(0);
      if (wave < 4) __syncthreads();
      weights(b0, n);
      convert_k(b2, kr);
      convert_v(b1, n + 1, vplace.there, vr);
      __builtin_amdgcn_sched_barrier(0);      // into the registers that these have left
      load_v(vr, n + 2, kplace);
      vplace = kplace;
      kplace = place_at(n + 3, e);
      load_k(kr, n + 3, kplace);
      e = entry(n + 4);
      if (wave >= 4) __syncthreads();
      __builtin_amdgcn_s_setprio(1);
      values(vt[b0]);
      scores(kt[b1]);      // of no tile after the last one: not used then
      // LDS operands AHEAD products ahead
      __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
      for (int i = 0; i < PS * CT + NS * KS - AHEAD; i++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
      if (n + 1 >= ntiles) break;
      const int b = b0;
      b0 = b1;
      b1 = b2;
      b2 = b;
    }
    __builtin_amdgcn_s_setprio(0);
    if (wave < 4) __syncthreads();
    __syncthreads();      // the next row block's tiles may be written

    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (factor == BAD && l > 0.f) l = NAN;      // some token is seen
#pragma unroll
    for (int g = 0; g < NG; g++) poison[g] += __shfl_xor(poison[g], 32);
    if (row < R.rows) {
      const bool whole = !turn.part, none = l == 0.f;
      const float by = whole ? none ? 0.f : 1.f / l : 1.f;
      float* part = turn.part + (wave * 32 + l32) * (DIM + 4);
#pragma unroll
      for (int c = 0; c < CT; c++)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const int d = c * 32 + 2 * i + 4 * half;
          float o[4];
#pragma unroll
          for (int j = 0; j < 4; j++) o[j] = (O[c][i + j] + poison[c / 2]) * by;
          if (!whole) *(f32x4*)(part + d) = f32x4{o[0], o[1], o[2], o[3]};
          else {
            v2u w;
#pragma unroll
            for (int j = 0; j < 2; j++)
              w[j] = (unsigned)__builtin_bit_cast(uint16_t, Elem<DT>::store(o[2 * j])) |
                     (unsigned)__builtin_bit_cast(uint16_t, Elem<DT>::store(o[2 * j + 1])) << 16;
            *(v2u_any*)((T*)a.out + to * DIM + d) = w;
          }
        }
      if (whole && a.lse && !half) a.lse[to] = none ? -INFINITY : lse_of<ROWS>(ref, l);
      if (!whole && !half) {
        part[DIM] = ref;
        part[DIM + 1] = l;
      }
    }
    if (!walk_on<ROWS>(a, W, turn)) return;
  }
}

// Joins the parts of the row blocks that several workgroups share: a row's four
// channels a thread, and SL threads of every SL-th part each for a row of more
// than four parts, joined in LDS.  An item is as many rows as 256 threads hold;
// each workgroup finds all row blocks that have parts and takes its stretch of
// their items, since a workgroup for every possible one costs more than the
// join itself (8192 of them take 20 us to end at once).
constexpr int MAX_GROUPS = 768;
template <int DIM, int ROWS>
__global__ __launch_bounds__(256) void k_attention_join(AttnArgs a, int groups) {
  constexpr int TH = DIM / 4, GR = 256 / TH, B = 4, EACH = MAX_GROUPS / 256;
  __shared__ int ends[MAX_GROUPS], waves[4];
  __shared__ f32x4 acc[GR][TH];
  __shared__ float tops[GR], sums[GR];
  const int tid = threadIdx.x, g = tid / TH, c = tid % TH;
  const auto slices = [](int n) {
    int s = 1;
    while (s < GR && 4 * s < n) s *= 2;
    return s;
  };
  int count[EACH], mine = 0;
#pragma unroll
  for (int i = 0; i < EACH; i++) {
    const int at = tid * EACH + i;
    count[i] = 0;
    if (at < groups) {
      const AttnShare sh = a.shares[at];
      const int per = GR / slices(sh.count);
      if (sh.count >= 2) count[i] = (min(ROWS, sh.rows - sh.r0) + per - 1) / per;
    }
    mine += count[i];
  }
  int to = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(to, d);
    if ((tid & 63) >= d) to += o;
  }
  if ((tid & 63) == 63) waves[tid >> 6] = to;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (i < tid >> 6) to += waves[i];
    total += waves[i];
  }
  to -= mine;
#pragma unroll
  for (int i = 0; i < EACH; i++) ends[tid * EACH + i] = to += count[i];
  __syncthreads();

  int item = (int)((int64_t)total * blockIdx.x / gridDim.x);
  const int last = (int)((int64_t)total * (blockIdx.x + 1) / gridDim.x);
  if (item >= last) return;
  int first = 0;      // the first row block that ends past `item`
  for (int hi = groups - 1; first < hi;) {
    const int mid = (first + hi) >> 1;
    if (ends[mid] > item) hi = mid; else first = mid + 1;
  }
  for (; item < last; item++) {
    while (ends[first] <= item) first++;
    const AttnShare sh = a.shares[first];
    const int n = sh.count, SL = slices(n), per = GR / SL, s = g / per;
    const int r = (item - (first ? ends[first - 1] : 0)) * per + g % per, row = sh.r0 + r;
    const bool in = r < ROWS && row < sh.rows;
    // a row block's first part is its workgroup's last, its others their workgroups' first
    const auto part = [&](int p) {
      return a.part + ((int64_t)(p ? 2 * (first + p) : 2 * first + 1) * ROWS + r) * (DIM + 4);
    };
    float top = -INFINITY, sum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    const auto add = [&](float m, float l, const f32x4& x) {
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
      sum = fmaf(l, f, sum);
#pragma unroll
      for (int j = 0; j < 4; j++) o[j] = fmaf(x[j], f, o[j]);
    };
    if (in)
      for (int p0 = s; p0 < n; p0 += B * SL) {
        f32x4 x[B];
        float m[B], l[B];
#pragma unroll
        for (int i = 0; i < B; i++) {
          const float* p = part(min(p0 + i * SL, n - 1));
          m[i] = p[DIM];
          l[i] = p[DIM + 1];
          x[i] = *(const f32x4*)(p + 4 * c);
        }
        const float was = top;
#pragma unroll
        for (int i = 0; i < B; i++)
          if (p0 + i * SL < n) top = fmaxf(top, m[i]);
        const float keep = was == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(was - top);
        if (p0 != s) {
          sum *= keep;
#pragma unroll
          for (int j = 0; j < 4; j++) o[j] *= keep;
        }
#pragma unroll
        for (int i = 0; i < B; i++)
          if (p0 + i * SL < n) add(m[i], l[i], x[i]);
      }
    if (SL > 1) {
      acc[g][c] = o;
      if (c == 0) {
        tops[g] = top;
        sums[g] = sum;
      }
      __syncthreads();
      if (s == 0) {
        for (int i = 1; i < SL; i++) top = fmaxf(top, tops[i * per + g]);
        const f32x4 x = o;
        const float l = sum;
        sum = 0.f;
        o = f32x4{0.f, 0.f, 0.f, 0.f};
        add(tops[g], l, x);
        for (int i = 1; i < SL; i++) add(tops[i * per + g], sums[i * per + g], acc[i * per + g][c]);
      }
      __syncthreads();      // before the next item's
    }
    if (s || !in) continue;
    const bool none = sum == 0.f;
    const int64_t at = (sh.t0 + row / a.each) * a.heads_q + sh.h * a.each + row % a.each;
#pragma unroll
    for (int j = 0; j < 4; j++) store_any(a.out, at * DIM + 4 * c + j, none ? 0.f : o[j] / sum, a.dtype);
    if (a.lse && c == 0) a.lse[at] = none ? -INFINITY : lse_of<ROWS>(top, sum);
  }
}
template <int DIM, int ROWS>
static void launch_join(const AttnArgs& a, int groups, hipStream_t s) {
  const int items = (groups * ROWS + 1024 / DIM - 1) / (1024 / DIM);
  k_attention_join<DIM, ROWS><<<items < 1024 ? items : 1024, 256, 0, s>>>(a, groups);
}

// k_attention_chunk takes a call whose sequences have about this many rows a
// cache head and whose work (query heads x tokens x (tiles + 4)) is enough.  4
// sequences of 8001, chunk against split in us: 64 rows 51 / 59, 40 rows 56 /
// 52 (128 channels); 96 rows 53 / 60, 64 rows 46 / 42 (64); 128 rows 159 / 199,
// 64 rows 136 / 105 (256).  One of 1500 with 512 rows (114 K) 39 / 54, one of
// 128 with 512 rows (24 K) 21 / 17.
static bool chunk_pays(int dim, int64_t rows, int64_t work) { return rows >= (dim == 128 ? 48 : 96) && work >= 65536; }
// Up to this many tiles a workgroup takes a whole row block and cache head, and
// nothing is joined; fewer where that leaves most of the chip idle (256 tokens
// after 768: 50 us, shared by all 42; 512 tokens after none: 35, shared 41).
constexpr int WHOLE_TILES = 16, WHOLE_TILES_FEW = 8, FEW = 128;

struct Plan {
  int rows;                  // of a row block: 4 (k_attention_split) or 256 (k_attention_chunk)
  int whole, blocks, groups; // AttnArgs::whole, ::blocks; workgroups
};
// One workgroup per row block and cache head where lengths are short; else as
// many as are resident at once (a CU holds three of four waves where 168
// registers do, two elsewhere, one of eight for k_attention_chunk), but not
// below four tiles each: a part costs its join about that much.
static bool attention_plan(int heads_q, int heads_kv, int dim, int dtype, int64_t tokens, int batch, bool starts,
                           int64_t max_new, int64_t max_len, Plan* p) {
  const int each = heads_q / heads_kv;
  const int64_t tiles = max_len > 0 && max_len < 1 << 26 ? (max_len + 63) / 64 : 1 << 20;
  p->rows = dtype != EXTERND_F32 && chunk_pays(dim, max_new * each, tokens * heads_q * (tiles + 4)) ? 256 : 4;
  const int64_t blocks = starts ? tokens * each / p->rows + batch : (int64_t)batch * ((each + p->rows - 1) / p->rows);
  if (blocks * heads_kv > INT32_MAX) return false;
  p->blocks = (int)blocks;
  p->whole = tiles <= (p->rows == 256 && blocks * heads_kv < FEW ? WHOLE_TILES_FEW : WHOLE_TILES) &&
             blocks * heads_kv <= MAX_THREADS / 512;
  if (p->whole) {
    p->groups = (int)(blocks * heads_kv);
    return true;
  }
  static_assert(MAX_GROUPS >= 768, "the join looks at as many shares");
  const int64_t most = p->rows == 256 ? 256 : dim <= 128 ? 768 : 512;
  const int64_t fit = (blocks * heads_kv * tiles + 3) / 4;
  p->groups = (int)(most < fit ? most : fit);
  return true;
}
static size_t plan_bytes(const Plan& p, int dim) {
  if (p.whole) return 0;
  return ((size_t)p.groups * (2 * p.rows * (dim + 4) * sizeof(float) + sizeof(AttnShare)) + 255) & ~(size_t)255;
}

template <int DIM>
static void launch_attention(const AttnArgs& a, const Plan& p, hipStream_t s) {
  if (p.rows == 4) {
    if (a.dtype == EXTERND_F32) k_attention_split<DIM, true><<<p.groups, 256, 0, s>>>(a);
    else k_attention_split<DIM, false><<<p.groups, 256, 0, s>>>(a);
    if (!a.whole) launch_join<DIM, 4>(a, p.groups, s);
  } else {
    if (a.dtype == EXTERND_BF16) k_attention_chunk<DIM, EXTERND_BF16><<<p.groups, 512, 0, s>>>(a);
    else k_attention_chunk<DIM, EXTERND_F16><<<p.groups, 512, 0, s>>>(a);
    if (!a.whole) launch_join<DIM, 256>(a, p.groups, s);
  }
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
  Plan p;
  // either form of the call (starts or none) fits
  size_t most = 0;
  for (int starts = 0; starts < 2; starts++) {
    if (!attention_plan(heads_q, heads_kv, head_dim, dtype, tokens, batch, starts, max_new, max_len, &p)) return 0;
    const size_t n = plan_bytes(p, head_dim);
    most = n > most ? n : most;
  }
  return most;
}

int32_t externd_kv4_attention_block_rows(int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t dtype,
                                         int64_t tokens, int32_t batch, int32_t max_new, int64_t max_len) {
  Plan p;
  if (!attention_sizes_ok(heads_q, heads_kv, head_dim, dtype, tokens, batch, max_new, max_len) ||
      !attention_plan(heads_q, heads_kv, head_dim, dtype, tokens, batch, true, max_new, max_len, &p))
    return 0;
  return p.rows;      // the same with and without starts
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
  // rows of a sequence are counted in whole blocks of 256, and the units of a row block over all cache heads
  if (tokens > INT32_MAX || tokens * heads_q > INT32_MAX - 1024 || batch > 65535 || heads_q > 65535 || table_pages > INT32_MAX)
    return EXTERND_EUNSUPPORTED;
  const int64_t room = table_pages * page_tokens < INT32_MAX ? table_pages * page_tokens : INT32_MAX;
  if ((room / 64 + 16) * heads_kv > INT32_MAX) return EXTERND_EUNSUPPORTED;
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
  a.dtype = dtype;
  a.q_vec = rows_aligned(q, q_token_stride, q_head_stride, dtype_bytes(dtype));
  Plan p;
  if (!attention_plan(heads_q, heads_kv, head_dim, dtype, tokens, batch, starts != nullptr, max_new, max_len, &p))
    return EXTERND_EUNSUPPORTED;
  a.whole = p.whole;
  a.blocks = p.blocks;
  a.part = (float*)workspace;
  a.shares = p.whole ? nullptr : (AttnShare*)(a.part + (size_t)p.groups * 2 * p.rows * (head_dim + 4));
  const hipStream_t s = (hipStream_t)stream;
  if (head_dim == 64) launch_attention<64>(a, p, s);
  else if (head_dim == 128) launch_attention<128>(a, p, s);
  else launch_attention<256>(a, p, s);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
