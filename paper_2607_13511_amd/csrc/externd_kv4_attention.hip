// Attention over the cache in 4 bits.
#include <math.h>

#include "externd_decode.hpp"

namespace externd {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

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
  int nsplit, chunk;      // parts of a sequence (grid x), and the least tokens of a part (a multiple of 256)
  int row_blocks;         // row blocks a launch starts per sequence and cache head
  float* part;            // per (row, part): DIM sums, then the maximum and the sum of weights
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

// The queries of one sequence and cache head are rows: row r is new token
// r / each, query head r % each of the cache head.  A row block (ROWS rows)
// sees the tokens lo .. hi - 1 among it, in `parts` parts of `part` tokens.
struct RowBlock {
  int64_t t0;          // first new token of the sequence
  int rows, first;     // rows of the sequence; position of its first new token
  int lo, hi, part, parts;
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
  const int r0 = rb * ROWS, r1 = min(r.rows, r0 + ROWS) - 1;
  r.hi = min(held, r.first + (r1 < 0 ? 0 : r1 / a.each) + 1);
  r.lo = a.window > 0 ? max(0, r.first + r0 / a.each - a.window + 1) & ~63 : 0;
  const int total = max(0, r.hi - r.lo);
  const int each = (total + a.nsplit - 1) / a.nsplit;
  r.part = max(a.chunk, (each + 255) & ~255);
  r.parts = (total + r.part - 1) / r.part;
  return r;
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

__device__ __forceinline__ float scale_of(unsigned word) {
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(word & 0xFFF0u));
}

// Four signed base-256 digits of a whole number below 2^31 - 2^23, lowest first.
__device__ __forceinline__ unsigned digits_of(int u) { return ((unsigned)u + 0x00808080u) ^ 0x00808080u; }

// Attention of up to 4 RT rows over one part of a sequence, by integer matrix
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
// Four waves share a part; each takes every fourth tile of 64 tokens with its
// own running maximum, and they are joined at the end.
template <int DIM, int RT, bool FINE>
__global__ __launch_bounds__(256, DIM * RT <= 128 ? 3 : 2) void k_attention_split(AttnArgs a) {
  constexpr int NG = DIM / KV4_GROUP, HALF = DIM / 2, ROWS = 4 * RT;
  constexpr int NU = DIM == 256 ? 2 : 1;     // 16-byte K loads of a lane and token
  constexpr int NC = DIM / 32;               // 16-byte V loads of a lane: 16 byte columns each
  constexpr int QROW = 80, PROW = 80;        // bytes of a digit row of 64 in LDS (padded against bank conflicts)
  constexpr int ACC = DIM + 4;               // floats of a row when waves join
  constexpr int SHARED_Q = RT * NG * 16 * QROW, SHARED_P = 4 * NG * (16 * PROW + 64), SHARED_O = 4 * ROWS * ACC * 4;
  constexpr int SHARED = SHARED_Q + SHARED_P > SHARED_O ? SHARED_Q + SHARED_P : SHARED_O;
  __shared__ __align__(16) uint8_t lds[SHARED];
  __shared__ float row_factor[ROWS];
  __shared__ int row_sums[ROWS][NG][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, seg = lane >> 4;
  const int b = blockIdx.z, h = blockIdx.y % a.c.heads;
  const int P = 1 << a.c.page_log2;

  for (int rb = blockIdx.y / a.c.heads;; rb += a.row_blocks) {
    const RowBlock R = row_block<ROWS>(a, b, rb);
    if (rb * ROWS >= R.rows) break;
    const int sp = blockIdx.x;
    if (R.parts == 0 && sp == 0) {      // rows that see nothing
      for (int i = threadIdx.x; i < ROWS * DIM; i += 256) {
        const int r = rb * ROWS + i / DIM;
        if (r >= R.rows) break;
        const int64_t o = (R.t0 + r / a.each) * a.heads_q + h * a.each + r % a.each;
        store_any(a.out, o * DIM + i % DIM, 0.f, a.dtype);
        if (a.lse && i % DIM == 0) a.lse[o] = -INFINITY;
      }
    }
    if (sp >= R.parts) continue;
    const int c0 = R.lo + sp * R.part, c1 = (int)min((int64_t)R.hi, (int64_t)c0 + R.part);

    // ---- the rows' digits, one wave per row ----
    for (int r = wave; r < ROWS; r += 4) {
      const int row = rb * ROWS + r;
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
        uint8_t* to = lds + (((r >> 2) * NG + g) * 16 + (r & 3) * 4) * QROW + slot;
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
    v4i Q[RT][NG];
    float factor[RT], m[RT], l[RT];
    int qhi[RT][NG], qlo[RT][NG], last[RT], least[RT];
    float O[RT][2 * NC], poison[RT][NG];
#pragma unroll
    for (int p = 0; p < RT; p++) {
      const int r = p * 4 + seg, row = rb * ROWS + r;
#pragma unroll
      for (int g = 0; g < NG; g++) {
        Q[p][g] = *(const v4i*)(lds + ((p * NG + g) * 16 + l16) * QROW + seg * 16);
        qhi[p][g] = row_sums[r][g][0];
        qlo[p][g] = row_sums[r][g][1];
        poison[p][g] = 0.f;
      }
      factor[p] = row_factor[r];
      m[p] = -INFINITY;
      l[p] = 0.f;
      const int pos = R.first + row / a.each;
      last[p] = row < R.rows ? min(pos, c1 - 1) : -1;
      least[p] = a.window > 0 ? pos - a.window + 1 : 0;
#pragma unroll
      for (int i = 0; i < 2 * NC; i++) O[p][i] = 0.f;
    }
    uint8_t* const pbuf = lds + SHARED_Q + wave * (NG * (16 * PROW + 64));
    uint8_t* const zbuf = pbuf + NG * 16 * PROW;

    const int ntiles = (c1 - c0 + 63) >> 6;
    constexpr int NW = NG == 1 ? 1 : NG / 2;    // 32-bit loads of a token's K words (V's likewise; one for both at 64)
    v4u kr[4][NU], vr[NC];
    unsigned kw[4][NW], vw[4][NW];
    unsigned ok = 0;        // bit t: block t of the tile has a page
    // page of this lane's block (seg) of a tile, or -1
    auto lookup = [&](int tile) -> int {
      const int tok = c0 + tile * 64 + seg * 16;
      if (tile >= ntiles || tok >= c1) return -1;
      const int page = a.s.table[(int64_t)b * a.s.table_pages + (tok >> a.c.page_log2)];
      return page >= 0 && page < a.c.num_pages ? page : -1;
    };
    auto base_of = [&](uint64_t off, int t) -> const uint8_t* {
      const unsigned lo = __builtin_amdgcn_readlane((unsigned)off, 16 * t);
      const unsigned hi = __builtin_amdgcn_readlane((unsigned)(off >> 32), 16 * t);
      return a.cache + ((uint64_t)hi << 32 | lo);
    };
    auto offset_of = [&](int page) -> uint64_t {
      return (uint64_t)((int64_t)max(page, 0) * a.c.heads + h) * (uint64_t)a.c.head_bytes;
    };
    auto load_k = [&](int tile, int page) {
      const uint64_t off = offset_of(page);
#pragma unroll
      for (int t = 0; t < 4; t++) {
        const uint8_t* base = base_of(off, t);
        const unsigned o = (unsigned)((c0 + tile * 64 + 16 * t) & (P - 1)) + l16;
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
    auto load_v = [&](int tile, int page) {
      const uint64_t off = offset_of(page);
      const int tok = c0 + tile * 64;
      ok = 0;
#pragma unroll
      for (int t = 0; t < 4; t++) {
        if constexpr (NG > 1) {
          const unsigned o = (unsigned)((tok + 16 * t) & (P - 1)) + l16;
          const unsigned* wp = (const unsigned*)(base_of(off, t) + (unsigned)P * DIM + o * (4 * NG)) + NW;
#pragma unroll
          for (int g = 0; g < NW; g++) vw[t][g] = wp[g];
        }
        ok |= (unsigned)(__builtin_amdgcn_readlane(page, 16 * t) >= 0) << t;
      }
      const uint8_t* vp = a.cache + off + (unsigned)P * HALF + ((unsigned)((tok + 16 * seg) & (P - 1)) >> 4) * (HALF * 16) + l16 * 16;
#pragma unroll
      for (int c = 0; c < NC; c++) vr[c] = *(const v4u*)(vp + c * 256);
    };
    auto k_word = [&](int t, int g) -> unsigned { return g & 1 ? kw[t][g / 2] >> 16 : kw[t][g / 2] & 0xFFFFu; };
    auto v_word = [&](int t, int g) -> unsigned {
      if (NG == 1) return vw[t][0] >> 16;
      return g & 1 ? vw[t][g / 2] >> 16 : vw[t][g / 2] & 0xFFFFu;
    };

    // One tile: K's registers are free once the scores are there and take the
    // next tile's K then; V's likewise at the end.
    auto compute = [&](int tile, int next_page) {
      const int tok = c0 + tile * 64 + l16;
      const v4i zero = {0, 0, 0, 0};
      float x[RT][4];
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
#pragma unroll
        for (int p = 0; p < RT; p++) {
          float sum = 0.f;
#pragma unroll
          for (int g = 0; g < NG; g++) {
            const unsigned word = k_word(t, g);
            const v4i r = __builtin_amdgcn_mfma_i32_16x16x64_i8(Q[p][g], kop[g], zero, 0, 0, 0);
            const int z = (int)(word & 15);
            const int hi = (r[3] << 8) + r[2] - __mul24(z, qhi[p][g]);
            const int lo = (r[1] << 8) + r[0] - __mul24(z, qlo[p][g]);
            sum = fmaf(scale_of(word), fmaf((float)hi, 65536.f, (float)lo), sum);
          }
          x[p][t] = sum * factor[p];
        }
        if constexpr (RT * NG >= 4) __builtin_amdgcn_sched_barrier(0);      // one block's registers at a time
      }
      if constexpr (NG == 1) {
#pragma unroll
        for (int t = 0; t < 4; t++) vw[t][0] = kw[t][0];
      }
      const bool more = tile + 4 < ntiles;
      if (more) load_k(tile + 4, next_page);
      // ---- zero points of the values, negated, for the accumulators' start ----
#pragma unroll
      for (int t = 0; t < 4; t++)
#pragma unroll
        for (int g = 0; g < NG; g++)
          zbuf[g * 64 + 16 * t + l16] = (uint8_t)(0u - (v_word(t, g) & 15));
#pragma unroll
      for (int p = 0; p < RT; p++) {
        // ---- softmax weights of this lane's row and tokens ----
        bool seen[4];
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; t++) {
          const int pos = tok + 16 * t;
          seen[t] = (ok >> t & 1) && pos <= last[p] && pos >= least[p];
          x[p][t] = seen[t] ? x[p][t] : -INFINITY;
          top = fmaxf(top, x[p][t]);
        }
        const float mn = fmaxf(m[p], row_max(top)), at = mn == -INFINITY ? 0.f : mn;
        const float keep = __builtin_amdgcn_exp2f(m[p] - at);
        m[p] = mn;
        float w[4];
        l[p] *= keep;
#pragma unroll
        for (int t = 0; t < 4; t++) {
          w[t] = __builtin_amdgcn_exp2f(x[p][t] - at);
          l[p] += w[t];
        }
        // ---- times the values' scales, as whole numbers of the tile's largest, four digits ----
        float ws[NG][4];
#pragma unroll
        for (int g = 0; g < NG; g++)
#pragma unroll
          for (int t = 0; t < 4; t++) {
            ws[g][t] = seen[t] ? w[t] * scale_of(v_word(t, g)) : 0.f;
            poison[p][g] = fmaf(ws[g][t], 0.f, poison[p][g]);
          }
#pragma unroll
        for (int c = 0; c < 2 * NC; c++) O[p][c] *= keep;
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
            O[p][c] = fmaf(f0, back[glo], O[p][c]);
            O[p][NC + c] = fmaf(f1, back[ghi], O[p][NC + c]);
          }
          // 16-bit results end here: what is left is below 2^-30 of the tile's largest weight.  fp32 results keep
          // every weight's own 24 bits: again with what is left (twice in all where no weight is below 2^-37), until
          // that is below the smallest normal number.  A round leaves less than 2^-29 of the largest weight, or
          // less than 2^-126: weights are at most 4352, so six rounds at most.
          // masks anew each time: kept, they cost 32 registers
          if (FINE || RT > 1)
#pragma unroll
            for (int c = 0; c < NC; c++) asm volatile("" : "+v"(vr[c]));
          if (!FINE || !__any(left >= 1.17549435e-38f)) break;
        }
        if constexpr (RT > 1) __builtin_amdgcn_sched_barrier(0);      // one row tile's registers at a time
      }
      if (more) load_v(tile + 4, next_page);
    };

    int page = lookup(wave);
    if (wave < ntiles) {
      load_k(wave, page);
      load_v(wave, page);
    }
    page = lookup(wave + 4);
    for (int tile = wave; tile < ntiles; tile += 4) {
      const int after = lookup(tile + 8);
      compute(tile, page);
      page = after;
    }

    // ---- join the four waves: lane (row, channel) sums of each, then by the row's maximum ----
    __syncthreads();
    float* const acc = (float*)lds;
#pragma unroll
    for (int p = 0; p < RT; p++) {
      const int r = p * 4 + seg;
      float* o = acc + (wave * ROWS + r) * ACC;
      const float sum = row_sum(l[p]);
#pragma unroll
      for (int c = 0; c < NC; c++) {
        const int glo = c / 4, ghi = DIM == 64 ? 0 : NG / 2 + c / 4;
        o[16 * c + l16] = O[p][c] + row_sum(poison[p][glo]);
        o[HALF + 16 * c + l16] = O[p][NC + c] + row_sum(poison[p][ghi]);
      }
      if (l16 == 0) {
        o[DIM] = m[p];
        o[DIM + 1] = sum;
      }
    }
    __syncthreads();
    const bool whole = R.parts == 1;
    for (int i = threadIdx.x; i < ROWS * DIM; i += 256) {
      const int r = i / DIM, d = i % DIM, row = rb * ROWS + r;
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
      if (whole) {
        const bool none = sum == 0.f;
        store_any(a.out, to * DIM + d, none ? 0.f : o / sum, a.dtype);
        if (a.lse && d == 0) a.lse[to] = none ? -INFINITY : (top + log2f(sum)) * 0.69314718055994530942f;
      } else {
        float* part = a.part + (to * a.nsplit + sp) * (DIM + 2);
        part[d] = o;
        if (d == 0) {
          part[DIM] = top;
          part[DIM + 1] = sum;
        }
      }
    }
    __syncthreads();
  }
}

// Joins the parts of a row: one workgroup of DIM threads per new token and
// query head.
template <int DIM, int ROWS>
__global__ __launch_bounds__(DIM) void k_attention_join(AttnArgs a) {
  const int64_t t = blockIdx.x;
  const int hq = blockIdx.y, d = threadIdx.x;
  const int b = sequence_of(a.s, t);
  const int64_t t0 = a.s.starts ? a.s.starts[b] : b;
  const int row = (int)(t - t0) * a.each + hq % a.each;
  if (row < 0) return;
  const RowBlock R = row_block<ROWS>(a, b, row / ROWS);
  if (R.parts < 2) return;      // written by k_attention_split
  const int64_t to = t * a.heads_q + hq;
  const float* part = a.part + to * a.nsplit * (DIM + 2);
  float top = -INFINITY;
  for (int p = 0; p < R.parts; p++) top = fmaxf(top, part[p * (DIM + 2) + DIM]);
  const float at = top == -INFINITY ? 0.f : top;
  float o = 0.f, sum = 0.f;
  for (int p = 0; p < R.parts; p++) {
    const float f = __builtin_amdgcn_exp2f(part[p * (DIM + 2) + DIM] - at);
    o = fmaf(part[p * (DIM + 2) + d], f, o);
    sum = fmaf(part[p * (DIM + 2) + DIM + 1], f, sum);
  }
  const bool none = sum == 0.f;
  store_any(a.out, to * DIM + d, none ? 0.f : o / sum, a.dtype);
  if (a.lse && d == 0) a.lse[to] = none ? -INFINITY : (top + log2f(sum)) * 0.69314718055994530942f;
}

// Row tiles of four that a workgroup takes (registers allow two at 256 channels).
static int row_tiles(int rows, int dim) { return rows <= 4 ? 1 : rows <= 8 || dim == 256 ? 2 : 4; }

struct SplitPlan {
  int rt, row_blocks, nsplit, chunk;
};
// Parts of about equal size: enough workgroups to fill the chip (two of four
// waves a CU resident, in one pass), a part no shorter than four waves' tile each.
static SplitPlan split_plan(int each, int heads_kv, int dim, int batch, int64_t max_new, int64_t max_len) {
  SplitPlan p;
  const int64_t rows = max_new * each;
  p.rt = row_tiles((int)(rows > 64 ? 64 : rows), dim);
  const int64_t blocks = (rows + 4 * p.rt - 1) / (4 * p.rt);
  p.row_blocks = (int)(blocks > 16384 / heads_kv ? (16384 / heads_kv > 0 ? 16384 / heads_kv : 1) : blocks);
  const int64_t units = (int64_t)batch * heads_kv * p.row_blocks;
  const int64_t len = max_len < 1 ? 65536 : max_len;
  int64_t n = (512 + units - 1) / units;
  const int64_t most = (len + 255) / 256;
  n = n > most ? most : n;
  n = n > 256 ? 256 : n < 1 ? 1 : n;
  int64_t chunk = ((len + n - 1) / n + 255) & ~(int64_t)255;
  if (chunk > (1 << 30)) chunk = 1 << 30;
  p.chunk = (int)chunk;
  p.nsplit = (int)((len + chunk - 1) / chunk);
  if (p.nsplit < 1) p.nsplit = 1;
  return p;
}

template <int DIM, int RT>
static void launch_split(const AttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.nsplit, (unsigned)(a.c.heads * a.row_blocks), (unsigned)a.s.batch);
  if (a.dtype == EXTERND_F32) k_attention_split<DIM, RT, true><<<grid, 256, 0, s>>>(a);
  else k_attention_split<DIM, RT, false><<<grid, 256, 0, s>>>(a);
  if (a.nsplit > 1)
    k_attention_join<DIM, 4 * RT><<<dim3((unsigned)a.s.tokens, (unsigned)a.heads_q), DIM, 0, s>>>(a);
}
template <int DIM>
static void launch_split(const AttnArgs& a, int rt, hipStream_t s) {
  if (rt == 1) launch_split<DIM, 1>(a, s);
  else if (rt == 2) launch_split<DIM, 2>(a, s);
  else if constexpr (DIM != 256) launch_split<DIM, 4>(a, s);
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
  const SplitPlan p = split_plan(heads_q / heads_kv, heads_kv, head_dim, batch, max_new, max_len);
  if (p.nsplit == 1) return 0;
  return ((size_t)tokens * heads_q * p.nsplit * (head_dim + 2) * 4 + 255) & ~(size_t)255;
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
  if (tokens > INT32_MAX || tokens * heads_q > INT32_MAX || batch > 65535 || heads_q > 65535 || table_pages > INT32_MAX) return EXTERND_EUNSUPPORTED;
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
  const SplitPlan p = split_plan(a.each, heads_kv, head_dim, batch, max_new, max_len);
  a.nsplit = p.nsplit;
  a.chunk = p.chunk;
  a.row_blocks = p.row_blocks;
  a.part = (float*)workspace;
  const hipStream_t s = (hipStream_t)stream;
  if (head_dim == 64) launch_split<64>(a, p.rt, s);
  else if (head_dim == 128) launch_split<128>(a, p.rt, s);
  else launch_split<256>(a, p.rt, s);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
