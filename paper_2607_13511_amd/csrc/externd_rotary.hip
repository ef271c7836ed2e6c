// Rotary positions: every pair (a, b) of a head's first rot_dim entries is
// turned by its token's position times the pair's frequency.
#include <math.h>

#include "externd_decode.hpp"

namespace externd {

struct RotarySide {
  const void* in;
  void* out;
  int64_t its, ihs, ots, ohs;   // token and head strides of in and out, in elements
  int heads;
};
struct RotaryArgs {
  RotarySide side[2];
  const int64_t* positions;
  const uint64_t* freqs;
  int64_t tokens;
  int dim, rot, interleaved;
  float amplitude, sign;
};

// sin and cos of a phase in units of 2^-64 turns.  The phase is cut to 2^-32
// turns (1.5e-9 radians), reduced to the nearest quarter turn in whole
// numbers, and the rest, at most pi / 4, goes through the Taylor sums (the
// terms left out are below 2e-9).
__device__ __forceinline__ void sincos_turns(uint64_t phase, float* s, float* c) {
  const unsigned t = (unsigned)(phase >> 32);
  const unsigned quarter = (t + 0x20000000u) >> 30;
  const float x = (float)(int)(t - (quarter << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
  const float x2 = x * x;
  const float sn = x * fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
  const float cs = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24),
                                 -0.5f), 1.f);
  const float u = quarter & 1 ? cs : sn, v = quarter & 1 ? sn : cs;
  *s = quarter & 2 ? -u : u;
  *c = (quarter + 1) & 2 ? -v : v;
}

// One form for all variants of the kernel, so that they agree bit for bit: a
// fused multiply-add in fp32, not fused with the rounding to the storage type.
__device__ __forceinline__ float turned(float a, float c, float b, float s) {
  float r = fmaf(a, c, b * s);
  asm("" : "+v"(r));
  return r;
}

// A workgroup takes TW tokens and `span` heads of q and k side by side: sin and
// cos of its tokens' pairs once, in LDS, then units of N entries (of both
// partners, N each), the unit index running through a head first.  Bound by
// memory: 8191 tokens of 40 heads of 128 in bf16, 168 MB, in 32 us (5.2 TB/s)
// where all of a head is turned, 37 us where half of it is.
template <int DT, int N, bool VEC>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a, int tw, int span) {
  typedef typename Elem<DT>::T T;
  extern __shared__ float2 turn[];      // tw x rot / 2: cos, sin
  const int half = a.rot / 2, heads = a.side[0].heads + a.side[1].heads;
  const int64_t t0 = (int64_t)blockIdx.x * tw;
  const int nt = (int)min((int64_t)tw, a.tokens - t0);
  const int h0 = blockIdx.y * span, nh = min(span, heads - h0);
  for (int e = threadIdx.x; e < nt * half; e += 256) {
    const int t = e / half;
    float s, c;
    sincos_turns((uint64_t)a.positions[t0 + t] * a.freqs[e - t * half], &s, &c);
    turn[e] = make_float2(c * a.amplitude, s * a.sign * a.amplitude);
  }
  __syncthreads();
  const int pairs = (a.interleaved ? a.rot : half) / N;      // units that turn
  constexpr int RN = VEC ? N : 1;      // entries of a unit that is only copied
  const int units = pairs + (a.dim - a.rot) / RN;
  const int total = nt * nh * units;
  const float by_units = 1.f / units, by_heads = 1.f / nh;
  constexpr int U = VEC ? 2 : 1;      // units of a thread in flight (8191 tokens, half turned: 39, 37, 41 us with 1, 2, 4)
  for (int e0 = threadIdx.x; e0 < total; e0 += 256 * U) {
    T* out[U];
    const float2* cs[U];
    float x[U][N], y[U][N];
#pragma unroll
    for (int i = 0; i < U; i++) {
      // e / units and th / nh: exact below 2^20, and a workgroup's units are fewer
      const int e = min(e0 + 256 * i, total - 1), th = (int)(((float)e + 0.5f) * by_units), u = e - th * units;
      const int t = (int)(((float)th + 0.5f) * by_heads), h = h0 + th - t * nh;
      const RotarySide& sd = h < a.side[0].heads ? a.side[0] : a.side[1];
      const int hh = h < a.side[0].heads ? h : h - a.side[0].heads;
      // entries behind the turned ones: cs null
      const int d = u < pairs ? u * N : a.rot + (u - pairs) * RN;
      const T* in = (const T*)sd.in + (t0 + t) * sd.its + hh * sd.ihs + d;
      out[i] = (T*)sd.out + (t0 + t) * sd.ots + hh * sd.ohs + d;
      cs[i] = u < pairs ? turn + t * half + (a.interleaved ? d / 2 : d) : nullptr;
      if (VEC || u < pairs) load_n<DT, N, VEC>(in, x[i]);
      else load_n<DT, RN, VEC>(in, x[i]);
      if (!a.interleaved && (VEC || u < pairs)) load_n<DT, N, VEC>(u < pairs ? in + half : in, y[i]);
    }
#pragma unroll
    for (int i = 0; i < U; i++) {
      if (e0 + 256 * i >= total) break;
      if (!cs[i]) store_n<DT, RN, VEC>(out[i], x[i]);
      else if (a.interleaved) {
        float p[N];
#pragma unroll
        for (int j = 0; j < N; j += 2) {
          const float2 w = cs[i][j / 2];
          p[j] = turned(x[i][j], w.x, -x[i][j + 1], w.y);
          p[j + 1] = turned(x[i][j + 1], w.x, x[i][j], w.y);
        }
        store_n<DT, N, VEC>(out[i], p);
      } else {
        float p[N], q[N];
#pragma unroll
        for (int j = 0; j < N; j++) {
          const float2 w = cs[i][j];
          p[j] = turned(x[i][j], w.x, -y[i][j], w.y);
          q[j] = turned(y[i][j], w.x, x[i][j], w.y);
        }
        store_n<DT, N, VEC>(out[i], p);
        store_n<DT, N, VEC>(out[i] + half, q);
      }
    }
  }
}

template <int DT>
static void launch_rotary(const RotaryArgs& a, bool vec, hipStream_t s) {
  constexpr int E = Vec<DT>::E;
  const int half = a.rot / 2, heads = a.side[0].heads + a.side[1].heads;
  // 16 bytes, pairs or single entries, as halves and alignment allow: 4096 tokens of 40 heads of 128 in bf16 with 112
  // entries turned 19 us (16 bytes), 116 31 us (pairs), 114 43 us (single)
  const int n = vec ? E : a.interleaved || !(half & 1) ? 2 : 1;
  const int units = (a.interleaved ? a.rot : half) / n + (a.dim - a.rot) / (vec ? n : 1);
  // a workgroup's work: about eight units a thread (sin and cos are made once for them), fewer where that leaves CUs
  // without any (512 workgroups wanted)
  int64_t per = a.tokens * heads * units / 512;
  per = per > 2048 ? 2048 : per < 256 ? 256 : per;
  int tw = (int)(per / (heads * units));
  tw = tw < 1 ? 1 : tw * half > 4096 ? (4096 / half > 1 ? 4096 / half : 1) : tw;
  int span = tw > 1 ? heads : (int)(per / units);
  span = span < 1 ? 1 : span > heads ? heads : span;
  const size_t lds = (size_t)tw * half * sizeof(float2);
  const int64_t most = MAX_THREADS / 256 * tw;      // tokens of a launch
  for (int64_t t0 = 0; t0 < a.tokens; t0 += most) {
    RotaryArgs p = a;
    p.tokens = a.tokens - t0 < most ? a.tokens - t0 : most;
    p.positions += t0;
    for (RotarySide& sd : p.side) {
      sd.in = (const typename Elem<DT>::T*)sd.in + t0 * sd.its;
      sd.out = (typename Elem<DT>::T*)sd.out + t0 * sd.ots;
    }
    const dim3 grid((unsigned)((p.tokens + tw - 1) / tw), (unsigned)((heads + span - 1) / span));
    if (vec) k_rotary<DT, E, true><<<grid, 256, lds, s>>>(p, tw, span);
    else if (n == 2) k_rotary<DT, 2, false><<<grid, 256, lds, s>>>(p, tw, span);
    else k_rotary<DT, 1, false><<<grid, 256, lds, s>>>(p, tw, span);
  }
}

}  // namespace externd

using namespace externd;

extern "C" {

int externd_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, int64_t original_length,
                               double beta_fast, double beta_slow, uint64_t* freqs, double* amplitude) {
  if (!freqs || rot_dim < 2 || rot_dim > 1024 || (rot_dim & 1) || !(base > 1) || !std::isfinite(base))
    return EXTERND_EINVAL;
  if (scaling < EXTERND_ROPE_PLAIN || scaling > EXTERND_ROPE_PARTS) return EXTERND_EINVAL;
  if (scaling != EXTERND_ROPE_PLAIN && (!(factor >= 1) || !std::isfinite(factor))) return EXTERND_EINVAL;
  if (scaling == EXTERND_ROPE_BASE && rot_dim < 4) return EXTERND_EINVAL;
  if (scaling == EXTERND_ROPE_PARTS && (original_length < 1 || !(beta_fast > beta_slow) || !std::isfinite(beta_fast) ||
                                        !std::isfinite(beta_slow)))
    return EXTERND_EINVAL;
  const long double two_pi = 6.283185307179586476925286766559L;
  long double b = base;
  if (scaling == EXTERND_ROPE_BASE) b *= powl(factor, (long double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < rot_dim / 2; i++) {
    long double th = powl(b, -2.0L * i / rot_dim);
    if (scaling == EXTERND_ROPE_LINEAR) th /= factor;
    if (scaling == EXTERND_ROPE_PARTS) {
      long double g = (original_length * th / two_pi - beta_slow) / ((long double)beta_fast - beta_slow);
      g = g < 0 ? 0 : g > 1 ? 1 : g;
      th = th * (g + (1 - g) / factor);
    }
    freqs[i] = (uint64_t)(th / two_pi * 18446744073709551616.0L + 0.5L);
  }
  if (amplitude) *amplitude = scaling == EXTERND_ROPE_PARTS ? 0.1 * log(factor) + 1.0 : 1.0;
  return EXTERND_OK;
}

int externd_rotary(const void* q, void* q_out, int64_t q_token_stride, int64_t q_head_stride,
                   int64_t q_out_token_stride, int64_t q_out_head_stride, int32_t heads_q, const void* k, void* k_out,
                   int64_t k_token_stride, int64_t k_head_stride, int64_t k_out_token_stride,
                   int64_t k_out_head_stride, int32_t heads_k, int32_t dtype, int64_t tokens, int32_t head_dim,
                   int32_t rot_dim, int32_t interleaved, int32_t inverse, const int64_t* positions,
                   const uint64_t* freqs, float amplitude, void* stream) {
  if (!dtype_ok(dtype) || tokens < 0 || head_dim < 2 || rot_dim < 2 || (rot_dim & 1) || rot_dim > head_dim ||
      heads_q < 1 || (interleaved & ~1) || (inverse & ~1) || !std::isfinite(amplitude))
    return EXTERND_EINVAL;
  if (!freqs || (tokens && (!q || !q_out || !positions)) || (k != nullptr) != (k_out != nullptr) || (k && heads_k < 1))
    return EXTERND_EINVAL;
  if (head_dim > 1024 || (int64_t)heads_q + (k ? heads_k : 0) > 65535 || tokens > INT32_MAX) return EXTERND_EUNSUPPORTED;
  if (!tokens) return EXTERND_OK;
  RotaryArgs a;
  a.side[0] = {q, q_out, q_token_stride, q_head_stride, q_out_token_stride, q_out_head_stride, heads_q};
  a.side[1] = {k, k_out, k_token_stride, k_head_stride, k_out_token_stride, k_out_head_stride, heads_k};
  a.positions = positions;
  a.freqs = freqs;
  a.tokens = tokens;
  a.dim = head_dim;
  a.rot = rot_dim;
  a.interleaved = interleaved;
  a.amplitude = amplitude;
  a.sign = inverse ? -1.f : 1.f;
  if (!k) a.side[1] = {};
  const int es = dtype_bytes(dtype), e = 16 / es;
  // 16-byte units: no unit may straddle the halves, the turned part or the head
  bool vec = !((interleaved ? rot_dim : rot_dim / 2) % e) && !((head_dim - rot_dim) % e);
  for (int i = 0; i < (k ? 2 : 1); i++)
    vec = vec && rows_aligned(a.side[i].in, a.side[i].its, a.side[i].ihs, es) &&
          rows_aligned(a.side[i].out, a.side[i].ots, a.side[i].ohs, es);
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) launch_rotary<EXTERND_F32>(a, vec, s);
  else if (dtype == EXTERND_BF16) launch_rotary<EXTERND_BF16>(a, vec, s);
  else launch_rotary<EXTERND_F16>(a, vec, s);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
