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

// One workgroup per token and side: its threads go over the heads' entries,
// a pair (or an entry that is only copied) at a time.
template <int DT>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a) {
  typedef typename Elem<DT>::T T;
  const int64_t t = blockIdx.x;
  const RotarySide sd = a.side[blockIdx.y];
  const int half = a.rot / 2, rest = a.dim - a.rot, per = half + rest;
  const uint64_t pos = (uint64_t)a.positions[t];
  for (int e = threadIdx.x; e < sd.heads * per; e += 256) {
    const int h = e / per, i = e - h * per;
    const T* in = (const T*)sd.in + t * sd.its + h * sd.ihs;
    T* out = (T*)sd.out + t * sd.ots + h * sd.ohs;
    if (i >= half) {
      out[a.rot + i - half] = in[a.rot + i - half];
      continue;
    }
    const int p = a.interleaved ? 2 * i : i, q = a.interleaved ? 2 * i + 1 : i + half;
    float s, c;
    sincos_turns(pos * a.freqs[i], &s, &c);
    s *= a.sign * a.amplitude;
    c *= a.amplitude;
    const float x = Elem<DT>::load(in[p]), y = Elem<DT>::load(in[q]);
    out[p] = Elem<DT>::store(x * c - y * s);
    out[q] = Elem<DT>::store(y * c + x * s);
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
  if (head_dim > 1024 || heads_q > 65535 || (k && heads_k > 65535) || tokens > INT32_MAX) return EXTERND_EUNSUPPORTED;
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
  const dim3 grid((unsigned)tokens, k ? 2 : 1);
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == EXTERND_F32) k_rotary<EXTERND_F32><<<grid, 256, 0, s>>>(a);
  else if (dtype == EXTERND_BF16) k_rotary<EXTERND_BF16><<<grid, 256, 0, s>>>(a);
  else k_rotary<EXTERND_F16><<<grid, 256, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? EXTERND_OK : EXTERND_EHIP;
}

}  // extern "C"
