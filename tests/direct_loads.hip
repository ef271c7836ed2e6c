// Loads of operands that go straight into LDS, issued on the host: where each
// would read.  Compiled for the host alone by test_direct_loads_cpu.py.
#include <cstdio>
#include <cstdlib>

#include "externd_gemm.hpp"

using namespace externd;

// All loads of a product over K rows of an operand by columns, from the first stage to the last
// one that the loop issues: an access that the buffer's size lets through lies in the operand, and
// none is let through past the last step.
template <int X, int EV>
static long columns(int64_t stride, int64_t count, int64_t K, int stages) {
  typedef Direct<true, X, 64, EV> D;
  const int64_t bytes = 16 / EV, steps = (K + 63) / 64, end = ((K - 1) * stride + count) * bytes;
  char* const p = (char*)((int64_t)1 << 44);      // never read
  long wrong = 0;
  for (int thread = 0; thread < GEMM_THREADS; thread++)
    for (int64_t x0 : {(int64_t)0, (count - 1) / X * X}) {
      D d;
      d.init(Operand{p, stride}, x0, count - x0, 0, K, thread);
      for (int64_t n = 0; n < stages + steps - 1; n++, d.next())
        for (int i = 0; i < D::LOADS; i++) {
          if (d.offset[i] > d.room() || d.room() - d.offset[i] < 16) continue;      // the hardware gives zeros
          const int64_t at = d.base + d.offset[i] - p;
          wrong += at < 0 || at + 16 > end || n >= steps;
        }
    }
  return wrong;
}

// The same of an operand by rows of K entries, of which `count` are there: no load past a row's end either.
template <int X, int BK, int EV>
static long rows(int64_t stride, int64_t count, int64_t K, int stages) {
  typedef Direct<false, X, BK, EV> D;
  const int64_t bytes = 16 / EV, steps = (K + BK - 1) / BK;
  char* const p = (char*)((int64_t)1 << 44);
  long wrong = 0;
  for (int thread = 0; thread < GEMM_THREADS; thread++)
    for (int64_t x0 : {(int64_t)0, (count - 1) / X * X}) {
      D d;
      d.init(Operand{p, stride}, x0, count - x0, 0, K, thread);
      for (int64_t n = 0; n < stages + steps - 1; n++, d.next()) {
        if (n == 4 && steps > 16) {      // on to the last steps
          for (; n < steps - 4; n++) d.next();
        }
        for (int i = 0; i < D::LOADS; i++) {
          int r, v;
          D::T::place(i * GEMM_THREADS + thread, &r, &v);
          if (d.k_left < BK && v * EV >= d.k_left) continue;      // as issue() has it
          if (d.offset[i] > d.room() || d.room() - d.offset[i] < 16) continue;
          const int64_t at = d.base + d.offset[i] - p, row = at / (stride * bytes), column = at % (stride * bytes);
          wrong += at < 0 || row >= count || column + 16 > K * bytes || n >= steps;
        }
      }
    }
  return wrong;
}

int main() {
  const int64_t most = ((int64_t)1 << 25) + 768;      // the longest row of G
  long wrong = 0;
  for (int64_t K : {1, 2, 3, 4, 5, 31, 32, 33, 63, 64, 65, 100, 128, 129, 300})
    for (int64_t stride : {(int64_t)264, ((int64_t)1 << 20) + 256, ((int64_t)1 << 22) - 8, ((int64_t)1 << 24) - 256, (int64_t)1 << 24,
                           ((int64_t)1 << 24) + 256, (int64_t)25000192, ((int64_t)1 << 25) - 256, (int64_t)1 << 25, most}) {
      if (K > 64 && K * stride > ((int64_t)1 << 27)) continue;      // rows of a piece hold no more than this together
      for (int64_t count : {(int64_t)8, (int64_t)264, stride}) {
        long w = 0;
        for (int stages : {2, 3, 4}) w += columns<256, 8>(stride, count, K, stages) + columns<32, 8>(stride, count, K, stages) + columns<128, 8>(stride, count, K, stages);
        if (w) printf("%lld rows of %lld, %lld columns: %ld loads\n", (long long)K, (long long)stride, (long long)count, w);
        wrong += w;
      }
    }
  for (int64_t stride : {(int64_t)264, (int64_t)4096, ((int64_t)1 << 22) - 8, most})
    for (int64_t count : {(int64_t)1, (int64_t)3, (int64_t)32, (int64_t)100, (int64_t)300})
      for (int64_t K : {(int64_t)8, (int64_t)256, (int64_t)264, stride}) {
        if (K > stride || (stride == most && count > 32)) continue;      // G's rows: no more than a piece holds
        long w = 0;
        for (int stages : {2, 3, 4, 6})
          w += rows<256, 64, 8>(stride, count, K, stages) + rows<128, 64, 8>(stride, count, K, stages) + rows<32, 64, 8>(stride, count, K, stages) +
               rows<64, 256, 8>(stride, count, K, stages) + rows<256, 32, 4>(stride, count, K, stages);
        if (w) printf("%lld rows of %lld, %lld k: %ld loads\n", (long long)count, (long long)stride, (long long)K, w);
        wrong += w;
      }
  printf("%ld loads outside\n", wrong);
  return wrong != 0;
}
