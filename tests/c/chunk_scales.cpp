// The power of two that a row's query is taken by in the chunk attention, for every exponent of its
// largest entry and every softmax scale: the scale of its logits is a normal number, and small enough
// that products of logits of ordinary size are normal numbers, too.
#include <cmath>
#include <cstdio>
#include <initializer_list>

#include "qv_chunk.h"

using namespace qv;

#define CHECK(x)                                                                        \
  do {                                                                                  \
    if (!(x)) {                                                                         \
      printf("line %d: %s (ex %d, scale 2^%d %g)\n", __LINE__, #x, ex, log_scale, part); \
      return 1;                                                                         \
    }                                                                                   \
  } while (0)

int main() {
  for (int log_scale = -64; log_scale <= 64; ++log_scale)
    for (float part : {1.f, 1.2f, 1.3862944f, 1.3862945f, 1.5f, 1.9999999f}) {
      if (log_scale == 64 && part > 1.f) continue;
      // as the host does
      const float scale_log2 = std::ldexp(part, log_scale) * 1.44269504088896340736f;
      int scale_exp;
      const float m = std::frexp(scale_log2, &scale_exp);
      for (int ex = -126; ex <= 127; ++ex) {
        const int shift = chunk_query_shift(ex, scale_exp);
        const float sc = std::ldexp(m, scale_exp + shift);
        CHECK(sc >= 0x1p-126f && sc < 0x1p100f);
        // the largest entries of such a row (the smallest of all with ex = -126), and the smallest
        const float most = ex == -126 ? 0x1p-133f : std::ldexp(1.f, ex);
        CHECK(std::ldexp(std::ldexp(most, -shift), shift) == most);
        // where products with the largest keys are out of range, logits of them are
        const double row = std::ldexp(1.9921875 * most, -shift);
        CHECK(row <= 0x1p-19 || (row * 128 * 127 < 0x1p127 && sc >= 1.f));
      }
    }
  printf("ok\n");
  return 0;
}
