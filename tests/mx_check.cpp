// mx.h on the host: the scale byte of every bf16 value, and of values beside each border, is the
// least exponent that holds it.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "mx.h"

template <bool FP4>
int check(uint32_t bits) {
  float x;
  std::memcpy(&x, &bits, 4);
  const int got = dash::mx_byte<FP4>(bits);
  int want = 255;
  if (std::isfinite(x)) {
    const double most = FP4 ? 6.0 : 448.0, v = std::fmin((double)x, std::ldexp(1.5, 127));
    want = 10;
    while (v > std::ldexp(most, want - 127)) ++want;
  }
  if (got == want) return 0;
  std::printf("%s: %g (%08x): byte %d, want %d\n", FP4 ? "e2m1" : "e4m3", x, bits, got, want);
  return 1;
}

int main() {
  int bad = 0;
  for (uint32_t h = 0; h < 0x8000u && bad < 10; ++h) bad += check<false>(h << 16) + check<true>(h << 16);
  for (uint32_t e = 0; e < 255 && bad < 10; ++e)
    for (int32_t d = -2; d <= 2; ++d)
      for (uint32_t m : {0x0u, 0x400000u, 0x600000u}) {
        const uint32_t x = (e << 23 | m) + (uint32_t)d;
        if (x < 0x80000000u) bad += check<false>(x) + check<true>(x);
      }
  std::printf(bad ? "bad\n" : "ok\n");
  return bad != 0;
}
