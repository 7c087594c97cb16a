// The sine and cosine of csrc/rope_turn.h against 64 bits, and the errors that its comment states: every STEP-th argument of a whole
// turn, the borders of its eighths and of their neighbours among them.  Prints the largest errors in units of 2^-24.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>

#include "../../paper_2508_16201_b200/csrc/rope_turn.h"

int main(int argc, char** argv) {
  const uint64_t step = argc > 1 ? strtoull(argv[1], nullptr, 10) : 61;
  const double two_pi = 6.283185307179586476925;
  double worst_s = 0, worst_c = 0, poly_s = 0, poly_c = 0;
  auto look = [&](uint32_t turn) {
    float s, c;
    specvlm::turn_sincos(turn, s, c);
    // reduced exactly first: a quarter of a turn at a time
    const uint32_t quarter = (turn + 0x20000000u) >> 30;
    const double a = two_pi * ((double)(int32_t)(turn - (quarter << 30)) * 0x1p-32), sn = std::sin(a), cs = std::cos(a);
    const double want_s[4] = {sn, cs, -sn, -cs}, want_c[4] = {cs, -sn, -cs, sn};
    // the eighths around 0 and a half turn take the one polynomial for the sine, the others the other
    const double es = std::fabs(s - want_s[quarter]), ec = std::fabs(c - want_c[quarter]);
    worst_s = std::max(worst_s, quarter & 1 ? ec : es);
    worst_c = std::max(worst_c, quarter & 1 ? es : ec);
    const double x = (double)(int32_t)(turn - (quarter << 30)) * 0x1p-32, u = x * x;
    poly_s = std::max(poly_s, std::fabs(x * (6.2831854820251465 + u * (-41.3416633605957 + u * (81.5925521850586 - u * 75.40206909179688))) - sn));
    poly_c = std::max(poly_c, std::fabs(1.0 + u * (-19.739208221435547 + u * (64.93931579589844 + u * (-85.44285583496094 + u * 59.22040557861328))) - cs));
  };
  for (uint64_t t = 0; t < (1ull << 32); t += step) look((uint32_t)t);
  for (int e = 0; e < 8; ++e)
    for (int d = -1000; d <= 1000; ++d) look((uint32_t)e * 0x20000000u + (uint32_t)d);
  printf("%.4f %.4f %.3e %.3e\n", worst_s * 0x1p24, worst_c * 0x1p24, poly_s, poly_c);
  return 0;
}
