// Relative error of the gated block's distribution function against long double: lines "max LO HI error", and what special values give.
#include <stdio.h>

#include "normal_cdf.hpp"

int main() {
  const double edges[] = {-13, -8, -4, -2, -1, 0, 14};
  const int n = sizeof edges / sizeof *edges - 1;
  double worst[n] = {}, far = 0.0, least = 0.0;
  for (int i = -1300000; i <= 1300000; ++i) {
    const float v = (float)(i * 1e-5);
    float e;
    const double p = scmoe::normal_cdf(v, e);
    const long double want = 0.5L * erfcl(-(long double)v / sqrtl(2.0L)), f = expl(-0.5L * (long double)v * v);
    const double off = (double)(fabsl(p - want) / want), off_e = (double)(fabsl(e - f) / f) / (4.0 + 2.0 * v * v) * 16777216.0;
    for (int q = 0; q < n; ++q)
      if (v >= edges[q] && v < edges[q + 1] && off > worst[q]) worst[q] = off;
    if (off_e > far) far = off_e;
    if (p < least) least = p;
  }
  for (int q = 0; q < n; ++q) printf("max %g %g %.4e\n", edges[q], edges[q + 1], worst[q]);
  float e;
  const float inf = INFINITY;
  printf("e %.4f\nleast %g\n", far, least);
  printf("special %g %g", scmoe::normal_cdf(inf, e), e);
  printf(" %g %g", scmoe::normal_cdf(-inf, e), e);
  printf(" %g %g %d\n", scmoe::normal_cdf(-3e19f, e), scmoe::normal_cdf(3e19f, e), scmoe::normal_cdf(NAN, e) != scmoe::normal_cdf(NAN, e));
  return 0;
}
