// Shares of a launch's workgroups: arguments tiles1 cost1 tiles2 cost2 resident cus, several times; prints the first product's workgroups an XCD.
#include <stdio.h>
#include <stdlib.h>

#include "pair_share.hpp"

int main(int n, char** v) {
  for (int i = 1; i + 5 < n; i += 6)
    printf("%d\n", scmoe::share_pair(atof(v[i]), atof(v[i + 1]), atof(v[i + 2]), atof(v[i + 3]), atoi(v[i + 4]), atoi(v[i + 5])).first);
  return 0;
}
