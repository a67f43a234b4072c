// The tile of the weights' gradient from kept rows: reads lines "places experts rows columns", prints a number for each.
#include <cstdio>

#include "../../paper_2607_19058_amd/csrc/kept_internal.h"

int main() {
  long long places, experts, n, m;
  while (scanf("%lld %lld %lld %lld", &places, &experts, &n, &m) == 4) printf("%d\n", moe::kept_tile(places, experts, n, m));
  return 0;
}
