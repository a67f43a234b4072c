// The rounds in which the weights' gradient takes an expert's places (moe::round_length), at the largest number of places:
// every place once, in order, with no sum beyond 32 bits on the way (run under the undefined-behaviour sanitizer).
#include <cstdio>
#include <cstdlib>

#include "../../paper_2607_19058_amd/csrc/moe_internal.h"

static void check(int places, int most) {
  long long covered = 0;
  for (int base = 0; base < places;) {
    const int n = moe::round_length(base, places, most);
    if (n < 1 || n > most || base != covered || (long long)base + n > places) {
      printf("round at %d of %d: length %d\n", base, places, n);
      exit(1);
    }
    covered += n;
    base += n;
  }
  if (covered != places) exit(1);
}

int main() {
  const int most = 1024, top = 0x7FFFFFFF;
  for (int n = 0; n < 3 * most; n += 7) check(n, most);
  for (int n = 0; n < 5; n++) check(top - n, most);
  check(top - most, most);
  printf("rounds checked\n");
  return 0;
}
