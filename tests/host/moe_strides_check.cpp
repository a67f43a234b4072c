// Which rows have byte offsets below 2^31 (moe::short_rows), up to the largest strides that the C ABI takes: a single row may
// have any (run under the undefined-behaviour sanitizer).
#include <cstdio>
#include <cstdlib>

#include "../../paper_2607_19058_amd/csrc/moe_internal.h"

int main() {
  const int64_t top = 0x7FFFFFFFFFFFFFFF, most = 0x7FFFFFFF;
  const int64_t counts[] = {0, 1, 2, 40, 255, 256, 16382, 16383, most - 1, most};
  const int64_t strides[] = {1, 2, 8, 63, 1 << 16, (1 << 22) - 1, 1 << 22, 1 << 30, (int64_t)1 << 31, (int64_t)1 << 59, top - 1, top};
  for (int64_t rows : counts)
    for (int64_t ld : strides) {
      const bool want = (__int128)(rows + 1) * ld * 2 < ((__int128)1 << 31);
      if (moe::short_rows(rows, ld) != want) {
        printf("short_rows(%lld, %lld) is not %d\n", (long long)rows, (long long)ld, want);
        return 1;
      }
    }
  printf("strides checked\n");
  return 0;
}
