// Host build (g++ -fsanitize=undefined) of num_pages (paper_2404_15778_amd/csrc/attn_plan.h): pages for lengths up to the end of the 32-bit range, compared
// with a count in 64 bits.  Prints "ok <cases>" and exits 0, or the first difference and exits 1.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "attn_plan.h"

int main() {
  int cases = 0;
  for (int64_t page : {32, 64, 96, 160, 4096, 1 << 20, 1 << 30, (INT_MAX / 32) * 32})
    for (int64_t around : {(int64_t)0, page, 2 * page, 1000 * page, INT_MAX / page * page, (int64_t)INT_MAX})
      for (int64_t tokens = around - 3; tokens <= around + 3; ++tokens) {
        if (tokens < 0 || tokens > INT_MAX) continue;
        ++cases;
        const int got = bass::num_pages((int)tokens, (int)page);
        if (got != (tokens + page - 1) / page) {
          printf("FAIL: %lld tokens, pages of %lld: %d\n", (long long)tokens, (long long)page, got);
          return 1;
        }
      }
  printf("ok %d\n", cases);
  return 0;
}
