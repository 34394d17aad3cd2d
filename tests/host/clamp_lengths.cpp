// Host build (g++ -fsanitize=undefined) of clamp_lengths (paper_2404_15778_amd/csrc/attn_plan.h) on lengths at the ends of the 32-bit range: prints a
// line "L nq kmax Lcap -> L nq clamped" per case, for the test beside it to compare with whole numbers of any size.
#include <climits>
#include <cstdio>
#include <initializer_list>

#include "attn_plan.h"

int main() {
  for (int Lcap : {1, 7, 1000, INT_MAX - 31, INT_MAX})
    for (int kmax : {1, 8, 64})
      for (int n : {INT_MIN, -1, 0, 1, 8, 64, INT_MAX})
        for (int L : {INT_MIN, INT_MIN + 1, -1, 0, 1, 993, 999, 1000, 1001, INT_MAX - 64, INT_MAX - 8, INT_MAX - 1, INT_MAX}) {
          int l = L, q = n;
          const bool bad = bass::clamp_lengths(l, q, kmax, Lcap);
          printf("%d %d %d %d -> %d %d %d\n", L, n, kmax, Lcap, l, q, (int)bad);
        }
  return 0;
}
