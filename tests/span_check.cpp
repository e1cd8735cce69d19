// Which units and tokens of a request are attended over (Span in csrc/pkv_kernels.h) against the definition, token by token.  Run by
// tests/test_span.py (host code only, no GPU).
#include "pkv_kernels.h"
#include <cstdio>
#include <vector>

int main() {
  using namespace pkv;
  long checked = 0, wrong = 0;
  for (int L = 0; L <= 150; ++L)
    for (int window : {0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 64, 100, 149, 150, 1000})
      for (int sinks : {0, 1, 4, 15, 16, 17, 20, 32, 33, 64, 100, 150, 1000}) {
        const Span span = {window, sinks};
        std::vector<int> found(L + 32, 0);
        const int n = span.units(L);
        int last = -1;
        for (int b = 0; b < n; ++b) {
          const int u = span.unit(b, L);
          const uint32_t seen = span.seen(u, L);
          if (u <= last || seen == 0 || seen > 0xffff) wrong++;   // in order, each with a token
          last = u;
          for (int i = 0; i < kBlockTokens; ++i)
            if ((seen >> i) & 1) {
              if (kBlockTokens * u + i >= L) wrong++;
              else found[kBlockTokens * u + i]++;
            }
        }
        for (int t = 0; t < L; ++t)
          if (found[t] != (t >= L - window || t < sinks)) wrong++;
        if (n > span.most_units(150)) wrong++;
        checked++;
      }
  // sizes at the end of 32 bits
  const Span wide = {INT32_MAX, INT32_MAX};
  if (wide.units(INT32_MAX) != (1 << 27) || wide.left_out(INT32_MAX) != 0 || wide.most_units(INT32_MAX) != (1 << 27)) wrong++;
  const Span ends = {1, 0};
  if (ends.units(INT32_MAX) != 1 || ends.unit(0, INT32_MAX) != (1 << 27) - 1 || ends.seen((1 << 27) - 1, INT32_MAX) != 1u << 14) wrong++;
  printf("checked %ld, wrong=%ld\n", checked, wrong);
  return wrong != 0;
}
