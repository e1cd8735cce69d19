// Which new tokens fall into a block (tokens_in_block in csrc/pkv_kernels.h) against the definition in 64 bits, with as many blocks asked for as a launch
// has slots, padding behind the last request among them.  Run by tests/test_block_parts.py (host code only, no GPU).
#include "pkv_kernels.h"
#include <algorithm>
#include <cstdio>

static long checked = 0, wrong = 0;

// New tokens [start, start + n) of a context of L, asked for in its k-th block from the first one on.
static void check(int start, int64_t n, int64_t L, int64_t k, int log_block) {
  const int64_t B = 1 << log_block, first = std::max<int64_t>(L - n, 0), block = first / B + k;
  const int64_t from = std::max(first, block * B), to = std::min(L, (block + 1) * B);
  const pkv::InBlock at = pkv::tokens_in_block(7, start, (int)(start + n), (int)L, (int)k, log_block);
  const bool any = n > 0 && to > from;
  // as the kernel takes it: a count in 32 bits, nothing to do where it is not positive
  const int count = (int)((uint32_t)at.to - (uint32_t)at.from);
  if (any ? count != to - from || at.from != from || at.s != 7 || at.token != start + n - (L - from) : count > 0) {
    if (wrong < 5) printf("start %d n %ld L %ld k %ld B %ld: %d to %d, not %ld to %ld\n", start, (long)n, (long)L, (long)k, (long)B, at.from, at.to, (long)from, (long)to);
    wrong++;
  }
  checked++;
}

int main() {
  for (int log_block : {4, 5, 6}) {
    const int B = 1 << log_block;
    for (int L = 0; L <= 3 * B + 2; ++L)
      for (int n = 0; n <= 4 * B; ++n)
        for (int k = 0; k <= n / B + 4; ++k) check(5, n, L, k, log_block);
    // the longest context, and those whose end a launch's last slots are 2^31 tokens from
    const int64_t most = (int64_t)INT32_MAX - 4096, tokens = (1 << 24) - 1, slots = tokens / B + 2;
    for (int64_t L : {most, most - 1, most - B, most - tokens, (int64_t)INT32_MAX + 1 - tokens, (int64_t)1 << 30})
      for (int64_t n : {(int64_t)0, (int64_t)1, (int64_t)B, (int64_t)5000, tokens - 1})
        for (int64_t k = 0; k <= slots; k += k < 1000 || k > slots - 1000 ? 1 : 37) check((int)(tokens - 1 - n), n, L, k, log_block);
  }
  printf("checked %ld, wrong=%ld\n", checked, wrong);
  return wrong != 0;
}
