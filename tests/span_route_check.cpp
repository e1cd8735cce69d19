// The host's choice of a way through the attention calls with windows and over 4-bit pools, from the C-ABI layer itself: linked against stand-ins
// for the launches, it asks for each batch twice, with a tight bound on the lengths and with a loose one.  Where the tight one alone leads to a
// workgroup for each segment, the general launch has to find that out on the device by the same numbers, for no bit of a row depends on the bound:
// no more segments than a launch has workgroups, of the same length at most.  Run by tests/test_span_routes.py (host code
// only, no GPU).
#include "../include/pkv.h"
#include "pkv_kernels.h"
#include <cstdio>

static pkv::AttnLaunch got;

namespace pkv {
hipError_t launch_attn_span(const AttnLaunch& a, const Span*, hipStream_t) {
  got = a;
  return hipSuccess;
}
hipError_t launch_attn_reduce(const AttnLaunch&, const AttnLayers*, hipStream_t) { return hipSuccess; }
hipError_t launch_copy(const void*, void*, int64_t, hipStream_t) { return hipSuccess; }
}  // namespace pkv

int main() {
  using namespace pkv;
  char* const base = reinterpret_cast<char*>((uintptr_t)1 << 40);   // addresses only
  const int32_t* ints = reinterpret_cast<const int32_t*>((uintptr_t)1 << 39);
  char* p[4];
  for (int i = 0; i < 4; ++i) p[i] = base + ((uintptr_t)(i + 1) << 36);
  long batches = 0, tight_only = 0, cut = 0, wrong = 0;
  for (int dim : {64, 128, 256})
    for (int kind = 0; kind < 3; ++kind)
      for (int seqs : {1, 8, 9, 32, 33, 45, 48, 64, 65, 255, 256, 257, 300, 383, 384, 512, 513})
        for (int hkv : {1, 8})
          for (int bound : {1, 16, 100, 300, 384, 700, 768, 769, 1536, 1537, 4000})
            for (int window : {-1, 0, 1, 64, 300, 700, 740, 1500, 5000, 2147483647})
              for (int sinks : {0, 4, 100, 2147483647}) {
                if (window < 0 && (kind != 2 || sinks != 0)) continue;   // no window: tiles
                AttnLaunch by[2];
                for (int loose = 0; loose < 2; ++loose) {
                  const pkv_attn_shape sh = {seqs, 4 * hkv, hkv, dim, 16, 10000 / 16, 0, loose ? 10000 : bound, 1000};
                  const size_t need = (size_t)1 << 33;
                  const int rc =
                      window < 0 ? paged_decode_attn_fp4kv(p[0], p[1], p[2], ints, ints, 1.f, p[3], &sh, base, need, nullptr)
                      : kind == 0 ? paged_decode_attn_window(p[0], p[1], p[2], ints, ints, 1.f, window, sinks, p[3], &sh, base, need, nullptr)
                      : kind == 1 ? paged_decode_attn_window_fp8kv(p[0], p[1], p[2], ints, ints, 1.f, 1.f, 1.f, window, sinks, p[3], &sh, base, need, nullptr)
                                  : paged_decode_attn_window_fp4kv(p[0], p[1], p[2], ints, ints, 1.f, window, sinks, p[3], &sh, base, need, nullptr);
                  if (rc != PKV_OK) return printf("status %d\n", rc), 1;
                  by[loose] = got;
                }
                batches++;
                cut += !by[0].leaves_records;
                if (by[0].leaves_records == by[1].leaves_records) continue;
                tight_only++;
                const bool found = !by[0].leaves_records && (int64_t)seqs * hkv <= by[1].waves / group_waves(dim) && by[0].short_blocks == by[1].short_blocks;
                if (!found && wrong++ < 10)
                  printf("D=%d kind %d, %d requests on %d KV heads, bound %d, window %d, sinks %d\n", dim, kind, seqs, hkv, bound, window, sinks);
              }
  printf("%ld batches, %ld cut by the tight bound, %ld by that alone, wrong=%ld\n", batches, cut, tight_only, wrong);
  return wrong != 0 || cut == 0 || tight_only == 0;
}
