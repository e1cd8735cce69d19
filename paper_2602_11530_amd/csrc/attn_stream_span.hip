// Launches of the stream pass for requests that see part of their context.
#include "attn_stream.h"

namespace pkv {
namespace {

template <int kD, bool kLarge>
void launch(const AttnLaunch& a, const SpanLayer& layer, size_t lds, hipStream_t stream) {
  const dim3 grid(a.waves / group_waves(kD)), block(group_waves(kD) * 64);
  if (a.kv_fp8) hipLaunchKernelGGL((attn_stream_kernel<kD, true, SpanLayer, kLarge && kD == 256>), grid, block, lds, stream, a, layer);
  else hipLaunchKernelGGL((attn_stream_kernel<kD, false, SpanLayer, kLarge>), grid, block, lds, stream, a, layer);
}

}  // namespace

hipError_t launch_attn_span(const AttnLaunch& a_in, const Span* span, hipStream_t stream) {
  AttnLaunch a = a_in;
  const bool fp4 = a.kv_fp8 == kFp4Pools;
  const StreamLds l = stream_lds(a.S, a.G, a.D, a.kv_fp8);
  a.staged_max = l.staged_max;
  a.wave_lds_floats = l.wave;
  a.turns = !fp4 && l.turn_bytes > 0;
  const size_t lds = l.bytes + (fp4 ? 0 : l.turn_bytes);
  if (!a.leaves_records) {
    // two records for each wavefront: nothing else is staged there
    a.wave_lds_floats = 2 * record_floats(a.G, a.D);
    a.staged_max = 1;
    const size_t small = (l.prefix + group_waves(a.D) * a.wave_lds_floats) * sizeof(float) + (a.turns ? l.turn_bytes : 0);
    return launch_attn_span_whole(a, span, small, stream);
  }
  if (fp4) return launch_attn_fp4(a, span, lds, stream);
  SpanLayer layer;
  layer.span = *span;
  AttnLaunch seen = a;   // the rules for long and short shares go by what is attended over
  seen.max_ctx = (int)(kBlockTokens * span->most_units(a.max_ctx));
  if (a.D == 64) launch<64, false>(a, layer, lds, stream);
  else if (a.D == 128) short_at_128(seen) ? launch<128, false>(a, layer, lds, stream) : launch<128, true>(a, layer, lds, stream);
  else if (a.D == 256) large_at_256(seen) ? launch<256, true>(a, layer, lds, stream) : launch<256, false>(a, layer, lds, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pkv
