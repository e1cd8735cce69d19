// Launches of the stream pass for requests that see part of their context.
#include "attn_stream.h"

namespace pkv {
namespace {

template <int kD>
void launch_dim(const AttnLaunch& a, const SpanLayer& layer, size_t lds, hipStream_t stream) {
  constexpr bool kLarge = kD == 128;
  const dim3 grid(a.waves / group_waves(kD)), block(group_waves(kD) * 64);
  if (a.kv_fp8) hipLaunchKernelGGL((attn_stream_kernel<kD, true, SpanLayer, false>), grid, block, lds, stream, a, layer);
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
  if (!a.leaves_records) return launch_attn_span_whole(a, span, lds, stream);
  if (fp4) return launch_attn_fp4(a, span, lds, stream);
  SpanLayer layer;
  layer.span = *span;
  if (a.D == 64) launch_dim<64>(a, layer, lds, stream);
  else if (a.D == 128) launch_dim<128>(a, layer, lds, stream);
  else if (a.D == 256) launch_dim<256>(a, layer, lds, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pkv
