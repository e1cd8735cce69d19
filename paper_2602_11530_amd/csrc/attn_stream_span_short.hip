// Launches of the stream pass with a workgroup for each segment: requests that see part of their context, E2M1 tiles, and both.
#include "attn_stream.h"

namespace pkv {
namespace {

template <int kD, bool kFp8, typename Layer>
void launch(const AttnLaunch& a, const Layer& layer, size_t lds, hipStream_t stream) {
  hipLaunchKernelGGL((attn_stream_kernel<kD, kFp8, Layer, false>), dim3(a.Hkv, 1, a.S), dim3(group_waves(kD) * 64), lds, stream, a, layer);
}

template <int kD>
void launch_dim(const AttnLaunch& a, const Span* span, size_t lds, hipStream_t stream) {
  if (!span) return launch<kD, true>(a, WholeFp4Layer{}, lds, stream);
  WholeFp4SpanLayer tiles;
  WholeSpanLayer rows;
  tiles.span = rows.span = *span;
  if (a.kv_fp8 == kFp4Pools) launch<kD, true>(a, tiles, lds, stream);
  else if (a.kv_fp8) launch<kD, true>(a, rows, lds, stream);
  else launch<kD, false>(a, rows, lds, stream);
}

}  // namespace

hipError_t launch_attn_span_whole(const AttnLaunch& a, const Span* span, size_t lds, hipStream_t stream) {
  if (a.D == 64) launch_dim<64>(a, span, lds, stream);
  else if (a.D == 128) launch_dim<128>(a, span, lds, stream);
  else if (a.D == 256) launch_dim<256>(a, span, lds, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pkv
