// Launches of the stream pass over E2M1 tiles.
#include "attn_stream.h"

namespace pkv {
namespace {

template <int kD>
void launch_dim(const AttnLaunch& a, const Span* span, size_t lds, hipStream_t stream) {
  const dim3 grid(a.waves / group_waves(kD)), block(group_waves(kD) * 64);
  if (span) {
    Fp4SpanLayer layer;
    layer.span = *span;
    hipLaunchKernelGGL((attn_stream_kernel<kD, true, Fp4SpanLayer, false>), grid, block, lds, stream, a, layer);
  } else {
    hipLaunchKernelGGL((attn_stream_kernel<kD, true, Fp4Layer, false>), grid, block, lds, stream, a, Fp4Layer{});
  }
}

}  // namespace

hipError_t launch_attn_fp4(const AttnLaunch& a, const Span* span, size_t lds, hipStream_t stream) {
  if (a.D == 64) launch_dim<64>(a, span, lds, stream);
  else if (a.D == 128) launch_dim<128>(a, span, lds, stream);
  else if (a.D == 256) launch_dim<256>(a, span, lds, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pkv
