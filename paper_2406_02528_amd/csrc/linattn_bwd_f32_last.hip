// Linear attention over chunks: fp32 operands in three parts, o in bf16: the backward
// of one segment, whose state behind the last token is a result.
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_bwd_f32_last(const LinattnPass* p, int n, hipStream_t stream) {
  using namespace la;
  return launch_passes<kF32, kF32, kF32, false, 3, 3, false>(p, n, stream);
}
}  // namespace mmf
