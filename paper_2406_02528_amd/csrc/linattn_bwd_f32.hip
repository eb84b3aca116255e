// Linear attention over chunks: fp32 operands, o in bf16 (backward).
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_bwd_f32(const LinattnPass* p, int n, hipStream_t stream) {
  using namespace la;
  return launch_passes<kF32, kF32, kF32, false, false>(p, n, stream);
}
}  // namespace mmf
