// Linear attention over chunks, backward: fp32 inputs and gradients.
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_bwd_f32(const LinattnPass& p, hipStream_t stream) {
  using namespace la;
  return launch_pass<kF32, kF32, kF32, false, 2, 2, false>(p, stream);
}
}  // namespace mmf
