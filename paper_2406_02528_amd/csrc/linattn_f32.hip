// Linear attention over chunks: fp32 inputs and outputs.
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_f32(const LinattnPass& p, bool state, hipStream_t stream) {
  using namespace la;
  return state ? launch_pass<kF32, kF32, kF32, true, 3, 3, true>(p, stream)
               : launch_pass<kF32, kF32, kF32, true, 3, 3, false>(p, stream);
}
}  // namespace mmf
