// Linear attention over chunks: fp32 operands; o in fp32, and the states' sums.
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_f32(const LinattnPass* p, int n, hipStream_t stream) {
  using namespace la;
  return launch_passes<kF32, kF32, kF32, true, false>(p, n, stream);
}
hipError_t launch_linattn_states_f32(const LinattnPass* p, int n, hipStream_t stream) {
  using namespace la;
  return launch_passes<kF32, kF32, kF32, true, true>(p, n, stream);
}
}  // namespace mmf
