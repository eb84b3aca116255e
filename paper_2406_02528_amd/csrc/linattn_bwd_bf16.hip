// Linear attention over chunks, backward: bf16 inputs and gradients.
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_bwd_bf16(const LinattnPass& p, hipStream_t stream) {
  using namespace la;
  return launch_pass<kBf16, kBf16, kBf16, false, 2, 2, false>(p, stream);
}
}  // namespace mmf
