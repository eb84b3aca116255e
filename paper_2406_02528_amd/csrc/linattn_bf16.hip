// Linear attention over chunks: bf16 inputs and outputs.
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_bf16(const LinattnPass& p, bool state, hipStream_t stream) {
  using namespace la;
  return state ? launch_pass<kBf16, kBf16, kBf16, false, 2, 3, true>(p, stream)
               : launch_pass<kBf16, kBf16, kBf16, false, 2, 3, false>(p, stream);
}
}  // namespace mmf
