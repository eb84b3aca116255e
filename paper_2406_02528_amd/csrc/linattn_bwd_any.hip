// Linear attention over chunks, backward: bf16 and fp32 among the operands.
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_bwd_any(const LinattnPass& p, bool state, hipStream_t stream) {
  using namespace la;
  return state ? launch_pass<kEither, kEither, kEither, true, 3, 3, true>(p, stream)
               : launch_pass<kEither, kEither, kEither, false, 2, 2, false>(p, stream);
}
}  // namespace mmf
