// Linear attention over chunks: operands of both types, o in bf16 (backward); and
// the states' sums.
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_bwd_any(const LinattnPass* p, int n, hipStream_t stream) {
  using namespace la;
  return launch_passes<kEither, kEither, kEither, false, false>(p, n, stream);
}
hipError_t launch_linattn_states_any(const LinattnPass* p, int n, hipStream_t stream) {
  using namespace la;
  return launch_passes<kEither, kEither, kEither, true, true>(p, n, stream);
}
}  // namespace mmf
