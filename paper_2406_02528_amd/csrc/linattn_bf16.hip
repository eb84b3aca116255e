// Linear attention over chunks: bf16 operands and o; and the states' sums.
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_bf16(const LinattnPass* p, int n, hipStream_t stream) {
  using namespace la;
  return launch_passes<kBf16, kBf16, kBf16, false, false>(p, n, stream);
}
hipError_t launch_linattn_states_bf16(const LinattnPass* p, int n, hipStream_t stream) {
  using namespace la;
  return launch_passes<kBf16, kBf16, kBf16, false, true>(p, n, stream);
}
}  // namespace mmf
