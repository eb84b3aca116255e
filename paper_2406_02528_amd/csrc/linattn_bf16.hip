// Linear attention over chunks: bf16 operands and o; the state within a segment to
// 2^-16 of each key, or (last: it is the result) to 2^-24; and the states' sums.
#include "linattn_chunk.h"

namespace mmf {
hipError_t launch_linattn_bf16(const LinattnPass* p, int n, bool last, hipStream_t stream) {
  using namespace la;
  return last ? launch_passes<kBf16, kBf16, kBf16, false, 2, 3, false>(p, n, stream)
              : launch_passes<kBf16, kBf16, kBf16, false, 2, 2, false>(p, n, stream);
}
hipError_t launch_linattn_states_bf16(const LinattnPass* p, int n, hipStream_t stream) {
  using namespace la;
  return launch_passes<kBf16, kBf16, kBf16, false, 2, 3, true>(p, n, stream);
}
}  // namespace mmf
