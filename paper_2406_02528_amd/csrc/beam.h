// Internal launchers of the beam search kernels.  Shapes are validated by the
// C-ABI layer before any of these is called.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mmf {

// The n best of W x V candidates of each of B batches; done, new_done may be
// nullptr, end < 0: no such token.
constexpr int kBeamMax = 64;          // beams, and candidates kept
constexpr int kBeamMaxV = 1 << 18;    // tokens
struct BeamSelectArgs {
  const void* logits;
  bool is_f32;
  const float* scores;
  const uint8_t* done;
  int end;
  int64_t B;
  int W, V, n;
  float* new_scores;
  int32_t* tokens;
  int32_t* parents;
  uint8_t* new_done;
};
size_t beam_select_bytes(int64_t B, int W, int V, int n);
hipError_t launch_beam_select(const BeamSelectArgs& a, void* scratch, hipStream_t stream);

// Rows [B W] of row_bytes[i] bytes of each of `count` arrays, row (b, j) from
// row (b, parents[b][j]); dst[i] may be src[i].
struct BeamReorderArgs {
  const void* const* src;
  void* const* dst;
  const int64_t* row_bytes;
  int64_t count;
  const int32_t* parents;
  int64_t B;
  int W;
};
hipError_t launch_beam_reorder(const BeamReorderArgs& a, hipStream_t stream);

}  // namespace mmf
