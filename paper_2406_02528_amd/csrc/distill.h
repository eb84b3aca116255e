// Internal launcher of the distillation kernel.  Shapes are validated by the
// C-ABI layer before it is called.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mmf {

// M rows of V student logits and K teacher entries.  dz nullptr: the loss
// alone (dloss is then not read); loss may be nullptr with dz.  dz may be z.
constexpr int kDistillMaxK = 1024;
struct DistillArgs {
  const void* z;
  bool z_is_f32;
  const int32_t* idx;
  const void* t;
  bool t_is_f32;
  float tau;
  const float* dloss;
  void* dz;
  bool dz_is_f32;
  float* loss;
  int64_t M, V, K;
};
hipError_t launch_distill(const DistillArgs& a, hipStream_t stream);

}  // namespace mmf
