// K-split contraction of few token rows: the GLU gate's gradients, from rows of
// q (the training forward leaves no tiled ones).
#include "skinny_impl.h"

namespace mmf {

hipError_t launch_skinny_glu_grad(const ContractArgs& a, int fm, int fn, bool tiled, hipStream_t stream) {
  return a.epilogue == Epilogue::kGluGradF32 ? skinny::dispatch<Epilogue::kGluGradF32>(a, fm, fn, tiled, stream)
                                             : skinny::dispatch<Epilogue::kGluGradBf16>(a, fm, fn, tiled, stream);
}

}  // namespace mmf
