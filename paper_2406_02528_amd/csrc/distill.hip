// Distillation from a teacher's K best tokens.  For each row of student logits
// z [V] and teacher logits t [K] at the tokens idx [K] (entries outside [0, V)
// or of -inf are none), with the temperature tau:
//   p = softmax(t / tau),  ln q = ln softmax(z / tau)
//   loss = tau^2 sum_j p_j (ln p_j - ln q[idx_j])
//   dz = dloss tau (q - p at idx)
//
// One workgroup of 1024 threads takes a row and keeps it in registers (up to
// kHeld values per thread), so that the maximum, the sum and the gradient are
// one pass over memory; longer rows are read again from the caches.  The K
// teacher entries are handled in LDS; their gradients are written again after
// the row's, behind a barrier.
//
// fp32 with the sums of 4 or 8 exponentials and the rest in fp64; the loss in
// fp64 (p ln p - p ln q cancels where the student agrees).  Bound by HBM: one
// read of z, one write of dz.
#include "distill.h"
#include "mmf_device.h"
#include "row_vec.h"

namespace mmf {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr double kLog2e = 1.4426950408889634074;

template <typename T>
__device__ __forceinline__ float value(const T* p) {
  if constexpr (sizeof(T) == 4) return *p;
  else return bf16_to_f32(*p);
}

struct Shared {
  double sum[kWaves];
  float max[kWaves];
  double part[kWaves];
  int idx[kDistillMaxK];
  float z[kDistillMaxK];
  double p[kDistillMaxK];
};

__device__ __forceinline__ float block_max(float v, float* slot) {
  v = wave_max_f32(v);
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = slot[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) m = fmaxf(m, slot[i]);
  return m;
}
__device__ __forceinline__ double block_sum(double v, double* slot) {
  v = wave_sum_f64(v);
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = slot[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) s += slot[i];
  return s;
}

// The simple form: every pass over the row from memory, a value at a time.
template <typename T, typename D>
__global__ __launch_bounds__(kThreads) void distill_kernel(const DistillArgs a) {
  __shared__ Shared sh;
  const int64_t m = blockIdx.x;
  const int V = static_cast<int>(a.V), K = static_cast<int>(a.K);
  const T* const z = static_cast<const T*>(a.z) + m * V;
  D* const dz = a.dz != nullptr ? static_cast<D*>(a.dz) + m * V : nullptr;
  const double c = kLog2e / a.tau;
  const float cf = static_cast<float>(c);

  // the teacher's entries
  const int j = threadIdx.x;
  int ij = -1;
  float tj = -__builtin_inff();
  if (j < K) {
    ij = a.idx[m * K + j];
    if (ij < 0 || ij >= V) ij = -1;
    if (ij >= 0) tj = a.t_is_f32 ? static_cast<const float*>(a.t)[m * K + j] : bf16_to_f32(static_cast<const uint16_t*>(a.t)[m * K + j]);
    if (tj == -__builtin_inff()) ij = -1;
    sh.idx[j] = ij;
    sh.z[j] = ij >= 0 ? value(z + ij) : 0.0f;
  }
  const float w = a.dloss != nullptr ? a.dloss[m] : 0.0f;
  const bool none = !__syncthreads_or(ij >= 0);
  if (none || (dz != nullptr && w == 0.0f && a.loss == nullptr)) {
    if (threadIdx.x == 0 && a.loss != nullptr) a.loss[m] = 0.0f;
    if (dz != nullptr)
      for (int i = threadIdx.x; i < V; i += kThreads) dz[i] = static_cast<D>(0);
    return;
  }
  const float tm = block_max(tj, sh.max);
  const double u = ij >= 0 ? (static_cast<double>(tj) - tm) / a.tau : 0.0;
  const double eu = ij >= 0 ? exp(u) : 0.0;
  const double su = block_sum(eu, sh.sum);
  const double lnp = u - log(su), p = ij >= 0 ? eu / su : 0.0;
  if (j < K) sh.p[j] = p;

  float zm = -__builtin_inff();
  for (int i = threadIdx.x; i < V; i += kThreads) {
    const float x = value(z + i);
    zm = fmaxf(zm, x);
  }
  __syncthreads();
  zm = block_max(zm, sh.max);
  double s = 0.0;
  for (int i = threadIdx.x; i < V; i += kThreads) s += __builtin_amdgcn_exp2f((value(z + i) - zm) * cf);
  const double sum = block_sum(s, sh.part);
  double l = 0.0;
  if (ij >= 0 && p > 0.0) l = p * (lnp - ((static_cast<double>(sh.z[j]) - zm) / a.tau - log(sum)));
  __syncthreads();
  const double loss = block_sum(l, sh.sum);
  if (threadIdx.x == 0 && a.loss != nullptr) a.loss[m] = static_cast<float>(loss * a.tau * a.tau);
  if (dz == nullptr) return;
  const bool zero = w == 0.0f;
  const double wt = static_cast<double>(w) * a.tau;
  const float g = static_cast<float>(wt / sum);
  const auto put = [&](int i, float y) {
    if (zero) y = 0.0f;
    if constexpr (sizeof(D) == 4) dz[i] = y;
    else dz[i] = static_cast<uint16_t>(pack_bf16(y, 0.0f));
  };
  for (int i = threadIdx.x; i < V; i += kThreads) put(i, __builtin_amdgcn_exp2f((value(z + i) - zm) * cf) * g);
  __syncthreads();
  if (ij >= 0) {
    bool first = true;
    double ps = 0.0;
    for (int k = 0; k < K; ++k)
      if (sh.idx[k] == ij) {
        if (k < j) first = false;
        ps += sh.p[k];
      }
    if (first) put(ij, static_cast<float>((__builtin_amdgcn_exp2f((sh.z[j] - zm) * cf) / sum - ps) * wt));
  }
}

}  // namespace

hipError_t launch_distill(const DistillArgs& a, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(a.M));
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  };
  if (a.z_is_f32) return a.dz_is_f32 ? go(distill_kernel<float, float>) : go(distill_kernel<float, uint16_t>);
  return a.dz_is_f32 ? go(distill_kernel<uint16_t, float>) : go(distill_kernel<uint16_t, uint16_t>);
}

}  // namespace mmf
