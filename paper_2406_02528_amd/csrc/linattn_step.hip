// Linear attention with a decay per head, token by token:
//   S = l S + k v^T,   o = scale S^T q      (S [dk][dv] per sequence and head)
// for single tokens and runs of a few.  A workgroup keeps 32 columns of one
// head's state in registers (4 columns x every 32nd row per thread) over all
// tokens of the call, so the state is read and written once.
//
// fp32 throughout; the column sums of o go over a thread's rows, then the
// rows of a wave (lanes 8, 16 and 32 apart), then the four waves, in that
// order.  Bound by HBM (8 bytes per entry of the state) for batches, 45 sequences of
// 16 heads of 128 bf16 in 20 us, 4.8 TB/s; by its latency for one, 4 us.
#include "linattn.h"
#include "mmf_device.h"
#include "row_vec.h"

namespace mmf {
namespace {

constexpr int kThreads = 256;
constexpr int kCols = 32;                 // columns of the state per workgroup
constexpr int kRowStep = kThreads / 8;    // rows of the state one pass of the workgroup covers

__device__ __forceinline__ float ld1(const float* p) { return *p; }
__device__ __forceinline__ float ld1(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float4 ld4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 ld4(const uint16_t* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
}
__device__ __forceinline__ void st1(float* p, float v) { *p = v; }
__device__ __forceinline__ void st1(uint16_t* p, float v) { *p = static_cast<uint16_t>(pack_bf16(v, 0.0f)); }

// R: rows of the state per thread, 32 apart.
template <typename T, int R>
__global__ __launch_bounds__(kThreads) void linattn_step_kernel(const LinattnArgs a) {
  __shared__ float4 part[2][kThreads / kWave][8];
  const uint32_t tiles = static_cast<uint32_t>(a.dv + kCols - 1) / kCols;
  const uint32_t bh = blockIdx.x / tiles, tile = blockIdx.x % tiles;
  const int64_t b = bh / static_cast<uint32_t>(a.H), h = bh % static_cast<uint32_t>(a.H);
  const int c = threadIdx.x & 7, r = threadIdx.x >> 3, wave = threadIdx.x >> 6;
  const int e0 = static_cast<int>(tile) * kCols + 4 * c;
  const bool on = e0 < a.dv;
  const int64_t row = static_cast<int64_t>(a.H) * (2 * a.dk + a.dv);
  const T* const x = static_cast<const T*>(a.qkv) + b * a.T * row;
  const T* const q = x + h * a.dk;
  const T* const k = x + (a.H + h) * a.dk;
  const T* const v = x + 2 * static_cast<int64_t>(a.H) * a.dk + h * a.dv;
  T* const o = static_cast<T*>(a.o) + (b * a.T * a.H + h) * a.dv;
  const int64_t state = static_cast<int64_t>(bh) * a.dk * a.dv + e0;
  const float l = a.decay[h];

  float4 s[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int d = r + i * kRowStep;
    s[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (on && d < a.dk && a.s0 != nullptr) s[i] = ld4(a.s0 + state + static_cast<int64_t>(d) * a.dv);
  }
  for (int64_t t = 0; t < a.T; ++t) {
    float4 vt = make_float4(0.0f, 0.0f, 0.0f, 0.0f), sum = vt;
    if (on) vt = ld4(v + t * row + e0);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int d = r + i * kRowStep;
      const float kd = d < a.dk ? ld1(k + t * row + d) : 0.0f;
      const float qd = d < a.dk ? ld1(q + t * row + d) : 0.0f;
      s[i].x = fmaf(kd, vt.x, l * s[i].x);
      s[i].y = fmaf(kd, vt.y, l * s[i].y);
      s[i].z = fmaf(kd, vt.z, l * s[i].z);
      s[i].w = fmaf(kd, vt.w, l * s[i].w);
      sum.x = fmaf(qd, s[i].x, sum.x);
      sum.y = fmaf(qd, s[i].y, sum.y);
      sum.z = fmaf(qd, s[i].z, sum.z);
      sum.w = fmaf(qd, s[i].w, sum.w);
    }
#pragma unroll
    for (int x = 8; x < kWave; x *= 2) {
      sum.x += __shfl_xor(sum.x, x);
      sum.y += __shfl_xor(sum.y, x);
      sum.z += __shfl_xor(sum.z, x);
      sum.w += __shfl_xor(sum.w, x);
    }
    // the slots in turn: a wave writes one again only after the barrier of
    // the token between, which every reader of it has passed
    if ((threadIdx.x & 63) < 8) part[t & 1][wave][c] = sum;
    __syncthreads();
    if (threadIdx.x < kCols && static_cast<int>(tile) * kCols + static_cast<int>(threadIdx.x) < a.dv) {
      float y = 0.0f;
#pragma unroll
      for (int w = 0; w < kThreads / kWave; ++w) y += reinterpret_cast<const float*>(part[t & 1][w])[threadIdx.x];
      st1(o + t * a.H * a.dv + tile * kCols + threadIdx.x, y * a.scale);
    }
  }
  if (on && a.s_last != nullptr) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int d = r + i * kRowStep;
      if (d < a.dk) *reinterpret_cast<float4*>(a.s_last + state + static_cast<int64_t>(d) * a.dv) = s[i];
    }
  }
}

template <typename T>
hipError_t launch(const LinattnArgs& a, hipStream_t stream) {
  const uint32_t tiles = static_cast<uint32_t>((a.dv + kCols - 1) / kCols);
  const dim3 grid(static_cast<uint32_t>(a.B * a.H) * tiles);
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  };
  if (a.dk <= kRowStep) return go(linattn_step_kernel<T, 1>);
  if (a.dk <= 2 * kRowStep) return go(linattn_step_kernel<T, 2>);
  if (a.dk <= 4 * kRowStep) return go(linattn_step_kernel<T, 4>);
  return go(linattn_step_kernel<T, 8>);
}

}  // namespace

hipError_t launch_linattn_step(const LinattnArgs& a, hipStream_t stream) {
  return a.is_f32 ? launch<float>(a, stream) : launch<uint16_t>(a, stream);
}

}  // namespace mmf
