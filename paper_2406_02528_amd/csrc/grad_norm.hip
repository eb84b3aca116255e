// The norm over all elements of a set of gradients, and the set scaled to it:
//   norm = sqrt(sum over the arrays of sum g^2)   (squares and sums in fp64)
//   c = max_norm / (norm + 1e-6),  out = g min(c, 1)   (fp32)
//
// A launch covers up to kSet arrays, whose addresses and sizes travel in its
// arguments; their elements are cut into pieces of kPiece (the last of an
// array shorter), one workgroup each.  Every piece's sum of squares is a
// partial of its own, and one workgroup adds them in a fixed order: the same
// bits on every call, with no atomics.
#include "mmf_device.h"
#include "mmf_launch.h"
#include "row_vec.h"

namespace mmf {
namespace {

constexpr int kBlock = 256;
constexpr int kSet = 128;                           // arrays per launch (its arguments take 3.6 KB)
constexpr int64_t kPiece = 16384;                   // elements per workgroup
constexpr int64_t kMaxPieces = int64_t(1) << 23;    // workgroups per launch
static_assert(kMaxPieces * kPiece >= kGradMaxCount, "an array fits a launch");

struct Set {
  const void* src[kSet];
  void* dst[kSet];
  int64_t count[kSet];
  uint32_t first[kSet];    // first piece of each array, from this launch's first
  uint32_t f32[kSet / 32];
  int n;
};

// The array and the piece of it that workgroup `blk` takes (REV: an array's
// pieces from its last to its first).
struct Piece {
  int i;
  int64_t begin, end;
  bool f32;
};
template <bool REV>
__device__ __forceinline__ Piece piece_of(const Set& s, uint32_t blk) {
  int lo = 0, hi = s.n - 1;  // the last array whose first piece is at most blk
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (s.first[mid] <= blk) lo = mid;
    else hi = mid - 1;
  }
  int64_t p = blk - s.first[lo];
  if constexpr (REV) p = (s.count[lo] - 1) / kPiece - p;
  const int64_t begin = p * kPiece;
  const int64_t end = begin + kPiece < s.count[lo] ? begin + kPiece : s.count[lo];
  return {lo, begin, end, ((s.f32[lo / 32] >> (lo % 32)) & 1u) != 0};
}

// Elements [begin, end) of an array: whole vectors of E, then the rest one by
// one (arrays and pieces start on 16 bytes).
template <typename T, typename F, typename G>
__device__ __forceinline__ void each(int64_t begin, int64_t end, F&& vec, G&& one) {
  constexpr int E = 16 / sizeof(T);
  const int64_t whole = begin + (end - begin) / E * E;
  for (int64_t i = begin + E * threadIdx.x; i < whole; i += E * kBlock) vec(i);
  const int64_t i = whole + threadIdx.x;
  if (i < end) one(i);
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[kBlock / kWave];
  v = wave_sum_f64(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

template <typename T>
__device__ __forceinline__ double sum_squares(const T* g, int64_t begin, int64_t end) {
  constexpr int E = 16 / sizeof(T);
  double ss = 0.0;
  each<T>(
      begin, end,
      [&](int64_t i) {
        RowVec<T, E> v;
        const uint4 w = *reinterpret_cast<const uint4*>(g + i);
        v.w[0] = w.x; v.w[1] = w.y; v.w[2] = w.z; v.w[3] = w.w;
#pragma unroll
        for (int e = 0; e < E; ++e) ss = sum_sq(ss, v.get(e));
      },
      [&](int64_t i) {
        if constexpr (sizeof(T) == 4) ss = sum_sq(ss, g[i]);
        else ss = sum_sq(ss, bf16_to_f32(g[i]));
      });
  return ss;
}

__global__ __launch_bounds__(kBlock) void grad_sumsq_kernel(const Set s, double* __restrict__ partials) {
  const Piece p = piece_of<false>(s, blockIdx.x);
  const double ss = p.f32 ? sum_squares(static_cast<const float*>(s.src[p.i]), p.begin, p.end)
                          : sum_squares(static_cast<const uint16_t*>(s.src[p.i]), p.begin, p.end);
  const double t = block_sum(ss);
  if (threadIdx.x == 0) partials[blockIdx.x] = t;
}

__global__ __launch_bounds__(kBlock) void grad_norm_kernel(const double* __restrict__ partials, int64_t n,
                                                           float* __restrict__ norm) {
  double v = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < n; i += kBlock) v += partials[i];
  const double t = block_sum(v);
  if (threadIdx.x == 0) norm[0] = static_cast<float>(__builtin_sqrt(t));
}

template <typename T>
__device__ __forceinline__ void scale(const T* g, T* o, int64_t begin, int64_t end, float c) {
  constexpr int E = 16 / sizeof(T);
  each<T>(
      begin, end,
      [&](int64_t i) {
        RowVec<T, E> v;
        const uint4 w = *reinterpret_cast<const uint4*>(g + i);
        v.w[0] = w.x; v.w[1] = w.y; v.w[2] = w.z; v.w[3] = w.w;
        float f[E];
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = v.get(e) * c;
        v.set(f);
        *reinterpret_cast<uint4*>(o + i) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
      },
      [&](int64_t i) {
        if constexpr (sizeof(T) == 4) o[i] = g[i] * c;
        else o[i] = static_cast<uint16_t>(pack_bf16(bf16_to_f32(g[i]) * c, 0.0f));
      });
}

// The arrays and their pieces from the last to the first: the sums of squares
// read them in the other order, so what they read last is still in the
// last-level cache.
__global__ __launch_bounds__(kBlock) void grad_scale_kernel(const Set s, const float* __restrict__ norm,
                                                            float max_norm) {
  float c = max_norm / (norm[0] + 1e-6f);
  if (c > 1.0f) c = 1.0f;  // a NaN stays
  const Piece p = piece_of<true>(s, blockIdx.x);
  if (c == 1.0f && s.src[p.i] == s.dst[p.i]) return;  // nothing changes
  if (p.f32) scale(static_cast<const float*>(s.src[p.i]), static_cast<float*>(s.dst[p.i]), p.begin, p.end, c);
  else scale(static_cast<const uint16_t*>(s.src[p.i]), static_cast<uint16_t*>(s.dst[p.i]), p.begin, p.end, c);
}

// Calls launch(set, pieces) for every launch's worth of arrays, from the first
// to the last or (reverse) from the last to the first.  An array's pieces fit
// a launch (counts are at most kGradMaxCount), so every round takes one.
template <typename F>
hipError_t for_sets(const GradSetArgs& a, bool reverse, F&& launch) {
  int64_t done = 0;
  while (done < a.n) {
    Set s{};
    int64_t pieces = 0;
    for (; done < a.n; ++done) {
      const int64_t i = reverse ? a.n - 1 - done : done;
      const int64_t p = (a.counts[i] + kPiece - 1) / kPiece;
      if (p == 0) continue;
      if (s.n == kSet || pieces + p > kMaxPieces) break;
      s.src[s.n] = a.src[i];
      s.dst[s.n] = a.dst != nullptr ? a.dst[i] : nullptr;
      s.count[s.n] = a.counts[i];
      s.first[s.n] = static_cast<uint32_t>(pieces);
      if (a.is_f32[i]) s.f32[s.n / 32] |= 1u << (s.n % 32);
      pieces += p;
      ++s.n;
    }
    if (pieces == 0) break;
    const hipError_t e = launch(s, static_cast<uint32_t>(pieces));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

int64_t grad_pieces(const int64_t* counts, int64_t n) {
  int64_t p = 0;
  for (int64_t i = 0; i < n; ++i) p += (counts[i] + kPiece - 1) / kPiece;
  return p;
}

hipError_t launch_grad_norm(const GradSetArgs& a, float* norm, double* partials, hipStream_t stream) {
  int64_t done = 0;
  const hipError_t e = for_sets(a, false, [&](const Set& s, uint32_t pieces) {
    hipLaunchKernelGGL(grad_sumsq_kernel, dim3(pieces), dim3(kBlock), 0, stream, s, partials + done);
    done += pieces;
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kBlock), 0, stream, partials, done, norm);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const GradSetArgs& a, const float* norm, float max_norm, hipStream_t stream) {
  return for_sets(a, true, [&](const Set& s, uint32_t pieces) {
    hipLaunchKernelGGL(grad_scale_kernel, dim3(pieces), dim3(kBlock), 0, stream, s, norm, max_norm);
    return hipGetLastError();
  });
}

}  // namespace mmf
