// The norm over all elements of a set of gradients, and the set scaled to it:
//   norm = sqrt(sum over the arrays of sum g^2)   (squares and sums in fp64)
//   c = max_norm / (norm + 1e-6),  out = g min(c, 1)   (fp32; c = 1 where
//   max_norm is infinite and norm is a number)
//
// A launch covers up to kSet arrays, whose addresses and sizes travel in its
// arguments; their elements are cut into pieces of kPiece (the last of an
// array shorter), one workgroup each.  Every piece's sum of squares is a
// partial of its own, and one workgroup adds them in a fixed order: the same
// bits on every call, with no atomics.
//
// Bound by HBM: 4 bytes read for the norm, 4 read and 4 written for the
// scaling.  All of it passes the caches as streams (nontemporal), at any size:
// a cached read pushes out lines that others wrote, which go to memory first,
// and what a backward pass leaves in the caches is mostly not the gradients.
// Norm and scaling in place, as streams / cached, us:
//   set of                      32 MB      64 MB      128 MB     192 MB     400 MB     800 MB
//   behind 1 GB of other work   29 / 28    44 / 47    76 / 83    109 / 119  227 / 240  457 / 466
//   the whole set just written  36 / 31    49 / 44    74 / 66    110 / 96   234 / 241  469 / 472
// Cached accesses gain where nothing but the gradients was written before (up
// to 192 MB), and leave up to that much for a reader that follows: both calls
// and an update that reads the gradients once, behind other work, 94 / 90 us
// at 64 MB, 167 / 162 at 128, 250 / 243 at 192, 523 / 559 at 400.
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

// The array and the piece of it that workgroup `blk` takes.
struct Piece {
  int i;
  int64_t begin, end;
  bool f32;
};
__device__ __forceinline__ Piece piece_of(const Set& s, uint32_t blk) {
  int lo = 0, hi = s.n - 1;  // the last array whose first piece is at most blk
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (s.first[mid] <= blk) lo = mid;
    else hi = mid - 1;
  }
  const int64_t begin = static_cast<int64_t>(blk - s.first[lo]) * kPiece;
  const int64_t end = begin + kPiece < s.count[lo] ? begin + kPiece : s.count[lo];
  return {lo, begin, end, ((s.f32[lo / 32] >> (lo % 32)) & 1u) != 0};
}

// Elements [begin, end) of an array: vec(raw, i) for whole vectors of 16 bytes,
// kAhead of a thread's loads in flight together, then one(i) for the rest
// (arrays and pieces start on 16 bytes).
constexpr int kAhead = 8;
typedef unsigned int v4u __attribute__((ext_vector_type(4)));
__device__ __forceinline__ v4u load16(const void* p) { return __builtin_nontemporal_load(static_cast<const v4u*>(p)); }
__device__ __forceinline__ void store16(void* p, v4u w) { __builtin_nontemporal_store(w, static_cast<v4u*>(p)); }
template <typename T, typename F, typename G>
__device__ __forceinline__ void each(const T* g, int64_t begin, int64_t end, F&& vec, G&& one) {
  constexpr int E = 16 / sizeof(T);
  const int n = static_cast<int>(end - begin);  // at most kPiece
  const T* const p = g + begin;
  const int whole = n / E;
  int v = threadIdx.x;
  for (; v + (kAhead - 1) * kBlock < whole; v += kAhead * kBlock) {
    v4u w[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) w[u] = load16(p + static_cast<int64_t>(v + u * kBlock) * E);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) vec(w[u], begin + static_cast<int64_t>(v + u * kBlock) * E);
  }
  for (; v < whole; v += kBlock) vec(load16(p + static_cast<int64_t>(v) * E), begin + static_cast<int64_t>(v) * E);
  const int i = whole * E + threadIdx.x;
  if (i < n) one(begin + i);
}

template <typename T>
__device__ __forceinline__ RowVec<T, 16 / sizeof(T)> row_vec(v4u w) {
  RowVec<T, 16 / sizeof(T)> v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v.w[i] = w[i];
  return v;
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
  each(
      g, begin, end,
      [&](v4u w, int64_t) {
        const auto v = row_vec<T>(w);
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
  const Piece p = piece_of(s, blockIdx.x);
  const double ss = p.f32 ? sum_squares(static_cast<const float*>(s.src[p.i]), p.begin, p.end)
                          : sum_squares(static_cast<const uint16_t*>(s.src[p.i]), p.begin, p.end);
  const double t = block_sum(ss);
  if (threadIdx.x == 0) partials[blockIdx.x] = t;
}

__global__ __launch_bounds__(kBlock) void grad_norm_kernel(const double* __restrict__ partials, int64_t n,
                                                           float* __restrict__ norm) {
  constexpr int kLoads = 16;
  double v = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += kLoads * kBlock) {
    double p[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) p[u] = i + u * kBlock < n ? partials[i + u * kBlock] : 0.0;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) v += p[u];
  }
  const double t = block_sum(v);
  if (threadIdx.x == 0) norm[0] = static_cast<float>(__builtin_sqrt(t));
}

template <typename T>
__device__ __forceinline__ void scale(const T* g, T* o, int64_t begin, int64_t end, float c) {
  constexpr int E = 16 / sizeof(T);
  each(
      g, begin, end,
      [&](v4u w, int64_t i) {
        auto v = row_vec<T>(w);
        float f[E];
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = v.get(e) * c;
        v.set(f);
        store16(o + i, v4u{v.w[0], v.w[1], v.w[2], v.w[3]});
      },
      [&](int64_t i) {
        if constexpr (sizeof(T) == 4) o[i] = g[i] * c;
        else o[i] = static_cast<uint16_t>(pack_bf16(bf16_to_f32(g[i]) * c, 0.0f));
      });
}

__global__ __launch_bounds__(kBlock) void grad_scale_kernel(const Set s, const float* __restrict__ norm,
                                                            float max_norm) {
  float c = max_norm / (norm[0] + 1e-6f);
  if (c > 1.0f) c = 1.0f;  // a NaN stays
  if (max_norm == __builtin_inff() && norm[0] == norm[0]) c = 1.0f;  // no limit, also for an infinite norm
  const Piece p = piece_of(s, blockIdx.x);
  if (c == 1.0f && s.src[p.i] == s.dst[p.i]) return;  // nothing changes
  if (p.f32) scale(static_cast<const float*>(s.src[p.i]), static_cast<float*>(s.dst[p.i]), p.begin, p.end, c);
  else scale(static_cast<const uint16_t*>(s.src[p.i]), static_cast<uint16_t*>(s.dst[p.i]), p.begin, p.end, c);
}

// Calls launch(set, pieces) for every launch's worth of arrays.  An array's
// pieces fit a launch (counts are at most kGradMaxCount), so every round takes
// one.
template <typename F>
hipError_t for_sets(const GradSetArgs& a, F&& launch) {
  int64_t done = 0;
  while (done < a.n) {
    Set s{};
    int64_t pieces = 0;
    for (; done < a.n; ++done) {
      const int64_t i = done;
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
  const hipError_t e = for_sets(a, [&](const Set& s, uint32_t pieces) {
    hipLaunchKernelGGL(grad_sumsq_kernel, dim3(pieces), dim3(kBlock), 0, stream, s, partials + done);
    done += pieces;
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kBlock), 0, stream, partials, done, norm);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const GradSetArgs& a, const float* norm, float max_norm, hipStream_t stream) {
  return for_sets(a, [&](const Set& s, uint32_t pieces) {
    hipLaunchKernelGGL(grad_scale_kernel, dim3(pieces), dim3(kBlock), 0, stream, s, norm, max_norm);
    return hipGetLastError();
  });
}

}  // namespace mmf
