// Distillation from a teacher's K best tokens.  For each row of student logits
// z [V] and teacher logits t [K] at the tokens idx [K] (entries outside [0, V)
// or of -inf are none), with the temperature tau:
//   p = softmax(t / tau),  ln q = ln softmax(z / tau)
//   loss = tau^2 sum_j p_j (ln p_j - ln q[idx_j])
//   dz = dloss tau (q - p at idx)
//
// A workgroup takes a row and keeps it in registers, so that the maximum, the
// sum and the gradient are one pass over memory; rows of more than 32768 bf16 or
// 65536 fp32 logits are read again for the gradient.  Rows are vectors of 8 values
// that start on 16 bytes in z and dz alike, and the few values before and after
// them.  What the teacher's entries need (their softmax, z at their tokens, which
// of them share a token) is done while the row's loads are in flight; their
// gradients are written again after the row's, behind a barrier.
//
// fp32 with the sums of 8 exponentials and the rest in fp64; the loss and the
// gradient at the entries in fp64 (p ln p - p ln q and q - p cancel where the
// student agrees).  Bound by HBM, one read of z and one write of dz: 8192 x 32000
// bf16, 64 entries, in 192 us, 5.5 TB/s; few rows by the row's chain of loads,
// maxima and sums (77 x 50001 fp32, the loss alone: 10 us).
#include "distill.h"
#include "mmf_device.h"
#include "row_vec.h"

namespace mmf {
namespace {

constexpr double kLog2e = 1.4426950408889634074;

template <typename T>
__device__ __forceinline__ float value(const T* p) {
  if constexpr (sizeof(T) == 4) return *p;
  else return bf16_to_f32(*p);
}

// The teacher's entries of a row in LDS: token (-1: none), z there, t and then p.
constexpr int kScan = 16;   // tokens that a comparison with all of them reads at once
constexpr int entries_room(int K) { return (K + kScan - 1) / kScan * kScan; }
constexpr size_t kEntryBytes = sizeof(double) + sizeof(float) + sizeof(int);
struct Entries {
  double* p;
  float* z;
  int* idx;   // those behind the last: none
};

// f(k, whether entry k has token i) for the K entries in order; reads of 16 bytes
// that do not wait for one another (one at a time they took 8 us for 64 entries).
template <typename F>
__device__ __forceinline__ void scan(const Entries& en, int K, int i, F&& f) {
  for (int k = 0; k < K; k += kScan) {
    int4 x[kScan / 4];
#pragma unroll
    for (int g = 0; g < kScan / 4; ++g) x[g] = *reinterpret_cast<const int4*>(&en.idx[k + 4 * g]);
#pragma unroll
    for (int g = 0; g < kScan / 4; ++g) {
      f(k + 4 * g, x[g].x == i);
      f(k + 4 * g + 1, x[g].y == i);
      f(k + 4 * g + 2, x[g].z == i);
      f(k + 4 * g + 3, x[g].w == i);
    }
  }
}

template <int W>
struct Slots {
  float tm[W], zm[W];
  double te[W], ze[W], loss[W];
};

template <int W>
__device__ __forceinline__ float max_of(const float* s) {
  float m = s[0];
#pragma unroll
  for (int i = 1; i < W; ++i) m = fmaxf(m, s[i]);
  return m;
}
template <int W>
__device__ __forceinline__ double sum_of(const double* s) {
  double t = s[0];
#pragma unroll
  for (int i = 1; i < W; ++i) t += s[i];
  return t;
}

// HELD: vectors per thread, kept in registers (0: read twice).
template <typename T, typename D, int THREADS, int HELD, bool NT>
__global__ __launch_bounds__(THREADS, 4) void distill_kernel(const DistillArgs a) {
  constexpr int W = THREADS / kWave, E = 8;
  extern __shared__ __attribute__((aligned(16))) double s_entries[];   // kEntryBytes for each of K, rounded up
  __shared__ Slots<W> sl;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int64_t m = blockIdx.x;
  const int V = static_cast<int>(a.V), K = static_cast<int>(a.K), room = entries_room(K);
  const Entries en{s_entries, reinterpret_cast<float*>(s_entries + room), reinterpret_cast<int*>(s_entries + room) + room};
  const T* const z = static_cast<const T*>(a.z) + m * V;
  D* const dz = a.dz != nullptr ? static_cast<D*>(a.dz) + m * V : nullptr;
  // values before the first whole vector, whole vectors, values after them
  const int ahead = static_cast<int>((E - m * V % E) % E);
  const int head = ahead < V ? ahead : V;
  const int nv = (V - head) / E, tail = V - head - nv * E;
  const auto rz = row_rsrc(z + head, nv * E, true);
  const int own = tid < head ? tid : tid >= E && tid - E < tail ? head + nv * E + tid - E : -1;  // a value outside the vectors

  RowVec<T, E> in[HELD > 0 ? HELD : 1];
  if constexpr (HELD > 0) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) in[i].template load<NT>(rz, tid + i * THREADS);
  }
  float zx = own >= 0 ? value(z + own) : -__builtin_inff();

  // --- the teacher's entries
  const double inv = 1.0 / a.tau;
  const float c = static_cast<float>(kLog2e / a.tau);
  float tm = -__builtin_inff();
  bool any = false;
  for (int j = K + tid; j < room; j += THREADS) en.idx[j] = -1;
  for (int j = tid; j < K; j += THREADS) {
    int i = a.idx[m * K + j];
    const float t = a.t_is_f32 ? static_cast<const float*>(a.t)[m * K + j]
                               : bf16_to_f32(static_cast<const uint16_t*>(a.t)[m * K + j]);
    if (i < 0 || i >= V || t == -__builtin_inff()) i = -1;
    en.idx[j] = i;
    en.z[j] = i >= 0 ? value(z + i) : 0.0f;
    en.p[j] = t;
    any |= i >= 0;
    if (i >= 0) tm = fmaxf(tm, t);
  }
  const float w = a.dloss != nullptr ? a.dloss[m] : 0.0f;
  const bool none = !__syncthreads_or(any);
  if (none || (w == 0.0f && a.loss == nullptr)) {
    if (tid == 0 && a.loss != nullptr) a.loss[m] = 0.0f;
    if (dz != nullptr) {
      RowVec<D, E> o;
#pragma unroll
      for (int i = 0; i < o.kWords; ++i) o.w[i] = 0;
      for (int v = tid; v < nv; v += THREADS) o.template store<NT>(dz + head, v);
      if (own >= 0) dz[own] = static_cast<D>(0);
    }
    return;
  }
  uint32_t twice = 0;   // which of the thread's entries, in turn, share their token with others
  static_assert(kDistillMaxK <= 32 * THREADS, "a bit for each");
  if (dz != nullptr) {
    for (int j = tid, n = 0; j < K; j += THREADS, ++n) {
      const int i = en.idx[j];
      int same = 0;
      scan(en, K, i, [&](int, bool is) { same += is; });
      if (same > 1 && i >= 0) twice |= 1u << n;
    }
  }

  // --- maxima
  float zm = zx;
  double ze = 0.0;
  if constexpr (HELD > 0) {
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (tid + i * THREADS < nv) {
#pragma unroll
        for (int e = 0; e < E; ++e) zm = fmaxf(zm, in[i].get(e));
      }
  } else {
    // The sum as well, against the thread's own running maximum.  While that is -inf
    // (masked tokens alone), against 0: the sum stays 0, or the NaN of one there.
    for (int v = tid; v < nv; v += THREADS) {
      RowVec<T, E> x;
      x.load(rz, v);
      float vm = zm;
#pragma unroll
      for (int e = 0; e < E; ++e) vm = fmaxf(vm, x.get(e));
      if (vm > zm) {
        ze *= __builtin_amdgcn_exp2f((zm - vm) * c);
        zm = vm;
      }
      const float from = zm == -__builtin_inff() ? 0.0f : zm;
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f((x.get(e) - from) * c);
      ze += s;
    }
  }
  const float own_max = zm;
  tm = wave_max_f32(tm);
  zm = wave_max_f32(zm);
  if (lane == 0) {
    sl.tm[wave] = tm;
    sl.zm[wave] = zm;
  }
  __syncthreads();
  tm = max_of<W>(sl.tm);
  zm = max_of<W>(sl.zm);

  // --- sums; the exponentials stay in place of the row
  float ex[HELD > 0 ? HELD : 1][E];
  if constexpr (HELD > 0) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      float s = 0.0f;
      const bool on = tid + i * THREADS < nv;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        ex[i][e] = __builtin_amdgcn_exp2f((in[i].get(e) - zm) * c);
        s += ex[i][e];
      }
      if (on) ze += s;
    }
    zx = __builtin_amdgcn_exp2f((zx - zm) * c);
    if (own >= 0) ze += zx;
  } else {
    // of a thread without a value above -inf 0 or NaN, which the factor 0 keeps; of a
    // row without one NaN
    ze = zm == -__builtin_inff() ? __builtin_nan("") : ze * __builtin_amdgcn_exp2f((own_max - zm) * c);
    zx = __builtin_amdgcn_exp2f((zx - zm) * c);
    if (own >= 0) ze += zx;
  }
  double te = 0.0;
  for (int j = tid; j < K; j += THREADS)
    if (en.idx[j] >= 0) {
      const double x = exp((en.p[j] - tm) * inv);
      te += x;
    }
  te = wave_sum_f64(te);
  ze = wave_sum_f64(ze);
  if (lane == 0) {
    sl.te[wave] = te;
    sl.ze[wave] = ze;
  }
  __syncthreads();
  te = sum_of<W>(sl.te);
  ze = sum_of<W>(sl.ze);

  // --- the loss, and p in place of t
  double loss = 0.0;
  if (wave * kWave < K) {
    const double lt = log(te), lz = log(ze);
    for (int j = tid; j < K; j += THREADS)
      if (en.idx[j] >= 0) {
        const double u = (en.p[j] - tm) * inv, p = exp(u) / te;
        if (!(p == 0.0)) loss += p * (u - lt - ((static_cast<double>(en.z[j]) - zm) * inv - lz));
        en.p[j] = p;
      }
  }
  if (a.loss != nullptr) {
    loss = wave_sum_f64(loss);
    if (lane == 0) sl.loss[wave] = loss;
  }

  // --- the gradient of the row
  const double wt = static_cast<double>(w) * a.tau;
  const float g = static_cast<float>(wt / ze);
  const auto put = [&](int i, float y) {
    if (w == 0.0f) y = 0.0f;
    if constexpr (sizeof(D) == 4) dz[i] = y;
    else dz[i] = static_cast<uint16_t>(pack_bf16(y, 0.0f));
  };
  if (dz != nullptr) {
    const bool zero = w == 0.0f;
    const auto vec = [&](int v, const float* x) {
      float y[E];
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = zero ? 0.0f : x[e] * g;
      RowVec<D, E> o;
      o.set(y);
      o.template store<NT>(dz + head, v);
    };
    if constexpr (HELD > 0) {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (tid + i * THREADS < nv) vec(tid + i * THREADS, ex[i]);
    } else {
      for (int v = tid; v < nv; v += THREADS) {
        RowVec<T, E> x;
        x.load(rz, v);
        float y[E];
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = __builtin_amdgcn_exp2f((x.get(e) - zm) * c);
        vec(v, y);
      }
    }
    if (own >= 0) put(own, zx * g);
  }
  __syncthreads();
  if (tid == 0 && a.loss != nullptr) a.loss[m] = static_cast<float>(sum_of<W>(sl.loss) * a.tau * a.tau);
  if (dz == nullptr) return;
  // --- and at the teacher's tokens
  for (int j = tid, n = 0; j < K; j += THREADS, ++n) {
    const int i = en.idx[j];
    if (i < 0) continue;
    double p = en.p[j];
    if ((twice >> n) & 1) {  // the lowest entry of a token for all of them
      bool first = true;
      p = 0.0;
      scan(en, K, i, [&](int k, bool is) {
        if (is) {
          first &= k >= j;
          p += en.p[k];
        }
      });
      if (!first) continue;
    }
    put(i, static_cast<float>((__builtin_amdgcn_exp2f((en.z[j] - zm) * c) / ze - p) * wt));
  }
}

template <typename T, typename D, bool NT>
hipError_t launch(const DistillArgs& a, hipStream_t stream) {
  const auto go = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(a.M)), dim3(threads), entries_room(static_cast<int>(a.K)) * kEntryBytes, stream, a);
    return hipGetLastError();
  };
  // The fewest threads that hold a row in registers: a row's steps wait for one
  // another, and the rows beside it on a compute unit hide that (8192 bf16 rows, 16
  // entries: of 1000 in 64 threads 18 us, in 256 30; of 2000 22, 31; of 4000 in 128
  // 34, in 256 39; of 8000 in 128 or 256 57; of 16000 in 256 95, in 512 105; of 32000
  // in 512 200, in 1024 273.  64 rows: equal to a tenth).
  const int64_t nv = a.V / 8;  // the most whole vectors of a row
  if (nv <= 2 * 64) return go(distill_kernel<T, D, 64, 2, NT>, 64);
  if (nv <= 4 * 64) return go(distill_kernel<T, D, 64, 4, NT>, 64);
  if (nv <= 4 * 128) return go(distill_kernel<T, D, 128, 4, NT>, 128);
  if (nv <= 8 * 128) return go(distill_kernel<T, D, 128, 8, NT>, 128);
  if (nv <= 8 * 256) return go(distill_kernel<T, D, 256, 8, NT>, 256);
  if (NT || nv <= 8 * 512) return go(distill_kernel<T, D, 512, 8, NT>, 512);
  if constexpr (!NT) {
    // one such row fills a compute unit's registers; of bf16, reading it again costs
    // less than that (1024 rows of 36000 37 against 49 us, 4096 of 50001 203 against
    // 218), of fp32 more (2048 of 50001 201 against 185)
    if constexpr (sizeof(T) == 4)
      if (nv <= 8 * 1024) return go(distill_kernel<T, D, 1024, 8, false>, 1024);
    return go(distill_kernel<T, D, 1024, 0, false>, 1024);
  }
}

}  // namespace

hipError_t launch_distill(const DistillArgs& a, hipStream_t stream) {
  // the loss alone: D does not matter
  const bool d32 = a.dz != nullptr && a.dz_is_f32;
  if (a.z_is_f32) return d32 ? launch<float, float, false>(a, stream) : launch<float, uint16_t, false>(a, stream);
  // Streams pass the caches where the arrays fill the last of them, of bf16 (8192
  // rows of 32000: 186 against 200 us, of 16000 117 against 112; fp32 loses by it,
  // 2048 rows of 50001 224 against 185), and not where a row is read again.
  const int64_t bytes = a.M * a.V * (2 + (a.dz == nullptr ? 0 : d32 ? 4 : 2));
  const bool nt = bytes >= kLastLevelBytes && a.V / 8 <= 8 * 512;
  if (d32) return nt ? launch<uint16_t, float, true>(a, stream) : launch<uint16_t, float, false>(a, stream);
  return nt ? launch<uint16_t, uint16_t, true>(a, stream) : launch<uint16_t, uint16_t, false>(a, stream);
}

}  // namespace mmf
