// Vectors of E consecutive row values in registers, read through buffer
// resources of the row's size: a vector past the row's end reads as zero with
// no memory access and no branch, so that every load of a row can be issued
// at once (guarded loads would each wait for the last).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mmf_device.h"

namespace mmf {

typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

// Two values rounded to bf16 (nearest even; NaN stays NaN), in one dword.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{a, b}, v2bf));
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// The resource of one row of K values; `on` false: of size 0.  Row pointers
// are wave-uniform.
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_rsrc(const T* row, int K, bool on) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(row), 0, on ? K * static_cast<int>(sizeof(T)) : 0,
                                           kBufferWord3);
}

// Streams.  A call whose arrays together fill the last-level cache (256 MB)
// reads and writes them without leaving them there (nontemporal: nothing of
// them would still be there for their next reader, and taking a line in pushes
// another out, which goes to memory first if it was written).  Smaller ones
// stay for their next reader.  Rows too long for registers are read through
// the caches always: the call reads them again.
constexpr int64_t kLastLevelBytes = int64_t(256) << 20;
constexpr int kNontemporal = 2;  // buffer cache policy: the nt bit

// load_words with the stream's cache policy.
template <int F, bool NT>
__device__ __forceinline__ Words<F> load_stream(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  constexpr int kPolicy = NT ? kNontemporal : 0;
  Words<F> p;
  if constexpr (F == 2) {
    const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, kPolicy));
    p.w[0] = v.x;
    p.w[1] = v.y;
  } else {
    static_assert(F == 4, "two or four words");
    const uint4 v = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, kPolicy));
    p.w[0] = v.x;
    p.w[1] = v.y;
    p.w[2] = v.z;
    p.w[3] = v.w;
  }
  return p;
}

// E values of T (uint16_t: bf16 bits, or float) of a row, from value E v.
template <typename T, int E>
struct RowVec {
  static_assert(E == 4 || E == 8, "8 to 32 bytes");
  static constexpr int kWords = E * static_cast<int>(sizeof(T)) / 4;
  static constexpr int kLoad = kWords < 4 ? kWords : 4;  // dwords per load
  uint32_t w[kWords];

  template <bool NT = false>
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int v) {
#pragma unroll
    for (int i = 0; i < kWords; i += kLoad) {
      const Words<kLoad> p = load_stream<kLoad, NT>(r, static_cast<uint32_t>(v) * (4u * kWords) + 4u * i);
#pragma unroll
      for (int j = 0; j < kLoad; ++j) w[i + j] = p.w[j];
    }
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    return e & 1 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
  }
  // The values rounded to T.
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f[i]);
      else w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
    }
  }
  // Values of -0, which x + v leaves any x as it is (+0 would turn -0 into +0).
  __device__ __forceinline__ void set_negative_zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
  }
  template <bool NT = false>
  __device__ __forceinline__ void store(T* row, int v) const {
    typedef unsigned int vec __attribute__((ext_vector_type(kLoad)));
    vec* const p = reinterpret_cast<vec*>(row + static_cast<int64_t>(v) * E);
#pragma unroll
    for (int i = 0; i < kWords / kLoad; ++i) {
      vec x;
#pragma unroll
      for (int j = 0; j < kLoad; ++j) x[j] = w[i * kLoad + j];
      if constexpr (NT) __builtin_nontemporal_store(x, p + i);
      else p[i] = x;
    }
  }
};

// All-reduction of a per-lane value over the W waves of a row: the wave's own
// total through `wave_total`, then the waves' totals in wave order through
// `slot` (one value per wave of the block).  Two calls of one block must use
// different slots unless a barrier lies between them.
template <int W, typename T, typename F>
__device__ __forceinline__ T row_combine(T wave_total, T* slot, int wave, F&& op) {
  if constexpr (W == 1) {
    return wave_total;
  } else {
    if ((threadIdx.x & 63) == 0) slot[wave] = wave_total;
    __syncthreads();
    const int first = wave / W * W;
    T t = slot[first];
#pragma unroll
    for (int i = 1; i < W; ++i) t = op(t, slot[first + i]);
    return t;
  }
}

}  // namespace mmf
