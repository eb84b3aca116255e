// Residual addition + RMSNorm + per-token absmax int8 quantisation, and its
// backward.
//
// Forward, per token row: s = x + branch (fp32, stored in the type of x), then
// the quantisation of the stored sum exactly as act_quant.hip does it.  The
// row is read once and stays in registers through its three statistics.
//
// Backward (straight through the quantiser): with y = (s r) gamma and the
// gradient dY of y,
//   ds = r g - (r^3 t / K) s + ds_out,  g = gamma dY,  t = sum_k g_k s_k,
//   dgamma = sum over rows of dY s r.
//
// Both are streams, bound by HBM.  Forward: 9 bytes per element with a bf16
// stream and an fp32 branch; 16384 x 5120 in 123 us (6.1 TB/s; cached accesses
// instead of streams 132), one row of 2048 in 2.6 us (the launch and three
// reductions).  Backward: 16 bytes with bf16 s and fp32 gradients; 8192 x 2048
// in 47 us (5.7 TB/s) and 4.5 us for the sums of dgamma's 256 partial rows.
// Medians of 61 calls one behind the other; the fastest took 114 and 45 us.
#include "mmf_device.h"
#include "mmf_launch.h"
#include "row_vec.h"

namespace mmf {
namespace {

constexpr int64_t kMaxBlocks = int64_t(1) << 20;  // rows past them: further passes of the row loop
constexpr int kOneWaveK = kWave * 32;             // longest row of one wave

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
struct FwdArgs {
  const void* x;
  const void* branch;  // nullptr: none
  const float* gamma;
  void* s;             // nullptr (without a branch): not stored
  int8_t* q;
  float* a_scale;
  int32_t* q_rowsum;
  float* rstd;
  int64_t M;
  int K;
};

// One row per W waves, VPL vectors of E values per lane (VPL == 0: any K, the
// stored sum read again for each further pass).  x and s may be the same
// array: every element is read and written by one lane.  NT: x, branch and s
// as streams (q stays for the contraction).
template <typename XT, typename BT, int E, int W, int VPL, bool NT>
__global__ __launch_bounds__(kWave*(W > 4 ? W : 4)) void add_quant_kernel(const FwdArgs a) {
  constexpr int kBlockWaves = W > 4 ? W : 4;
  constexpr int kRows = kBlockWaves / W;
  __shared__ double s_ss[kBlockWaves];
  __shared__ float s_amax[kBlockWaves];
  __shared__ int s_rs[kBlockWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rl = (wave % W) * kWave + (threadIdx.x & 63);  // lane within the row
  const int K = a.K, nvec = K / E;
  const XT* const x = static_cast<const XT*>(a.x);
  const BT* const branch = static_cast<const BT*>(a.branch);
  XT* const sum = static_cast<XT*>(a.s);
  const __amdgpu_buffer_rsrc_t grsrc = row_rsrc(a.gamma, K, a.gamma != nullptr);
  const auto addd = [](double u, double v) { return u + v; };
  const auto addi = [](int u, int v) { return u + v; };
  const auto maxf = [](float u, float v) { return fmaxf(u, v); };

  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * kRows; r0 < a.M; r0 += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t row = r0 + wave / W;
    const bool live = row < a.M;  // uniform per wave
    const int64_t at = (live ? row : 0) * K;
    int8_t* const qr = a.q + at;
    const __amdgpu_buffer_rsrc_t xrsrc = row_rsrc(x + at, K, live);
    const __amdgpu_buffer_rsrc_t brsrc = row_rsrc(branch == nullptr ? branch : branch + at, K, live && branch != nullptr);
    float r, amax = 0.0f;
    int rs = 0;
    auto quantise = [&](int v, const float* y, float sc) {
      uint32_t w[E / 4];
#pragma unroll
      for (int i = 0; i < E / 4; ++i) {
        w[i] = quantise4(y + 4 * i, sc);
        rs = byte_sum4(w[i], rs);
      }
      if constexpr (E == 8) *reinterpret_cast<uint2*>(qr + v * E) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<uint32_t*>(qr + v * E) = w[0];
    };
    if constexpr (VPL > 0) {
      RowVec<XT, E> xv[VPL];
      RowVec<BT, E> bv[VPL];
      RowVec<float, E> gv[VPL];
#pragma unroll
      for (int i = 0; i < VPL; ++i) xv[i].template load<NT>(xrsrc, rl + W * kWave * i);
#pragma unroll
      for (int i = 0; i < VPL; ++i) bv[i].template load<NT>(brsrc, rl + W * kWave * i);
#pragma unroll
      for (int i = 0; i < VPL; ++i) gv[i].load(grsrc, rl + W * kWave * i);
      __builtin_amdgcn_sched_barrier(0);  // all loads before the first wait
      if (branch == nullptr) {  // uniform
#pragma unroll
        for (int i = 0; i < VPL; ++i) bv[i].set_negative_zero();
      }
      double ss = 0.0;
      float f[VPL][E];
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int v = rl + W * kWave * i;
#pragma unroll
        for (int e = 0; e < E; ++e) f[i][e] = xv[i].get(e) + bv[i].get(e);
        xv[i].set(f[i]);
        if (sum != nullptr && live && v < nvec) xv[i].template store<NT>(sum + at, v);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          f[i][e] = xv[i].get(e);  // the stored value
          ss = sum_sq(ss, f[i][e]);
        }
      }
      ss = row_combine<W>(wave_sum_f64(ss), s_ss, wave, addd);
      r = rms_rstd(ss, K);
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          f[i][e] = f[i][e] * r;
          if (a.gamma != nullptr) f[i][e] = f[i][e] * gv[i].get(e);
          amax = fmaxf(amax, fabsf(f[i][e]));
        }
      amax = fmaxf(row_combine<W>(wave_max_f32(amax), s_amax, wave, maxf), 1e-5f);
      const float sc = 127.0f / amax;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int v = rl + W * kWave * i;
        if (live && v < nvec) quantise(v, f[i], sc);
      }
    } else {
      // each lane reads back the sums that it stored itself
      const XT* const src = sum != nullptr ? sum + at : x + at;
      double ss = 0.0;
      for (int v = rl; v < nvec; v += W * kWave) {
        RowVec<XT, E> xv;
        RowVec<BT, E> bv;
        xv.load(xrsrc, v);
        bv.load(brsrc, v);
        if (branch == nullptr) bv.set_negative_zero();
        float f[E];
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = xv.get(e) + bv.get(e);
        xv.set(f);
        if (sum != nullptr && live) xv.store(sum + at, v);
#pragma unroll
        for (int e = 0; e < E; ++e) ss = sum_sq(ss, xv.get(e));
      }
      ss = row_combine<W>(wave_sum_f64(ss), s_ss, wave, addd);
      r = rms_rstd(ss, K);
      auto normed = [&](int v, float* f) {
        RowVec<float, E> gv;
        gv.load(grsrc, v);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if constexpr (sizeof(XT) == 4) f[e] = src[v * E + e];
          else f[e] = bf16_to_f32(src[v * E + e]);
          f[e] = f[e] * r;
          if (a.gamma != nullptr) f[e] = f[e] * gv.get(e);
        }
      };
      for (int v = rl; live && v < nvec; v += W * kWave) {
        float f[E];
        normed(v, f);
#pragma unroll
        for (int e = 0; e < E; ++e) amax = fmaxf(amax, fabsf(f[e]));
      }
      amax = fmaxf(row_combine<W>(wave_max_f32(amax), s_amax, wave, maxf), 1e-5f);
      const float sc = 127.0f / amax;
      for (int v = rl; live && v < nvec; v += W * kWave) {
        float f[E];
        normed(v, f);
        quantise(v, f, sc);
      }
    }
    rs = row_combine<W>(wave_sum_i32(rs), s_rs, wave, addi);
    if (live && rl == 0) {
      a.a_scale[row] = amax / 127.0f;
      if (a.q_rowsum != nullptr) a.q_rowsum[row] = rs;
      if (a.rstd != nullptr) a.rstd[row] = r;
    }
    if constexpr (W > 1) __syncthreads();  // the slots are the next row's
  }
}

template <typename XT, typename BT, int E, int W, int VPL>
hipError_t launch_fwd_one(const FwdArgs& a, hipStream_t stream) {
  constexpr int kBlockWaves = W > 4 ? W : 4;
  constexpr int kRows = kBlockWaves / W;
  const int64_t blocks = (a.M + kRows - 1) / kRows;
  const dim3 grid(static_cast<unsigned>(blocks < kMaxBlocks ? blocks : kMaxBlocks));
  // as streams: rows in registers, and not the few short ones that share four waves
  constexpr bool kStream = VPL > 0 && !(W == 4 && W * kWave * VPL * E <= kOneWaveK);
  if (kStream && a.M * a.K * static_cast<int64_t>(2 * sizeof(XT) + sizeof(BT) + 1) >= kLastLevelBytes)
    hipLaunchKernelGGL((add_quant_kernel<XT, BT, E, W, VPL, kStream>), grid, dim3(kWave * kBlockWaves), 0, stream, a);
  else
    hipLaunchKernelGGL((add_quant_kernel<XT, BT, E, W, VPL, false>), grid, dim3(kWave * kBlockWaves), 0, stream, a);
  return hipGetLastError();
}

// The smallest compiled number of vectors per lane that holds the row (loads
// past the row's end return zeros but cost nearly a real load each); 16 waves
// have rows of more than 8192.
template <typename XT, typename BT, int E, int W>
hipError_t launch_fwd_w(const FwdArgs& a, hipStream_t stream) {
  const int vpl = (a.K / E + W * kWave - 1) / (W * kWave);
  if constexpr (W < 16) {
    if (vpl == 1) return launch_fwd_one<XT, BT, E, W, 1>(a, stream);
  }
  if constexpr (W < 16 || E == 8) {
    if (vpl == 2) return launch_fwd_one<XT, BT, E, W, 2>(a, stream);
  }
  switch (vpl) {
    case 3: return launch_fwd_one<XT, BT, E, W, 3>(a, stream);
    case 4: return launch_fwd_one<XT, BT, E, W, 4>(a, stream);
    default: break;
  }
  if constexpr (E == 4) {
    switch (vpl) {
      case 5: return launch_fwd_one<XT, BT, E, W, 5>(a, stream);
      case 6: return launch_fwd_one<XT, BT, E, W, 6>(a, stream);
      case 7: case 8: return launch_fwd_one<XT, BT, E, W, 8>(a, stream);
      default: break;
    }
  }
  if constexpr (W == 16) return launch_fwd_one<XT, BT, E, W, 0>(a, stream);
  return hipErrorInvalidValue;
}

// Waves per row: up to 32 values per lane (K <= 32768; what 16 waves hold in
// their 128 registers spills by up to 12 of them).  Up to a row per compute
// unit, four waves share a row of more than two vectors per lane, which one
// wave would keep to itself (1 and 4 waves, us, bf16 stream and fp32 branch,
// launches replayed back to back; fp32 streams alike):
//   K = 1024: 1 row 2.82 / 2.58, 64 3.14 / 2.96, 256 3.73 / 3.37, 512 3.97 / 3.87, 2048 7.21 / 8.07
//   K = 2048: 1 row 3.62 / 2.83, 64 3.98 / 3.21, 256 4.72 / 4.04, 512 5.08 / 4.82, 2048 10.1 / 10.4
//   K = 528:  1 row 2.65 / 2.64, 64 2.96 / 3.04, 256 3.22 / 3.24, 512 3.57 / 3.67, 2048 5.79 / 7.24
//   K = 1024, all bf16 (two vectors): 1 row 2.63 / 2.68, 64 2.93 / 3.04, 2048 6.57 / 8.00
// 16 in place of 4 never gain (K = 5120: 1 row 3.55 / 4.13, 64 4.50 / 4.97;
// K = 8192: 4.04 / 4.15 and 5.12 / 5.10).
// bf16 streams with fp32 branches go four values at a time (8-byte and 16-byte
// loads side by side), bf16 with bf16 eight.
constexpr int64_t kFewRows = 256;
template <typename XT, typename BT, int E>
hipError_t launch_fwd(const FwdArgs& a, hipStream_t stream) {
  int w = a.K <= kOneWaveK ? 1 : a.K <= 4 * kOneWaveK ? 4 : 16;
  if (w == 1 && a.M <= kFewRows && a.K > 2 * kWave * E) w = 4;
  if (w == 1) return launch_fwd_w<XT, BT, E, 1>(a, stream);
  if (w == 4) return launch_fwd_w<XT, BT, E, 4>(a, stream);
  return launch_fwd_w<XT, BT, E, 16>(a, stream);
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
struct BwdArgs {
  const void* dy;
  const float* ds_out;  // nullptr: zero; may be ds
  const void* s;
  const float* gamma;
  const float* rstd;
  float* ds;
  uint16_t* ds_bf16;    // nullptr: not stored
  double* dg_part;      // [gridDim.x][K], nullptr: not computed
  int64_t M;
  int K;
};

// Workgroups of W waves, each taking rows blockIdx.x, + gridDim.x, ...; every
// lane owns the same columns of each row and keeps their gamma and their
// dgamma sums (fp64) in registers.  The next row's loads are in flight while
// a row is reduced and written (not with 16 waves, whose 128 registers hold
// one row only).  VPL == 0: any K; the row is read twice and the column sums
// are kept in dg_part.  NT: every array but gamma and the sums as streams.
template <typename ST, typename DT, int E, int W, int VPL, bool NT>
__global__ __launch_bounds__(kWave* W) void add_quant_bwd_kernel(const BwdArgs a) {
  __shared__ double s_t[2][W];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rl = threadIdx.x;
  const int K = a.K, nvec = K / E;
  const DT* const dy = static_cast<const DT*>(a.dy);
  const ST* const s = static_cast<const ST*>(a.s);
  const __amdgpu_buffer_rsrc_t grsrc = row_rsrc(a.gamma, K, a.gamma != nullptr);
  const auto addd = [](double u, double v) { return u + v; };
  double* const part = a.dg_part == nullptr ? nullptr : a.dg_part + static_cast<int64_t>(blockIdx.x) * K;
  auto coef = [&](double t, float r) {
    const double rd = static_cast<double>(r);
    return static_cast<float>(rd * rd * rd * t / static_cast<double>(K));
  };
  auto emit = [&](int64_t at, int v, const float* o) {
    RowVec<float, E> ov;
    ov.set(o);
    ov.template store<NT>(a.ds + at, v);
    if (a.ds_bf16 != nullptr) {
      RowVec<uint16_t, E> hv;
      hv.set(o);
      hv.template store<NT>(a.ds_bf16 + at, v);
    }
  };
  int parity = 0;
  if constexpr (VPL > 0) {
    struct Row {
      RowVec<DT, E> dy[VPL];
      RowVec<ST, E> s[VPL];
      RowVec<float, E> res[VPL];
      float r;
    };
    auto load = [&](Row& w, int64_t row) {
      const bool live = row < a.M;
      const int64_t at = (live ? row : 0) * K;
      const __amdgpu_buffer_rsrc_t drsrc = row_rsrc(dy + at, K, live), srsrc = row_rsrc(s + at, K, live);
      const __amdgpu_buffer_rsrc_t orsrc =
          row_rsrc(a.ds_out == nullptr ? a.ds_out : a.ds_out + at, K, live && a.ds_out != nullptr);
#pragma unroll
      for (int i = 0; i < VPL; ++i) w.dy[i].template load<NT>(drsrc, rl + W * kWave * i);
#pragma unroll
      for (int i = 0; i < VPL; ++i) w.s[i].template load<NT>(srsrc, rl + W * kWave * i);
#pragma unroll
      for (int i = 0; i < VPL; ++i) w.res[i].template load<NT>(orsrc, rl + W * kWave * i);
      w.r = a.rstd[live ? row : 0];
    };
    RowVec<float, E> gv[VPL];
    double dg[VPL][E];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      gv[i].load(grsrc, rl + W * kWave * i);
#pragma unroll
      for (int e = 0; e < E; ++e) dg[i][e] = 0.0;
    }
    if (a.gamma == nullptr) {  // uniform
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) gv[i].w[e] = __float_as_uint(1.0f);
    }
    constexpr bool kAhead = W < 16;
    Row cur;
    if constexpr (kAhead) load(cur, blockIdx.x);
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
      Row next;
      load(kAhead ? next : cur, row + (kAhead ? gridDim.x : 0));
      __builtin_amdgcn_sched_barrier(0);
      const int64_t at = row * K;
      double t = 0.0;
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float d = cur.dy[i].get(e), sv = cur.s[i].get(e);
          t += static_cast<double>(gv[i].get(e) * d) * static_cast<double>(sv);
          dg[i][e] += static_cast<double>(d * (sv * cur.r));
        }
      t = row_combine<W>(wave_sum_f64(t), s_t[parity], wave, addd);
      parity ^= 1;
      const float c = coef(t, cur.r);
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int v = rl + W * kWave * i;
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e)
          o[e] = (cur.r * (gv[i].get(e) * cur.dy[i].get(e)) - c * cur.s[i].get(e)) + cur.res[i].get(e);
        if (v < nvec) emit(at, v, o);
      }
      if constexpr (kAhead) cur = next;
    }
    if (part != nullptr) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int v = rl + W * kWave * i;
        if (v < nvec) {
#pragma unroll
          for (int e = 0; e < E; e += 2)
            *reinterpret_cast<double2*>(part + v * E + e) = make_double2(dg[i][e], dg[i][e + 1]);
        }
      }
    }
  } else {
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
      const int64_t at = row * K;
      const __amdgpu_buffer_rsrc_t drsrc = row_rsrc(dy + at, K, true), srsrc = row_rsrc(s + at, K, true);
      const __amdgpu_buffer_rsrc_t orsrc = row_rsrc(a.ds_out == nullptr ? a.ds_out : a.ds_out + at, K, a.ds_out != nullptr);
      const float r = a.rstd[row];
      double t = 0.0;
      for (int v = rl; v < nvec; v += W * kWave) {
        RowVec<DT, E> dv;
        RowVec<ST, E> sv;
        RowVec<float, E> gv;
        dv.load(drsrc, v);
        sv.load(srsrc, v);
        gv.load(grsrc, v);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float g = a.gamma != nullptr ? gv.get(e) * dv.get(e) : dv.get(e);
          t += static_cast<double>(g) * static_cast<double>(sv.get(e));
        }
      }
      t = row_combine<W>(wave_sum_f64(t), s_t[parity], wave, addd);
      parity ^= 1;
      const float c = coef(t, r);
      for (int v = rl; v < nvec; v += W * kWave) {
        RowVec<DT, E> dv;
        RowVec<ST, E> sv;
        RowVec<float, E> gv, rv;
        dv.load(drsrc, v);
        sv.load(srsrc, v);
        gv.load(grsrc, v);
        rv.load(orsrc, v);
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float g = a.gamma != nullptr ? gv.get(e) * dv.get(e) : dv.get(e);
          o[e] = (r * g - c * sv.get(e)) + rv.get(e);
          if (part != nullptr) {
            const double dg = static_cast<double>(dv.get(e) * (sv.get(e) * r));
            part[v * E + e] = (row == blockIdx.x ? 0.0 : part[v * E + e]) + dg;
          }
        }
        emit(at, v, o);
      }
    }
  }
}

template <typename ST, typename DT, int E, int W>
hipError_t launch_bwd_w(const BwdArgs& a, unsigned blocks, hipStream_t stream) {
  const int vpl = (a.K / E + W * kWave - 1) / (W * kWave);
  const int64_t bytes = sizeof(ST) + sizeof(DT) + (a.ds_out ? 4 : 0) + 4 + (a.ds_bf16 ? 2 : 0);
  const bool nt = a.M * a.K * bytes >= kLastLevelBytes;
#define MMF_LAUNCH(V)                                                                                                \
  do {                                                                                                               \
    if (nt)                                                                                                          \
      hipLaunchKernelGGL((add_quant_bwd_kernel<ST, DT, E, W, V, true>), dim3(blocks), dim3(kWave * W), 0, stream, a); \
    else                                                                                                             \
      hipLaunchKernelGGL((add_quant_bwd_kernel<ST, DT, E, W, V, false>), dim3(blocks), dim3(kWave * W), 0, stream, a); \
  } while (0)
  constexpr int kLeast = W == 1 ? 1 : W == 4 ? 2 : 3;  // of the rows that bwd_waves gives W waves
  switch (vpl) {
    case 1:
      if constexpr (kLeast <= 1) MMF_LAUNCH(1);
      else return hipErrorInvalidValue;
      break;
    case 2:
      if constexpr (kLeast <= 2) MMF_LAUNCH(2);
      else return hipErrorInvalidValue;
      break;
    case 3: MMF_LAUNCH(3); break;
    case 4: MMF_LAUNCH(4); break;
    default:
      if constexpr (W == 16) MMF_LAUNCH(0);
      else return hipErrorInvalidValue;
  }
#undef MMF_LAUNCH
  return hipGetLastError();
}

// Waves per row: at most 16 values per lane (gamma, the fp64 column sums and
// two rows of operands are all in registers).
int bwd_waves(int K) {
  int w = 1;
  while (w < 16 && K > w * kWave * 16) w *= w == 1 ? 4 : 2;
  return w;
}

template <typename ST, typename DT>
hipError_t launch_bwd(const BwdArgs& a, unsigned blocks, hipStream_t stream) {
  switch (bwd_waves(a.K)) {
    case 1: return launch_bwd_w<ST, DT, 4, 1>(a, blocks, stream);
    case 4: return launch_bwd_w<ST, DT, 4, 4>(a, blocks, stream);
    case 8: return launch_bwd_w<ST, DT, 4, 8>(a, blocks, stream);
    default: return launch_bwd_w<ST, DT, 4, 16>(a, blocks, stream);
  }
}

}  // namespace

hipError_t launch_add_quant(const AddQuantArgs& p, hipStream_t stream) {
  if (p.M == 0) return hipSuccess;
  const FwdArgs a{p.x, p.branch, p.gamma, p.s, p.q, p.a_scale, p.q_rowsum, p.rstd, p.M, p.K};
  if (p.x_is_f32)
    return p.branch_is_f32 ? launch_fwd<float, float, 4>(a, stream) : launch_fwd<float, uint16_t, 4>(a, stream);
  return p.branch_is_f32 ? launch_fwd<uint16_t, float, 4>(a, stream) : launch_fwd<uint16_t, uint16_t, 8>(a, stream);
}

// Workgroups of the backward, each with a row of column sums: one wave per
// SIMD over 256 compute units, or one workgroup of more waves per unit (twice
// as many: 8192 x 2048 53 instead of 50 us, 8192 x 1024 31 instead of 28; half
// as many: 71 and 26), and for few rows at least two rows each, from 512 rows
// on towards four (1000 x 1024 with a row each 15.9 us, two 11.8, four 10.9,
// eight 13.0; 300 x 2048 9.8, 8.7, 9.1, 11.6).
int64_t add_quant_bwd_parts(int64_t M, int K) {
  const int w = bwd_waves(K);
  const int64_t most = w <= 4 ? 1024 / w : 256;
  const int64_t two = (M + 1) / 2 < 256 ? (M + 1) / 2 : 256;
  const int64_t few = (M + 3) / 4 > two ? (M + 3) / 4 : two;
  return few < most ? few : most;
}

hipError_t launch_add_quant_bwd(const AddQuantBwdArgs& p, hipStream_t stream) {
  if (p.M == 0) return hipSuccess;
  const BwdArgs a{p.dy, p.ds_out, p.s, p.gamma, p.rstd, p.ds, p.ds_bf16, p.dg_part, p.M, p.K};
  const unsigned blocks = static_cast<unsigned>(add_quant_bwd_parts(p.M, p.K));
  if (p.s_is_f32)
    return p.dy_is_f32 ? launch_bwd<float, float>(a, blocks, stream) : launch_bwd<float, uint16_t>(a, blocks, stream);
  return p.dy_is_f32 ? launch_bwd<uint16_t, float>(a, blocks, stream)
                     : launch_bwd<uint16_t, uint16_t>(a, blocks, stream);
}

}  // namespace mmf
