// Linear attention over chunks: how a pass is cut into segments, the joining
// of the segments' states, and the passes of the forward.
#include "linattn.h"
#include "mmf_device.h"

namespace mmf {

hipError_t launch_linattn_f32(const LinattnPass& p, bool state, hipStream_t stream);
hipError_t launch_linattn_bf16(const LinattnPass& p, bool state, hipStream_t stream);
hipError_t launch_linattn_bwd_bf16(const LinattnPass& p, hipStream_t stream);
hipError_t launch_linattn_bwd_f32(const LinattnPass& p, hipStream_t stream);
hipError_t launch_linattn_bwd_any(const LinattnPass& p, bool state, hipStream_t stream);

namespace {

constexpr int64_t kCus = 256;
constexpr int kJoinBlock = 256, kJoinAhead = 8;

__device__ __forceinline__ double power(double x, int64_t n) {
  double y = 1.0;
  for (; n != 0; n >>= 1) {
    if (n & 1) y *= x;
    x *= x;
  }
  return y;
}

// joined[seg] <- the state that enters segment seg: E_0 from s_in (with its
// decay to the first token, forward), E_{seg+1} = l^tokens E_seg + joined[seg].
__global__ __launch_bounds__(kJoinBlock) void linattn_join_kernel(const LinattnPass p) {
  const int64_t size = static_cast<int64_t>(p.Dk) * p.Dv;
  const uint32_t per = static_cast<uint32_t>((size + kJoinBlock - 1) / kJoinBlock);
  const int64_t bh = blockIdx.x / per;
  const int64_t at = static_cast<int64_t>(blockIdx.x % per) * kJoinBlock + threadIdx.x;
  if (at >= size) return;
  const double l = p.decay[bh % p.H];
  const float w = static_cast<float>(power(l, p.seg_tokens));
  float e = 0.0f;
  if (p.s_in != nullptr) {
    e = p.s_in[bh * size + at / p.Dv * p.in_d + at % p.Dv * p.in_e];
    if (!p.rev) e *= p.decay[bh % p.H];
  }
  float* const u = p.joined + bh * p.nseg * size + at;
  float last = 0.0f;
  if (p.join_last) last = u[(p.nseg - 1) * size];
  for (uint32_t s = 0; s < p.nseg; s += kJoinAhead) {
    float v[kJoinAhead];
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) v[i] = s + i + 1 < p.nseg ? u[(s + i) * size] : 0.0f;
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) {
      if (s + i >= p.nseg) break;
      u[(s + i) * size] = e;
      if (s + i + 1 < p.nseg) e = fmaf(w, e, v[i]);
    }
  }
  if (p.join_last) {
    const float wl = static_cast<float>(power(l, p.T - (p.nseg - 1) * p.seg_tokens));
    p.s_out[bh * size + at / p.Dv * p.in_d + at % p.Dv * p.in_e] = fmaf(wl, e, last);
  }
}

}  // namespace

LinattnPlan linattn_plan(int64_t B, int64_t T, int64_t H, int Dk, int Dv) {
  LinattnPlan plan;
  plan.et = Dv <= 64 || Dk > 128 ? 1 : 2;
  plan.tiles = static_cast<uint32_t>((Dv + 64 * plan.et - 1) / (64 * plan.et));
  const int64_t C = Dk > 128 ? 32 : 64;
  const int64_t chunks = (T + C - 1) / C, groups = B * H * plan.tiles;
  // rounds of workgroups x chunks of a segment, half as much again for the
  // segments' own sums
  int64_t best = 1, cost = ((groups + kCus - 1) / kCus) * chunks * 2;
  for (int64_t s = 2; s <= chunks && groups * (s - 1) < 4 * kCus; ++s) {
    const int64_t per = (chunks + s - 1) / s;
    const int64_t c = ((groups * s + kCus - 1) / kCus) * per * 3 + 4;
    if (c < cost) {
      best = s;
      cost = c;
    }
  }
  const int64_t per = (chunks + best - 1) / best;
  plan.nseg = static_cast<uint32_t>((chunks + per - 1) / per);
  plan.seg_tokens = per * C;
  plan.joined_bytes = sizeof(float) * static_cast<size_t>(B * H) * plan.nseg * Dk * Dv;
  return plan;
}

namespace {

LinattnPass with_plan(LinattnPass p, const LinattnPlan& plan, float* joined) {
  p.nseg = plan.nseg;
  p.tiles = plan.tiles;
  p.et = plan.et;
  p.seg_tokens = plan.seg_tokens;
  p.joined = plan.nseg > 1 || p.join_last ? joined : nullptr;
  return p;
}

hipError_t join(const LinattnPass& p, hipStream_t stream) {
  const uint32_t per = static_cast<uint32_t>((static_cast<int64_t>(p.Dk) * p.Dv + kJoinBlock - 1) / kJoinBlock);
  hipLaunchKernelGGL(linattn_join_kernel, dim3(p.B * p.H * per), dim3(kJoinBlock), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linattn_chunk(const LinattnArgs& a, float* joined, hipStream_t stream) {
  const int64_t size = a.is_f32 ? 4 : 2, ld = a.H * (2 * a.dk + a.dv);
  const char* const x = static_cast<const char*>(a.qkv);
  LinattnPass p{};
  p.q = {x, ld, a.is_f32};
  p.k = {x + a.H * a.dk * size, ld, a.is_f32};
  p.v = {x + 2 * a.H * a.dk * size, ld, a.is_f32};
  p.o = a.o;
  p.ldo = a.H * a.dv;
  p.decay = a.decay;
  p.alpha = 1.0f;
  p.beta = a.scale;
  p.s_in = a.s0;
  p.s_out = a.s_last;
  p.in_d = a.dv;
  p.in_e = 1;
  p.B = static_cast<uint32_t>(a.B);
  p.H = static_cast<uint32_t>(a.H);
  p.T = a.T;
  p.Dk = a.dk;
  p.Dv = a.dv;
  p = with_plan(p, linattn_plan(a.B, a.T, a.H, a.dk, a.dv), joined);
  const auto pass = a.is_f32 ? launch_linattn_f32 : launch_linattn_bf16;
  if (p.joined != nullptr) {
    if (hipError_t e = pass(p, true, stream)) return e;
    if (hipError_t e = join(p, stream)) return e;
  }
  return pass(p, false, stream);
}

size_t linattn_chunk_bytes(int64_t B, int64_t T, int64_t H, int dk, int dv) {
  const LinattnPlan plan = linattn_plan(B, T, H, dk, dv);
  return plan.nseg > 1 ? plan.joined_bytes : 0;
}

size_t linattn_bwd_bytes(int64_t B, int64_t T, int64_t H, int dk, int dv) {
  const size_t a = linattn_plan(B, T, H, dk, dv).joined_bytes, b = linattn_plan(B, T, H, dv, dk).joined_bytes;
  return a > b ? a : b;
}

hipError_t launch_linattn_bwd(const LinattnBwdArgs& a, float* joined, hipStream_t stream) {
  const int64_t size = a.is_f32 ? 4 : 2, ld = a.H * (2 * a.dk + a.dv);
  const char* const x = static_cast<const char*>(a.qkv);
  const LinattnOperand q{x, ld, a.is_f32}, k{x + a.H * a.dk * size, ld, a.is_f32},
      v{x + 2 * a.H * a.dk * size, ld, a.is_f32}, d{a.dout, a.H * a.dv, a.do_is_f32};
  uint16_t* const dq = a.dqkv;
  const bool bf16 = !a.is_f32 && !a.do_is_f32, f32 = a.is_f32 && a.do_is_f32;
  // [0] dq, [1] dk, [2] dv: the last writes ds0, which may be ds_last
  for (int i = 0; i < 3; ++i) {
    LinattnPass p{};
    p.q = i == 0 ? d : i == 1 ? v : k;
    p.k = i == 0 ? v : i == 1 ? d : q;
    p.v = i == 0 ? k : i == 1 ? q : d;
    p.o = dq + (i == 0 ? 0 : i == 1 ? a.H * a.dk : 2 * a.H * a.dk);
    p.ldo = ld;
    p.decay = a.decay;
    p.alpha = i == 0 ? 1.0f : a.scale;
    p.beta = i == 0 ? a.scale : 1.0f;
    p.rev = i != 0;
    p.s_in = i == 0 ? a.s0 : a.ds_last;
    p.join_last = i == 2 && a.ds0 != nullptr;
    p.B = static_cast<uint32_t>(a.B);
    p.H = static_cast<uint32_t>(a.H);
    p.T = a.T;
    p.Dk = i == 2 ? a.dk : a.dv;
    p.Dv = i == 2 ? a.dv : a.dk;
    p.in_d = i == 2 ? a.dv : 1;
    p.in_e = i == 2 ? 1 : a.dv;
    p = with_plan(p, linattn_plan(a.B, a.T, a.H, p.Dk, p.Dv), joined);
    if (p.joined != nullptr) {
      p.s_out = p.join_last ? a.ds0 : nullptr;
      const hipError_t e = bf16  ? launch_linattn_bf16(p, true, stream)
                           : f32 ? launch_linattn_f32(p, true, stream)
                                 : launch_linattn_bwd_any(p, true, stream);
      if (e != hipSuccess) return e;
      if (hipError_t e2 = join(p, stream)) return e2;
      p.s_out = nullptr;
    }
    const hipError_t e = bf16  ? launch_linattn_bwd_bf16(p, stream)
                         : f32 ? launch_linattn_bwd_f32(p, stream)
                               : launch_linattn_bwd_any(p, false, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mmf
