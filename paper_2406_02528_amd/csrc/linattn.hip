// Linear attention over chunks: how the passes are cut into segments, the
// joining of the segments' states, and the passes of both directions.
#include "linattn.h"
#include "mmf_device.h"

#include <initializer_list>

namespace mmf {

hipError_t launch_linattn_f32(const LinattnPass* p, int n, hipStream_t stream);
hipError_t launch_linattn_bf16(const LinattnPass* p, int n, hipStream_t stream);
hipError_t launch_linattn_bwd_f32(const LinattnPass* p, int n, hipStream_t stream);
hipError_t launch_linattn_bwd_any(const LinattnPass* p, int n, hipStream_t stream);
hipError_t launch_linattn_states_f32(const LinattnPass* p, int n, hipStream_t stream);
hipError_t launch_linattn_states_bf16(const LinattnPass* p, int n, hipStream_t stream);
hipError_t launch_linattn_states_any(const LinattnPass* p, int n, hipStream_t stream);

namespace {

// Workgroups that run at once: two on a compute unit, as for most forms of up to 128
// key entries.  (Of more key entries one stands there, and the plan counts too few
// rounds: 1 x 4000, 8 heads of 208 x 144 fp32 takes 120 us in 32 segments, 106 in 16;
// bf16 81, 72.)
constexpr int64_t kSlots = 512;
constexpr int kJoinBlock = 256;

__device__ __forceinline__ double power(double x, int64_t n) {
  double y = 1.0;
  for (; n != 0; n >>= 1) {
    if (n & 1) y *= x;
    x *= x;
  }
  return y;
}

// The states that enter the segments: E_0 is s_in (with its decay to the first
// token where the pass is forward), E_{s+1} = l^tokens E_s + u_s.  E_s takes the
// place of u_s; s_out (nullptr: not wanted; backward alone) is the state behind
// the last token, with its decay.
struct Join {
  float* u;         // [states][n][size]
  const float* s_in;
  float* s_out;
  bool rev;
};
struct Joins {
  Join j[2];
  const float* decay;
  uint32_t states, H, n;
  int64_t size, tokens, T;
};

template <int N>
__global__ __launch_bounds__(kJoinBlock) void linattn_join_kernel(const Joins a) {
  typedef float vec __attribute__((ext_vector_type(N)));
  const Join& j = a.j[blockIdx.y];
  const uint32_t per = static_cast<uint32_t>((a.size / N + kJoinBlock - 1) / kJoinBlock);
  const int64_t bh = blockIdx.x / per;
  const int64_t at = N * (static_cast<int64_t>(blockIdx.x % per) * kJoinBlock + threadIdx.x);
  if (at >= a.size) return;
  const float l = a.decay[bh % a.H];
  const auto load = [](const float* p) { return *reinterpret_cast<const vec*>(p); };
  vec e = 0.0f;
  if (j.s_in != nullptr) {
    e = load(j.s_in + bh * a.size + at);
    if (!j.rev) e *= l;
  }
  float* const u = j.u + bh * a.n * a.size + at;
  // a sum that nothing follows is not there unless s_out is wanted
  const uint32_t have = j.s_out != nullptr ? a.n : a.n - 1;
  const float full = static_cast<float>(power(l, a.tokens));
  constexpr uint32_t kAhead = 32 / N;   // loads in flight
  const float* from = u;
  float* to = u;
  for (uint32_t s = 0; s < a.n; s += kAhead) {
    vec v[kAhead];
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) {
      if (s + i < have) v[i] = load(from);
      from += a.size;
    }
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) {
      if (s + i >= a.n) break;
      *reinterpret_cast<vec*>(to) = e;
      to += a.size;
      if (s + i >= have) continue;
      float w = full;
      if (s + i + 1 == a.n) w = static_cast<float>(power(l, a.T - (s + i) * a.tokens));   // may have fewer tokens
#pragma unroll
      for (int c = 0; c < N; ++c) e[c] = fmaf(w, e[c], v[i][c]);
    }
  }
  if (j.s_out != nullptr) *reinterpret_cast<vec*>(j.s_out + bh * a.size + at) = e;
}

// How both directions are cut.
struct Plan {
  uint32_t nseg;
  int64_t seg_tokens;
};
int waves_of(int Dv) { return Dv <= 64 ? 4 : 8; }
uint32_t tiles_of(int Dv) {
  const int w = 16 * waves_of(Dv);
  return static_cast<uint32_t>((Dv + w - 1) / w);
}
// The backward's passes go in one launch where their kernels are the same: widths
// in the same class, workgroups of the same size.
bool one_launch(int dk, int dv) {
  const auto width = [](int d) { return d <= 64 ? 0 : d <= 128 ? 1 : 2; };
  return width(dk) == width(dv) && waves_of(dk) == waves_of(dv);
}
// launches: their passes, 1 (the forward), 3 or 2 and 1; sums: wanted of a single
// segment too; state_bytes: of all the states that enter one segment.
Plan plan_of(int64_t T, int64_t groups, std::initializer_list<int> launches, bool sums, int64_t state_bytes) {
  constexpr int64_t C = kLinattnChunk;
  const int64_t chunks = (T + C - 1) / C;
  // In tenths of a us: 32 tokens take about 4 where a compute unit has one
  // workgroup, two of them 6; a start 10; with segments, their sums about a third
  // of a pass each, 7 at least, and their states are joined at 4.5 TB/s after 5.
  // (us at the segments taken and at half and twice as many, fp32, heads of 128: forward
  // of 1 x 2048, 16 heads, 16: 56, 76, 61; of 4 x 2048, 8: 128, 138, 152; backward of
  // that, 4: 277, 331, 297; of 1 x 8000, 4 heads, 42: 92, 102, 101; forward of 16384 bf16,
  // 16 heads, 32: 132, 146, 160.  Backward in two launches, 4 x 1857, 12 heads of 96 x
  // 48, 5: 157; 3, as for one: 230.)
  const auto cost = [&](int64_t s) {
    const int64_t per = (chunks + s - 1) / s;
    int64_t work = 0;
    for (const int passes : launches) {
      const int64_t each = (groups * passes * s + kSlots / 2 - 1) / (kSlots / 2);
      work += each / 2 * (60 * per + 100) + each % 2 * (39 * per + 100);
    }
    return s == 1 && !sums ? work : work + (work > 210 ? work / 3 : 70) + state_bytes * s * 2 / 450000 + 50;
  };
  int64_t best = 1;
  for (int64_t s = 2; s <= chunks && groups * (s - 1) < 2 * kSlots; ++s)
    if (cost(s) < cost(best)) best = s;
  const int64_t per = (chunks + best - 1) / best;
  Plan plan;
  plan.nseg = static_cast<uint32_t>((chunks + per - 1) / per);
  plan.seg_tokens = per * C;
  return plan;
}
Plan plan_fwd(int64_t B, int64_t T, int64_t H, int dk, int dv) { return plan_of(T, B * H * tiles_of(dv), {1}, false, 4 * B * H * dk * dv); }
Plan plan_bwd(int64_t B, int64_t T, int64_t H, int dk, int dv, bool sums) {
  const uint32_t a = tiles_of(dv), b = tiles_of(dk);
  const int64_t groups = B * H * (a > b ? a : b), bytes = 8 * B * H * dk * dv;
  return one_launch(dk, dv) ? plan_of(T, groups, {3}, sums, bytes) : plan_of(T, groups, {2, 1}, sums, bytes);
}
size_t sums_bytes(const Plan& plan, int64_t states, int dk, int dv) {
  return sizeof(float) * static_cast<size_t>(states) * plan.nseg * dk * dv;
}

LinattnPass cut(LinattnPass p, const Plan& plan) {
  p.waves = waves_of(p.Dv);
  p.tiles = tiles_of(p.Dv);
  p.nseg = plan.nseg;
  p.seg_tokens = plan.seg_tokens;
  return p;
}
// The same for the sums alone; all: that of the last segment too.
LinattnPass sums_of(LinattnPass p, float* u, bool all) {
  p.segs = all ? p.nseg : p.nseg - 1;
  p.s_out = u;
  return p;
}
// The pass from the joined states u of sums [dk][dv]; `turned`: its state is
// their transpose.
LinattnPass from_joined(LinattnPass p, const float* u, bool turned) {
  const int64_t size = static_cast<int64_t>(p.Dk) * p.Dv;
  p.e_in = u;
  p.e_bh = size * p.nseg;
  p.e_seg = size;
  p.e_d = turned ? 1 : p.Dv;
  p.e_e = turned ? p.Dk : 1;
  p.e_decay = false;
  return p;
}

hipError_t join(const Join* j, int n, const LinattnPass& p, hipStream_t stream) {
  Joins a{};
  for (int i = 0; i < n; ++i) a.j[i] = j[i];
  a.decay = p.decay;
  a.states = p.B * p.H;
  a.H = p.H;
  a.n = p.nseg;
  a.size = static_cast<int64_t>(p.Dk) * p.Dv;
  a.tokens = p.seg_tokens;
  a.T = p.T;
  // Four entries side by side per lane where the lanes are still many (whole calls of
  // bf16, heads of 128, one entry and four: forward of 2^16 entries, 1 x 4096 with 4
  // heads, 32.4 us, 33.7; of 2^18, 16384 with 16 heads, 145.4, 146.0; of 2^19, 2 x 2048,
  // 58.7, 57.8; of 2^20, 4 x 2048, 91.2, 87.3; backward of that 191, 180)
  const bool wide = a.size * a.states * n >= int64_t(1) << 19;
  const int64_t lanes = a.size / (wide ? 4 : 1);
  const dim3 grid(a.states * static_cast<uint32_t>((lanes + kJoinBlock - 1) / kJoinBlock), static_cast<uint32_t>(n));
  if (wide) hipLaunchKernelGGL(linattn_join_kernel<4>, grid, dim3(kJoinBlock), 0, stream, a);
  else hipLaunchKernelGGL(linattn_join_kernel<1>, grid, dim3(kJoinBlock), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t linattn_chunk_bytes(int64_t B, int64_t T, int64_t H, int dk, int dv) {
  const Plan plan = plan_fwd(B, T, H, dk, dv);
  return plan.nseg > 1 ? sums_bytes(plan, B * H, dk, dv) : 0;
}

hipError_t launch_linattn_chunk(const LinattnArgs& a, float* scratch, hipStream_t stream) {
  const Plan plan = plan_fwd(a.B, a.T, a.H, a.dk, a.dv);
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
  p.B = static_cast<uint32_t>(a.B);
  p.H = static_cast<uint32_t>(a.H);
  p.T = a.T;
  p.Dk = a.dk;
  p.Dv = a.dv;
  p = cut(p, plan);
  if (plan.nseg == 1) {
    p.e_in = a.s0;
    p.e_bh = static_cast<int64_t>(a.dk) * a.dv;
    p.e_d = a.dv;
    p.e_e = 1;
    p.e_decay = true;
    p.s_out = a.s_last;
    return (a.is_f32 ? launch_linattn_f32 : launch_linattn_bf16)(&p, 1, stream);
  }
  const LinattnPass u = sums_of(p, scratch, false);
  if (hipError_t e = (a.is_f32 ? launch_linattn_states_f32 : launch_linattn_states_bf16)(&u, 1, stream)) return e;
  const Join j{scratch, a.s0, nullptr, false};
  if (hipError_t e = join(&j, 1, p, stream)) return e;
  p = from_joined(p, scratch, false);
  p.s_out = a.s_last;
  return (a.is_f32 ? launch_linattn_f32 : launch_linattn_bf16)(&p, 1, stream);
}

size_t linattn_bwd_bytes(int64_t B, int64_t T, int64_t H, int dk, int dv) {
  const size_t a = sums_bytes(plan_bwd(B, T, H, dk, dv, false), B * H, dk, dv);
  const size_t b = sums_bytes(plan_bwd(B, T, H, dk, dv, true), B * H, dk, dv);
  return 2 * (a > b ? a : b);
}

hipError_t launch_linattn_bwd(const LinattnBwdArgs& a, float* scratch, hipStream_t stream) {
  const bool bf16 = !a.is_f32 && !a.do_is_f32, f32 = a.is_f32 && a.do_is_f32;
  // Of one segment and one type dv's state behind its last token is ds0, which
  // comes from the sums else (64 x 64 tokens, 8 heads of 64, bf16: 22 us, by the
  // sums 35; fp32 37, 52; 7 x 600, 12 heads of 128, 66, 95; fp32 105, 133).
  const bool alike = bf16 || f32;
  const Plan plan = plan_bwd(a.B, a.T, a.H, a.dk, a.dv, a.ds0 != nullptr && !alike);
  const int64_t size = a.is_f32 ? 4 : 2, ld = a.H * (2 * a.dk + a.dv);
  const char* const x = static_cast<const char*>(a.qkv);
  const LinattnOperand q{x, ld, a.is_f32}, k{x + a.H * a.dk * size, ld, a.is_f32},
      v{x + 2 * a.H * a.dk * size, ld, a.is_f32}, d{a.dout, a.H * a.dv, a.do_is_f32};
  LinattnPass base{};
  base.decay = a.decay;
  base.B = static_cast<uint32_t>(a.B);
  base.H = static_cast<uint32_t>(a.H);
  base.T = a.T;
  base.ldo = ld;
  // dq, dk, dv; [3], [4]: the sums of S and of its gradient
  LinattnPass p[5];
  for (int i = 0; i < 5; ++i) {
    p[i] = base;
    const bool turned = i < 2;
    p[i].q = i == 0 ? d : i == 1 ? v : k;
    p[i].k = i == 0 ? v : i == 1 ? d : i == 3 ? k : q;
    p[i].v = i == 0 || i == 2 ? (i == 0 ? k : d) : i == 1 ? q : i == 3 ? v : d;
    p[i].o = a.dqkv + (i == 1 ? a.H * a.dk : i == 2 ? 2 * a.H * a.dk : 0);
    const bool s = i == 0 || i == 3;
    p[i].rev = !s;
    p[i].alpha = s ? 1.0f : a.scale;
    p[i].beta = s ? a.scale : 1.0f;
    p[i].Dk = turned ? a.dv : a.dk;
    p[i].Dv = turned ? a.dk : a.dv;
    p[i] = cut(p[i], plan);
    p[i].e_in = s ? a.s0 : a.ds_last;
    p[i].e_bh = static_cast<int64_t>(a.dk) * a.dv;
    p[i].e_d = turned ? 1 : a.dv;
    p[i].e_e = turned ? a.dv : 1;
    p[i].e_decay = s;
  }
  float* const us = scratch;
  float* const ug = scratch + sums_bytes(plan, a.B * a.H, a.dk, a.dv) / sizeof(float);
  const bool some = plan.nseg > 1;
  const bool by_dv = alike && !some && a.ds0 != nullptr;
  if (by_dv) p[2].s_out = a.ds0;
  if (some || (a.ds0 != nullptr && !by_dv)) {
    LinattnPass u[2];
    Join j[2];
    int n = 0;
    if (some) {
      u[n] = sums_of(p[3], us, false);
      j[n++] = {us, a.s0, nullptr, false};
    }
    u[n] = sums_of(p[4], ug, a.ds0 != nullptr);
    j[n++] = {ug, a.ds_last, a.ds0, true};
    const auto states = bf16 ? launch_linattn_states_bf16 : f32 ? launch_linattn_states_f32 : launch_linattn_states_any;
    if (hipError_t e = states(u, n, stream)) return e;
    if (hipError_t e = join(j, n, p[4], stream)) return e;
    if (some) p[0] = from_joined(p[0], us, true);
    // from here on ds_last may be overwritten by ds0
    p[1] = from_joined(p[1], ug, true);
    p[2] = from_joined(p[2], ug, false);
  }
  const auto passes = [&](const LinattnPass* first, int n) {
    return (bf16 ? launch_linattn_bf16 : f32 ? launch_linattn_bwd_f32 : launch_linattn_bwd_any)(first, n, stream);
  };
  // dv by itself where it writes over what dk reads
  if (one_launch(a.dk, a.dv) && !(by_dv && a.ds0 == a.ds_last)) return passes(p, 3);
  if (hipError_t e = passes(p, 2)) return e;
  return passes(p + 2, 1);
}

}  // namespace mmf
