// The MLGRU recurrence in training form, forward and backward, from the
// pre-activations z [B*T][3d] of the three gates (zf | zc | zg):
//   f = lb + (1 - lb) sigmoid(zf),  c = zc sigmoid(zc),  g = zg
//   h_t = f_t h_{t-1} + (1 - f_t) c_t,   o'_t = g_t sigmoid(h_t)
// Backward, with do = the gradient of o' and dh_last that of the last state:
//   dh_t = do_t g_t s(h_t) (1 - s(h_t)) + f_{t+1} dh_{t+1}
//   dzf = dh (h_{t-1} - c) (1 - lb) s(zf) (1 - s(zf))
//   dzc = dh (1 - f) s(zc) (1 + zc (1 - s(zc))),   dzg = do s(h)
//   dh0 = f_1 dh_1,   dlb = sum over tokens of dh (h_{t-1} - c) (1 - s(zf))
//
// Both recurrences are linear, so a run of tokens maps the value that enters
// it to a x + b.  A workgroup holds a chunk of kWaves x kTok tokens of 128
// channels in registers: each wave scans its kTok tokens (two channels per
// lane), the waves' maps are joined through LDS, and the chunks of a sequence
// through a carry pass.  The states entering the chunks are kept for the
// backward.  The backward's map needs no second sweep: with P_t the product
// of the forget gates from the chunk's start to t, the gradient that leaves
// at the chunk's start is P_end G + sum_t P_t e_t (G the gradient entering at
// its end, e_t the tokens' own), summed in the forward direction together
// with h.
#include "mmf_device.h"
#include "mmf_launch.h"
#include "row_vec.h"

namespace mmf {
namespace {

constexpr int kWaves = 8, kTok = 8;
constexpr int kChunk = kWaves * kTok;  // tokens per workgroup
constexpr int kCh = 2 * kWave;         // channels per workgroup
constexpr int kThreads = kWaves * kWave;

struct V2 {
  float x, y;
};
__device__ __forceinline__ V2 ld2(const float* p) {
  const float2 v = *reinterpret_cast<const float2*>(p);
  return {v.x, v.y};
}
__device__ __forceinline__ void st2(float* p, V2 v) { *reinterpret_cast<float2*>(p) = make_float2(v.x, v.y); }

// y = a x + b, and first p, then q.
struct Map {
  float a, b;
};
__device__ __forceinline__ Map then(Map p, Map q) { return {q.a * p.a, q.a * p.b + q.b}; }

__device__ __forceinline__ float forget(float zf, float lb) { return (1.0f - lb) * sigmoid_hw(zf) + lb; }
__device__ __forceinline__ float silu(float z) { return z * sigmoid_hw(z); }

// Where a workgroup and a lane stand.
struct Place {
  int64_t b, k, t0;    // sequence, chunk, first token of the wave (in its sequence)
  int64_t c;           // first of the lane's two channels
  bool col;            // inside d
  int wave, lane;
};
__device__ __forceinline__ Place place(int64_t d, int64_t nchunk) {
  Place p;
  p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  p.lane = threadIdx.x & 63;
  const int64_t ncg = (d + kCh - 1) / kCh;
  const int64_t bk = blockIdx.x / ncg;
  p.b = bk / nchunk;
  p.k = bk % nchunk;
  p.t0 = p.k * kChunk + p.wave * kTok;
  const int64_t c = (blockIdx.x % ncg) * kCh + 2 * p.lane;
  p.col = c < d;
  p.c = p.col ? c : d - 2;
  return p;
}
// Token t0 + u of the wave, or the sequence's last one past its end.
__device__ __forceinline__ int64_t token(const Place& p, int u, int64_t T) { return p.t0 + u < T ? p.t0 + u : T - 1; }

// The wave's map of the forward recurrence over its tokens, per channel.
__device__ __forceinline__ void chunk_map(const V2* f, const V2* c, Map& mx, Map& my) {
  mx = my = {1.0f, 0.0f};
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    mx = {mx.a * f[u].x, mlgru_step(mx.b, f[u].x, c[u].x)};
    my = {my.a * f[u].y, mlgru_step(my.b, f[u].y, c[u].y)};
  }
}

struct FwdArgs {
  const float* z;
  const float* lb;
  const float* h0;
  float *A, *Bs;       // chunk maps [B][nchunk][d]
  float* states;       // [B][nchunk][d]
  float* o;
  float* h_last;
  int64_t T, d, nchunk;
};

// APPLY false: the chunk's map into A, Bs.  APPLY true: o' from the chunk's
// entering state (one chunk: h0, stored in states here).
template <bool APPLY>
__global__ __launch_bounds__(kThreads) void mlgru_train_fwd_kernel(const FwdArgs a) {
  __shared__ Map maps[2][kWaves][kWave];
  const Place p = place(a.d, a.nchunk);
  const int64_t T = a.T, d = a.d;
  const float* z = a.z + p.b * T * 3 * d + p.c;
  V2 f[kTok], c[kTok], g[kTok];
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    const int64_t t = token(p, u, T);
    f[u] = ld2(z + t * 3 * d);
    c[u] = ld2(z + t * 3 * d + d);
    if constexpr (APPLY) g[u] = ld2(z + t * 3 * d + 2 * d);
  }
  const V2 lb = a.lb != nullptr ? ld2(a.lb + p.c) : V2{0.0f, 0.0f};
  const int64_t at = (p.b * a.nchunk + p.k) * d + p.c;
  V2 h = {0.0f, 0.0f};
  if constexpr (APPLY) {
    if (a.nchunk > 1) h = ld2(a.states + at);
    else if (a.h0 != nullptr) h = ld2(a.h0 + p.b * d + p.c);
  }
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    const bool in = p.t0 + u < T;  // past the end: f = 1 keeps the state
    f[u] = {in ? forget(f[u].x, lb.x) : 1.0f, in ? forget(f[u].y, lb.y) : 1.0f};
    c[u] = {silu(c[u].x), silu(c[u].y)};
  }
  Map mx, my;
  chunk_map(f, c, mx, my);
  maps[0][p.wave][p.lane] = mx;
  maps[1][p.wave][p.lane] = my;
  __syncthreads();
  if constexpr (!APPLY) {
    if (p.wave == 0 && p.col) {
#pragma unroll
      for (int w = 1; w < kWaves; ++w) {
        mx = then(mx, maps[0][w][p.lane]);
        my = then(my, maps[1][w][p.lane]);
      }
      st2(a.A + at, {mx.a, my.a});
      st2(a.Bs + at, {mx.b, my.b});
    }
  } else {
    if (a.nchunk == 1 && p.wave == 0 && p.col) st2(a.states + at, h);
    for (int w = 0; w < p.wave; ++w) {
      const Map u = maps[0][w][p.lane], v = maps[1][w][p.lane];
      h = {u.a * h.x + u.b, v.a * h.y + v.b};
    }
    float* o = a.o + p.b * T * d + p.c;
#pragma unroll
    for (int u = 0; u < kTok; ++u) {
      h = {mlgru_step(h.x, f[u].x, c[u].x), mlgru_step(h.y, f[u].y, c[u].y)};
      if (p.t0 + u < T && p.col)
        st2(o + (p.t0 + u) * d, {mlgru_out_gate(g[u].x, h.x), mlgru_out_gate(g[u].y, h.y)});
    }
    if (a.h_last != nullptr && p.col && p.t0 < T && p.t0 + kTok >= T) st2(a.h_last + p.b * d + p.c, h);
  }
}

// The value entering each chunk, composed over the chunks in order (REV:
// from the last): a workgroup owns kCarryCh channels of a sequence; each of
// its kSegs groups composes a run of chunks, one group joins the runs, and
// each walks its run again.  first: the value entering the first one (nullptr:
// 0), last: where the value that leaves the last one goes (nullptr: nowhere).
constexpr int kCarryCh = 32, kSegs = 32;
template <bool REV>
__global__ __launch_bounds__(kCarryCh* kSegs) void mlgru_train_carry_kernel(const float* __restrict__ A,
                                                                           const float* __restrict__ Bs,
                                                                           const float* first, int64_t nchunk,
                                                                           int64_t d, float* __restrict__ carry, float* last) {
  __shared__ Map seg[kSegs][kCarryCh];
  __shared__ float in[kSegs][kCarryCh];
  const int64_t nblk = (d + kCarryCh - 1) / kCarryCh;
  const int64_t b = blockIdx.x / nblk;
  const int c = threadIdx.x % kCarryCh, s = threadIdx.x / kCarryCh;
  const int64_t ch = (blockIdx.x % nblk) * kCarryCh + c;
  const bool col = ch < d;
  const int64_t per = (nchunk + kSegs - 1) / kSegs;
  const int64_t k0 = s * per < nchunk ? s * per : nchunk;
  const int64_t k1 = k0 + per < nchunk ? k0 + per : nchunk;
  auto at = [&](int64_t k) { return (b * nchunk + (REV ? nchunk - 1 - k : k)) * d + ch; };
  Map m = {1.0f, 0.0f};
  if (col) {
#pragma unroll 8
    for (int64_t k = k0; k < k1; ++k) m = then(m, {A[at(k)], Bs[at(k)]});
  }
  seg[s][c] = m;
  const float x0 = col && first != nullptr ? first[b * d + ch] : 0.0f;
  __syncthreads();
  if (s == 0) {
    float x = x0;
#pragma unroll 8
    for (int i = 0; i < kSegs; ++i) {
      in[i][c] = x;
      x = seg[i][c].a * x + seg[i][c].b;
    }
    if (col && last != nullptr) last[b * d + ch] = x;
  }
  __syncthreads();
  if (!col) return;
  float x = in[s][c];
#pragma unroll 8
  for (int64_t k = k0; k < k1; ++k) {
    const int64_t i = at(k);
    const float av = A[i], bv = Bs[i];
    carry[i] = x;
    x = av * x + bv;
  }
}

struct BwdArgs {
  const float* z;
  const float* lb;
  const float* states;
  const void* dout;     // [B*T][d] bf16 or fp32
  const float* dh_last; // nullptr: zero
  float *A, *Bs;        // maps of the gradient through each chunk
  const float* G;       // gradients entering the chunks at their ends
  uint16_t* dz;
  float* dh0;           // one chunk: stored here (nullptr: not stored)
  double* dlb_part;     // [B * nchunk][d], nullptr: not computed
  int64_t T, d, nchunk;
};

// APPLY false: the map of the gradient through the chunk (its product of
// forget gates, and sum_t P_t e_t).  APPLY true: dz from the gradient that
// enters at the chunk's end.
template <typename DT, bool APPLY>
__global__ __launch_bounds__(kThreads) void mlgru_train_bwd_kernel(const BwdArgs a) {
  __shared__ Map maps[2][kWaves][kWave];
  __shared__ Map back[2][kWaves][kWave];
  __shared__ double s_dlb[APPLY ? kWaves : 1][kCh];
  const Place p = place(a.d, a.nchunk);
  const int64_t T = a.T, d = a.d;
  const float* z = a.z + p.b * T * 3 * d + p.c;
  const DT* dout = static_cast<const DT*>(a.dout) + p.b * T * d + p.c;
  V2 zf[kTok], zc[kTok], zg[kTok], go[kTok];
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    const int64_t t = token(p, u, T);
    zf[u] = ld2(z + t * 3 * d);
    zc[u] = ld2(z + t * 3 * d + d);
    zg[u] = ld2(z + t * 3 * d + 2 * d);
    if constexpr (sizeof(DT) == 4) {
      go[u] = ld2(reinterpret_cast<const float*>(dout) + t * d);
    } else {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(dout + t * d);
      go[u] = {bf16_lo(w), bf16_hi(w)};
    }
  }
  const V2 lb = a.lb != nullptr ? ld2(a.lb + p.c) : V2{0.0f, 0.0f};
  const int64_t at = (p.b * a.nchunk + p.k) * d + p.c;
  V2 h = ld2(a.states + at);
  V2 G = {0.0f, 0.0f};
  if constexpr (APPLY) {
    if (a.nchunk > 1) G = ld2(a.G + at);
    else if (a.dh_last != nullptr) G = ld2(a.dh_last + p.b * d + p.c);
  }
  V2 f[kTok], c[kTok];
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    const bool in = p.t0 + u < T;  // past the end: f = 1 and no gradient of its own
    f[u] = {in ? forget(zf[u].x, lb.x) : 1.0f, in ? forget(zf[u].y, lb.y) : 1.0f};
    c[u] = {silu(zc[u].x), silu(zc[u].y)};
    if (!in) go[u] = {0.0f, 0.0f};
  }
  Map mx, my;
  chunk_map(f, c, mx, my);
  maps[0][p.wave][p.lane] = mx;
  maps[1][p.wave][p.lane] = my;
  __syncthreads();
  for (int w = 0; w < p.wave; ++w) {
    const Map u = maps[0][w][p.lane], v = maps[1][w][p.lane];
    h = {u.a * h.x + u.b, v.a * h.y + v.b};
  }
  // h before each token, and the gradient's map through the wave's tokens
  V2 hp[kTok], sh[kTok];
  Map gx = {1.0f, 0.0f}, gy = {1.0f, 0.0f};
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    hp[u] = h;
    h = {mlgru_step(h.x, f[u].x, c[u].x), mlgru_step(h.y, f[u].y, c[u].y)};
    sh[u] = {sigmoid_hw(h.x), sigmoid_hw(h.y)};
    gx.a *= f[u].x;
    gy.a *= f[u].y;
    gx.b += gx.a * (go[u].x * zg[u].x * (sh[u].x * (1.0f - sh[u].x)));
    gy.b += gy.a * (go[u].y * zg[u].y * (sh[u].y * (1.0f - sh[u].y)));
  }
  back[0][p.wave][p.lane] = gx;
  back[1][p.wave][p.lane] = gy;
  __syncthreads();
  if constexpr (!APPLY) {
    if (p.wave == kWaves - 1 && p.col) {
#pragma unroll
      for (int w = kWaves - 2; w >= 0; --w) {
        gx = then(gx, back[0][w][p.lane]);
        gy = then(gy, back[1][w][p.lane]);
      }
      st2(a.A + at, {gx.a, gy.a});
      st2(a.Bs + at, {gx.b, gy.b});
    }
  } else {
    for (int w = kWaves - 1; w > p.wave; --w) {
      const Map u = back[0][w][p.lane], v = back[1][w][p.lane];
      G = {u.a * G.x + u.b, v.a * G.y + v.b};
    }
    uint16_t* dz = a.dz + p.b * T * 3 * d + p.c;
    double dlx = 0.0, dly = 0.0;
#pragma unroll
    for (int u = kTok - 1; u >= 0; --u) {
      // one channel: its gradients, and G carried to the token before
      auto one = [](float zf, float zc, float zg, float go, float hp, float sh, float f, float c, float lb, float& G,
                    float& df, float& dc, float& dg, double& dl) {
        const float dh = G + go * zg * (sh * (1.0f - sh));
        const float sf = sigmoid_hw(zf), sc = sigmoid_hw(zc);
        const float w = dh * (hp - c);
        df = w * ((1.0f - lb) * sf * (1.0f - sf));
        dc = dh * (1.0f - f) * (sc * (1.0f + zc * (1.0f - sc)));
        dg = go * sh;
        dl += static_cast<double>(w * (1.0f - sf));
        G = f * dh;
      };
      if (p.t0 + u < T) {  // uniform per wave
        V2 df, dc, dg;
        one(zf[u].x, zc[u].x, zg[u].x, go[u].x, hp[u].x, sh[u].x, f[u].x, c[u].x, lb.x, G.x, df.x, dc.x, dg.x, dlx);
        one(zf[u].y, zc[u].y, zg[u].y, go[u].y, hp[u].y, sh[u].y, f[u].y, c[u].y, lb.y, G.y, df.y, dc.y, dg.y, dly);
        if (p.col) {
          uint32_t* row = reinterpret_cast<uint32_t*>(dz + (p.t0 + u) * 3 * d);
          row[0] = pack_bf16(df.x, df.y);
          *reinterpret_cast<uint32_t*>(dz + (p.t0 + u) * 3 * d + d) = pack_bf16(dc.x, dc.y);
          *reinterpret_cast<uint32_t*>(dz + (p.t0 + u) * 3 * d + 2 * d) = pack_bf16(dg.x, dg.y);
        }
      }
    }
    if (a.nchunk == 1 && p.wave == 0 && p.col && a.dh0 != nullptr) st2(a.dh0 + p.b * d + p.c, G);
    if (a.dlb_part != nullptr) {
      s_dlb[p.wave][2 * p.lane] = dlx;
      s_dlb[p.wave][2 * p.lane + 1] = dly;
      __syncthreads();
      if (p.wave == 0 && p.col) {
        double x = 0.0, y = 0.0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          x += s_dlb[w][2 * p.lane];
          y += s_dlb[w][2 * p.lane + 1];
        }
        *reinterpret_cast<double2*>(a.dlb_part + at) = make_double2(x, y);
      }
    }
  }
}

}  // namespace

int64_t mlgru_train_chunks(int64_t T) { return (T + kChunk - 1) / kChunk; }

int64_t mlgru_train_blocks(int64_t B, int64_t T, int64_t d) {
  return B * mlgru_train_chunks(T) * ((d + kCh - 1) / kCh);
}

hipError_t launch_mlgru_train_scan(const MlgruTrainArgs& p, float* o, float* h_last, float* states, float* ws,
                                   hipStream_t stream) {
  const int64_t nchunk = mlgru_train_chunks(p.T), n = p.B * nchunk * p.d;
  const FwdArgs a{p.z, p.lb, p.h0, ws, ws + n, states, o, h_last, p.T, p.d, nchunk};
  const dim3 grid(static_cast<unsigned>(mlgru_train_blocks(p.B, p.T, p.d)));
  if (nchunk > 1) {
    hipLaunchKernelGGL(mlgru_train_fwd_kernel<false>, grid, dim3(kThreads), 0, stream, a);
    hipLaunchKernelGGL(mlgru_train_carry_kernel<false>, dim3(static_cast<unsigned>(p.B * ((p.d + kCarryCh - 1) / kCarryCh))),
                       dim3(kCarryCh * kSegs), 0, stream, a.A, a.Bs, p.h0, nchunk, p.d, states,
                       static_cast<float*>(nullptr));
  }
  hipLaunchKernelGGL(mlgru_train_fwd_kernel<true>, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_mlgru_scan_bwd(const MlgruTrainArgs& p, const float* states, const void* dout, bool dout_is_f32,
                                 const float* dh_last, uint16_t* dz, float* dh0, float* ws, double* dlb_part,
                                 hipStream_t stream) {
  const int64_t nchunk = mlgru_train_chunks(p.T), n = p.B * nchunk * p.d;
  const BwdArgs a{p.z, p.lb, states, dout, dh_last, ws, ws + n, ws + 2 * n, dz, dh0, dlb_part, p.T, p.d, nchunk};
  const dim3 grid(static_cast<unsigned>(mlgru_train_blocks(p.B, p.T, p.d))), block(kThreads);
  if (nchunk > 1) {
    if (dout_is_f32)
      hipLaunchKernelGGL((mlgru_train_bwd_kernel<float, false>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((mlgru_train_bwd_kernel<uint16_t, false>), grid, block, 0, stream, a);
    hipLaunchKernelGGL(mlgru_train_carry_kernel<true>, dim3(static_cast<unsigned>(p.B * ((p.d + kCarryCh - 1) / kCarryCh))),
                       dim3(kCarryCh * kSegs), 0, stream, a.A, a.Bs, dh_last, nchunk, p.d, ws + 2 * n, dh0);
  }
  if (dout_is_f32)
    hipLaunchKernelGGL((mlgru_train_bwd_kernel<float, true>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((mlgru_train_bwd_kernel<uint16_t, true>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace mmf
