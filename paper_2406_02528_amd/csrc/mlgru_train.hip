// The MLGRU recurrence in training form, forward and backward, from the
// pre-activations z [B*T][3d] of the three gates (zf | zc | zg):
//   f = lb + (1 - lb) sigmoid(zf),  c = zc sigmoid(zc),  g = zg
//   h_t = f_t h_{t-1} + (1 - f_t) c_t,   o'_t = g_t sigmoid(h_t)
// Backward, with do = the gradient of o' and dh_last that of the last state:
//   dh_t = e_t + f_{t+1} dh_{t+1},  e_t = do_t g_t s(h_t) (1 - s(h_t))
//   dzf = dh (h_{t-1} - c) (1 - lb) s(zf) (1 - s(zf))
//   dzc = dh (1 - f) s(zc) (1 + zc (1 - s(zc))),   dzg = do s(h)
//   dh0 = f_1 dh_1,   dlb = sum over tokens of dh (h_{t-1} - c) (1 - s(zf)) (fp64)
//
// Both recurrences are linear, so a run of tokens maps the value that enters
// it to a x + b.  A workgroup holds a chunk of 128 tokens x 64 channels in
// registers: 16 half waves with 8 tokens each, two channels per lane; their
// maps are joined through LDS.  The chunks of a sequence are joined while
// they are held, so that z is read once each way (a chained scan with
// look-back, here over fixed runs): 16 chunks make a run; the last chunk of a
// run publishes the value after it, every other its map, and a chunk starts
// from the value before its run and the maps of the chunks before it in the
// run.  A value thus takes the same roundings whatever the order in which
// chunks are done.
//
// The words that chunks exchange: one of 64 bits per chunk and channel,
// written and read as relaxed device-scope atomics (which pass the XCDs' own
// L2s), each complete in itself, so no order between them matters: kEmpty
// before anything is published, then {a, b}, or {0, x} for a value.  a never
// has the bits of kEmpty's (a NaN is made the ordinary one).  Workgroups take
// their chunks by ticket, the chunks of a sequence in order: a workgroup waits
// only for lower tickets, whose owners run already, and the lowest unfinished
// one waits for none, so every wait ends; the counts of polls are bounded all
// the same, and a wait that ran out gives NaN.
//
// The backward's map needs no sweep of its own: with P_t the product of the
// forget gates from the chunk's start to t, the gradient that leaves at the
// chunk's start is P_end G + sum_t P_t e_t (G the gradient entering at its
// end), summed in the forward direction together with h.
//
// Bound by HBM: 16 bytes per token and channel forward, 22 backward (fp32 do).
// One sequence of 16384 tokens x 2048: forward 102 us (5.2 TB/s), backward 142
// us (5.2 TB/s; medians of 61 calls); as two sweeps (the chunks' maps first, z
// read again for the values) 155 and 300 us.  Waiting for other chunks is 5
// and 10 % of that.  The backward takes the 128 registers of four waves per
// SIMD and spills up to two; three waves with 164 measured 9 % slower for
// both directions together, as did 4 tokens per half wave with five (11 %).
#include "mmf_device.h"
#include "mmf_launch.h"
#include "row_vec.h"

namespace mmf {
namespace {

constexpr int kTok = 8, kSubs = 16, kLanes = 32;
constexpr int kChunk = kSubs * kTok;   // tokens per workgroup
constexpr int kCh = 2 * kLanes;        // channels per workgroup
constexpr int kThreads = kSubs * kLanes;

constexpr uint64_t kEmpty = ~uint64_t(0);
constexpr int kMaxPolls = 1 << 22;     // seconds
constexpr int kRun = kSubs;            // chunks of a run: each half wave reads at most one word

struct V2 {
  float x, y;
};
__device__ __forceinline__ V2 ld2(const float* p) {
  const float2 v = *reinterpret_cast<const float2*>(p);
  return {v.x, v.y};
}
__device__ __forceinline__ void st2(float* p, V2 v) { *reinterpret_cast<float2*>(p) = make_float2(v.x, v.y); }

// y = a x + b for each of a lane's two channels (one 16-byte LDS word).
struct __attribute__((aligned(16))) Map2 {
  float ax, bx, ay, by;
  __device__ __forceinline__ V2 operator()(V2 v) const { return {fmaf(ax, v.x, bx), fmaf(ay, v.y, by)}; }
};
constexpr Map2 kSame = {1.0f, 0.0f, 1.0f, 0.0f};
// first p, then q
__device__ __forceinline__ Map2 then(Map2 p, Map2 q) {
  return {q.ax * p.ax, fmaf(q.ax, p.bx, q.bx), q.ay * p.ay, fmaf(q.ay, p.by, q.by)};
}

// Where a workgroup and a lane stand.
struct Place {
  int64_t b, k;     // sequence and chunk
  int64_t row0;     // first row of the chunk in the [B*T] arrays
  int rows;         // of its tokens inside the sequence
  int64_t c0, c;    // first channel of the workgroup and of the lane's two
  bool col;         // inside d
  int sub, lane;    // half wave, lane in it
  int u0;           // its first token in the chunk
};

// A chunk's rows of `width` elements of `size` bytes: loads past the
// sequence's end or (off) past d read as zero and stores there go nowhere.
// Offsets stay below 2^31 (d <= 2^20: 128 rows of 3 d floats).  NT: as streams.
template <bool NT>
struct Rows {
  static constexpr int kPolicy = NT ? kNontemporal : 0;
  __amdgpu_buffer_rsrc_t r;
  uint32_t row_bytes, at;   // of a row; the lane's channel in its first token
  template <typename T>
  __device__ __forceinline__ Rows(T* base, const Place& p, int64_t width, uint32_t size) {
    row_bytes = static_cast<uint32_t>(width) * size;
    r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(reinterpret_cast<const char*>(base)) + p.row0 * row_bytes, 0,
                                          static_cast<int>(p.rows * row_bytes), kBufferWord3);
    at = p.col ? static_cast<uint32_t>(p.u0) * row_bytes + static_cast<uint32_t>(p.c) * size : 0x80000000u;
  }
  __device__ __forceinline__ V2 f32(int u, uint32_t off) const {
    const float2 v = __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(r, at + u * row_bytes + off, 0, kPolicy));
    return {v.x, v.y};
  }
  __device__ __forceinline__ V2 bf16(int u) const {
    const uint32_t w = __builtin_amdgcn_raw_buffer_load_b32(r, at + u * row_bytes, 0, kPolicy);
    return {bf16_lo(w), bf16_hi(w)};
  }
  __device__ __forceinline__ void store(int u, V2 v) const {
    typedef unsigned int v2u __attribute__((ext_vector_type(2)));
    __builtin_amdgcn_raw_buffer_store_b64(v2u{__float_as_uint(v.x), __float_as_uint(v.y)}, r, at + u * row_bytes, 0,
                                          kPolicy);
  }
  __device__ __forceinline__ void store_bf16(int u, uint32_t off, float x, float y) const {
    __builtin_amdgcn_raw_buffer_store_b32(pack_bf16(x, y), r, at + u * row_bytes + off, 0, kPolicy);
  }
};

template <bool MANY>
__device__ __forceinline__ Place place(int64_t T, int64_t d, int64_t B, int64_t nchunk, bool rev, uint32_t* tickets) {
  const uint32_t ncg = static_cast<uint32_t>((d + kCh - 1) / kCh);
  uint32_t n = blockIdx.x;
  if constexpr (MANY) {
    __shared__ uint32_t s_n;
    if (threadIdx.x == 0) s_n = __hip_atomic_fetch_add(tickets, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    n = __builtin_amdgcn_readfirstlane(s_n);
  }
  Place p;
  const uint32_t groups = static_cast<uint32_t>(B) * ncg;
  const uint32_t pos = n / groups, grp = n % groups;
  p.k = rev ? nchunk - 1 - pos : pos;
  p.b = grp / ncg;
  p.sub = threadIdx.x / kLanes;
  p.lane = threadIdx.x % kLanes;
  p.u0 = p.sub * kTok;
  p.row0 = p.b * T + p.k * kChunk;
  const int64_t left = T - p.k * kChunk;
  p.rows = left < kChunk ? static_cast<int>(left) : kChunk;
  p.c0 = static_cast<int64_t>(grp % ncg) * kCh;
  const int64_t c = p.c0 + 2 * p.lane;
  p.col = c < d;
  p.c = p.col ? c : d - 2;
  return p;
}

__device__ __forceinline__ uint64_t word(float a, float b) {
  const uint32_t lo = __float_as_uint(a != a ? __builtin_nanf("") : a);
  return (static_cast<uint64_t>(__float_as_uint(b)) << 32) | lo;
}
__device__ __forceinline__ void publish(uint64_t* w, Map2 m) {
  __hip_atomic_store(w, word(m.ax, m.bx), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(w + 1, word(m.ay, m.by), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The value that enters the chunk at position `pos` of its sequence, for the
// lane's channels; `words`: those of position 0, `first`: the value that
// enters the sequence.  Half wave i waits for the map of chunk i of the run,
// if that lies before this one; the last half wave (there is no chunk after
// its own) for the value before the run.
__device__ __forceinline__ V2 carry_in(const uint64_t* words, int64_t d, int64_t pos, V2 first, int sub, int lane,
                                       Map2 (*lds)[kLanes]) {
  const int i = static_cast<int>(pos % kRun);
  const int64_t run = pos - i;
  const bool value = sub == kRun - 1;
  if (sub < i || value) {
    Map2 m = {0.0f, first.x, 0.0f, first.y};
    if (!value || run > 0) {
      const uint64_t* w = words + (value ? run - 1 : run + sub) * d;
      uint64_t x, y;
      int polls = 0;
      do {
        x = __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        y = __hip_atomic_load(w + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (x != kEmpty && y != kEmpty) break;
        __builtin_amdgcn_s_sleep(1);
      } while (++polls < kMaxPolls);
      m = {__uint_as_float(static_cast<uint32_t>(x)), __uint_as_float(static_cast<uint32_t>(x >> 32)),
           __uint_as_float(static_cast<uint32_t>(y)), __uint_as_float(static_cast<uint32_t>(y >> 32))};
    }
    lds[sub][lane] = m;
  }
  __syncthreads();
  V2 h = {lds[kRun - 1][lane].bx, lds[kRun - 1][lane].by};
#pragma unroll 2
  for (int j = 0; j < i; ++j) h = lds[j][lane](h);
  return h;
}

// What a chunk publishes: its map as soon as it has it, or at a run's end the
// value after it; nothing where no chunk would read it.
__device__ __forceinline__ void publish_map(uint64_t* words, int64_t d, int64_t pos, int64_t nchunk, Map2 m) {
  if (pos % kRun != kRun - 1 && pos < nchunk - 1) publish(words + pos * d, m);
}
__device__ __forceinline__ void publish_end(uint64_t* words, int64_t d, int64_t pos, V2 end) {
  if (pos % kRun == kRun - 1) publish(words + pos * d, {0.0f, end.x, 0.0f, end.y});
}

struct FwdArgs {
  const float* z;
  const float* lb;
  const float* h0;
  uint64_t* words;     // [B][nchunk][d]
  uint32_t* tickets;
  float* states;       // [B][nchunk][d]
  float* o;
  float* h_last;
  int64_t B, T, d, nchunk;
};

template <bool MANY, bool NT>
__global__ __launch_bounds__(kThreads) void mlgru_train_fwd_kernel(const FwdArgs a) {
  __shared__ Map2 maps[kSubs][kLanes], look[MANY ? kSubs : 1][kLanes];
  const int64_t d = a.d;
  const Place p = place<MANY>(a.T, d, a.B, a.nchunk, false, a.tickets);
  const Rows<NT> z(a.z, p, 3 * d, 4), o(a.o, p, d, 4);
  const uint32_t gate = static_cast<uint32_t>(d) * 4u;
  V2 f[kTok], c[kTok], g[kTok];
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    f[u] = z.f32(u, 0);
    c[u] = z.f32(u, gate);
    g[u] = z.f32(u, 2 * gate);
  }
  const V2 lb = a.lb != nullptr ? ld2(a.lb + p.c) : V2{0.0f, 0.0f};
  V2 H = a.h0 != nullptr ? ld2(a.h0 + p.b * d + p.c) : V2{0.0f, 0.0f};
  Map2 m = kSame;
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    // f, and (1 - f) c in the place of c; past the end f = 1 keeps the state
    const bool in = p.u0 + u < p.rows;
    f[u].x = in ? fmaf(1.0f - lb.x, sigmoid_hw(f[u].x), lb.x) : 1.0f;
    f[u].y = in ? fmaf(1.0f - lb.y, sigmoid_hw(f[u].y), lb.y) : 1.0f;
    c[u].x = (1.0f - f[u].x) * (c[u].x * sigmoid_hw(c[u].x));
    c[u].y = (1.0f - f[u].y) * (c[u].y * sigmoid_hw(c[u].y));
    m = {m.ax * f[u].x, fmaf(f[u].x, m.bx, c[u].x), m.ay * f[u].y, fmaf(f[u].y, m.by, c[u].y)};
  }
  maps[p.sub][p.lane] = m;
  // h0 is read before the chunk's map is published: h_last, which may be the
  // same array, is written by a chunk that has read the maps before it
  asm volatile("" : "+v"(H.x), "+v"(H.y) : : "memory");
  __syncthreads();
  const int64_t at = (p.b * a.nchunk + p.k) * d + p.c;
  Map2 whole = kSame;
  if constexpr (MANY) {
    uint64_t* words = a.words + p.b * a.nchunk * d + p.c;
    if (p.sub == 0) {
#pragma unroll 2
      for (int i = 0; i < kSubs; ++i) whole = then(whole, maps[i][p.lane]);
      if (p.col) publish_map(words, d, p.k, a.nchunk, whole);
    }
    H = carry_in(words, d, p.k, H, p.sub, p.lane, look);
    if (p.sub == 0 && p.col) publish_end(words, d, p.k, whole(H));
  }
  if (p.sub == 0 && p.col) st2(a.states + at, H);
  V2 h = H;
#pragma unroll 2
  for (int i = 0; i < p.sub; ++i) h = maps[i][p.lane](h);
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    h = {fmaf(f[u].x, h.x, c[u].x), fmaf(f[u].y, h.y, c[u].y)};
    o.store(u, {mlgru_out_gate(g[u].x, h.x), mlgru_out_gate(g[u].y, h.y)});
  }
  if (a.h_last != nullptr && p.col && p.k == a.nchunk - 1 && p.u0 < p.rows && p.u0 + kTok >= p.rows)
    st2(a.h_last + p.b * d + p.c, h);
}

// The same value, unknown to the compiler: what it derives from it again is
// computed again instead of being kept in registers from one pass over the
// tokens to the next.
__device__ __forceinline__ float afresh(float v) {
  asm volatile("" : "+v"(v));
  return v;
}

// p.c, computed again from the lane's number in its wave: kept from one use to
// the next it is what the registers spill.
__device__ __forceinline__ int64_t channel_afresh(const Place& p, int64_t d) {
  int all = -1;
  asm volatile("" : "+s"(all));
  const int64_t c = p.c0 + 2 * (__builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0)) % kLanes);
  return p.col ? c : d - 2;
}

struct BwdArgs {
  const float* z;
  const float* lb;
  const float* states;
  const void* dout;      // [B*T][d] bf16 or fp32
  const float* dh_last;  // nullptr: zero
  uint64_t* words;       // [B][nchunk][d], from the last chunk to the first
  uint32_t* tickets;
  uint16_t* dz;
  float* dh0;            // nullptr: not stored
  double* dlb_part;      // [B * nchunk][d], nullptr: not computed
  int64_t B, T, d, nchunk;
};

template <typename DT, bool MANY, bool NT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(4))) void mlgru_train_bwd_kernel(const BwdArgs a) {
  __shared__ Map2 maps[kSubs][kLanes], back[kSubs][kLanes];
  __shared__ double2 s_dlb[kSubs][kLanes];
  const int64_t d = a.d;
  const Place p = place<MANY>(a.T, d, a.B, a.nchunk, true, a.tickets);
  const Rows<NT> z(a.z, p, 3 * d, 4), dz(a.dz, p, 3 * d, 2);
  const Rows<NT> dout(static_cast<const DT*>(a.dout), p, d, sizeof(DT));
  const uint32_t gate = static_cast<uint32_t>(d) * 4u, dgate = static_cast<uint32_t>(d) * 2u;
  V2 zf[kTok], zc[kTok], zg[kTok], go[kTok];
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    zf[u] = z.f32(u, 0);
    zc[u] = z.f32(u, gate);
    zg[u] = z.f32(u, 2 * gate);
    if constexpr (sizeof(DT) == 4) go[u] = dout.f32(u, 0);
    else go[u] = dout.bf16(u);
  }
  const V2 lb = a.lb != nullptr ? ld2(a.lb + p.c) : V2{0.0f, 0.0f};
  const int64_t at = (p.b * a.nchunk + p.k) * d + p.c;
  const V2 H = ld2(a.states + at);
  V2 G = a.dh_last != nullptr ? ld2(a.dh_last + p.b * d + p.c) : V2{0.0f, 0.0f};

  // sf = sigmoid(zf) in the place of zf, c in that of zc, and
  // q = s(zc) (1 + zc (1 - s(zc))); past the end f = 1 and e = 0
  V2 q[kTok];
  auto forget = [](float sf, float lb, bool in) { return in ? fmaf(1.0f - lb, sf, lb) : 1.0f; };
  Map2 m = kSame;
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    const bool in = p.u0 + u < p.rows;
    zf[u] = {sigmoid_hw(zf[u].x), sigmoid_hw(zf[u].y)};
    const float sx = sigmoid_hw(zc[u].x), sy = sigmoid_hw(zc[u].y);
    q[u] = {sx * fmaf(zc[u].x, 1.0f - sx, 1.0f), sy * fmaf(zc[u].y, 1.0f - sy, 1.0f)};
    zc[u] = {zc[u].x * sx, zc[u].y * sy};
    const float fx = forget(zf[u].x, lb.x, in), fy = forget(zf[u].y, lb.y, in);
    m = {m.ax * fx, fmaf(fx, m.bx, (1.0f - fx) * zc[u].x), m.ay * fy, fmaf(fy, m.by, (1.0f - fy) * zc[u].y)};
  }
  maps[p.sub][p.lane] = m;
  __syncthreads();
  V2 h = H;
#pragma unroll 2
  for (int i = 0; i < p.sub; ++i) h = maps[i][p.lane](h);
  // the state before each token, e in the place of zg, dz's third part, and
  // the map of the gradient through the half wave's tokens
  V2 hp[kTok];
  m = kSame;
#pragma unroll
  for (int u = 0; u < kTok; ++u) {
    const bool in = p.u0 + u < p.rows;
    hp[u] = h;
    zf[u] = {afresh(zf[u].x), afresh(zf[u].y)};
    const float fx = forget(zf[u].x, lb.x, in), fy = forget(zf[u].y, lb.y, in);
    h = {fmaf(fx, h.x, (1.0f - fx) * zc[u].x), fmaf(fy, h.y, (1.0f - fy) * zc[u].y)};
    const float sx = sigmoid_hw(h.x), sy = sigmoid_hw(h.y);
    const float gx = go[u].x * sx, gy = go[u].y * sy;
    dz.store_bf16(u, 2 * dgate, gx, gy);
    zg[u] = {in ? gx * (1.0f - sx) * zg[u].x : 0.0f, in ? gy * (1.0f - sy) * zg[u].y : 0.0f};
    m.ax *= fx;
    m.ay *= fy;
    m.bx = fmaf(m.ax, zg[u].x, m.bx);
    m.by = fmaf(m.ay, zg[u].y, m.by);
  }
  back[p.sub][p.lane] = m;
  asm volatile("" : "+v"(G.x), "+v"(G.y) : : "memory");  // dh_last is read by here, as h0 above: it may be dh0
  __syncthreads();
  Map2 whole = kSame;
  if constexpr (MANY) {
    const int64_t pos = a.nchunk - 1 - p.k;
    uint64_t* words = a.words + p.b * a.nchunk * d + channel_afresh(p, d);
    if (p.sub == 0) {
#pragma unroll 2
      for (int i = kSubs - 1; i >= 0; --i) whole = then(whole, back[i][p.lane]);
      if (p.col) publish_map(words, d, pos, a.nchunk, whole);
    }
    G = carry_in(words, d, pos, G, p.sub, p.lane, maps);  // `maps` is free by now
    if (p.sub == 0 && p.col) publish_end(words, d, pos, whole(G));
  }
#pragma unroll 2
  for (int i = kSubs - 1; i > p.sub; --i) G = back[i][p.lane](G);
  double dlx = 0.0, dly = 0.0;
#pragma unroll
  for (int u = kTok - 1; u >= 0; --u) {
    const bool in = p.u0 + u < p.rows;
    // one channel: its gradients, and G carried to the token before
    auto one = [in, &forget](float sf, float c, float q, float e, float hp, float lb, float& G, float& df, float& dc,
                             double& dl) {
      const float f = forget(sf, lb, in), dh = G + e, w = dh * (hp - c), k = w * (1.0f - sf);
      df = k * ((1.0f - lb) * sf);
      dc = dh * (1.0f - f) * q;
      dl += static_cast<double>(in ? k : 0.0f);
      G = f * dh;
    };
    float dfx, dfy, dcx, dcy;
    zf[u] = {afresh(zf[u].x), afresh(zf[u].y)};
    one(zf[u].x, zc[u].x, q[u].x, zg[u].x, hp[u].x, lb.x, G.x, dfx, dcx, dlx);
    one(zf[u].y, zc[u].y, q[u].y, zg[u].y, hp[u].y, lb.y, G.y, dfy, dcy, dly);
    dz.store_bf16(u, 0, dfx, dfy);
    dz.store_bf16(u, dgate, dcx, dcy);
  }
  if (p.k == 0 && p.sub == 0 && p.col && a.dh0 != nullptr) st2(a.dh0 + p.b * d + channel_afresh(p, d), G);
  if (a.dlb_part != nullptr) {
    s_dlb[p.sub][p.lane] = make_double2(dlx, dly);
    __syncthreads();
    if (p.sub == 0 && p.col) {
      double x = 0.0, y = 0.0;
#pragma unroll
      for (int i = 0; i < kSubs; ++i) {
        x += s_dlb[i][p.lane].x;
        y += s_dlb[i][p.lane].y;
      }
      *reinterpret_cast<double2*>(a.dlb_part + (p.b * a.nchunk + p.k) * d + channel_afresh(p, d)) = make_double2(x, y);
    }
  }
}

// Empties the words and sets the tickets to 0.
constexpr int kFill = 256;
__global__ __launch_bounds__(kFill) void mlgru_train_clear_kernel(ulonglong2* __restrict__ words, int64_t n2,
                                                                  uint32_t* __restrict__ tickets) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kFill + threadIdx.x;
  if (i < n2) words[i] = make_ulonglong2(kEmpty, kEmpty);
  if (i == 0) *tickets = 0u;
}

hipError_t clear(uint64_t* words, int64_t n, uint32_t* tickets, hipStream_t stream) {
  const int64_t n2 = n / 2;
  hipLaunchKernelGGL(mlgru_train_clear_kernel, dim3(static_cast<unsigned>((n2 + kFill - 1) / kFill)), dim3(kFill), 0,
                     stream, reinterpret_cast<ulonglong2*>(words), n2, tickets);
  return hipGetLastError();
}

}  // namespace

int64_t mlgru_train_chunks(int64_t T) { return (T + kChunk - 1) / kChunk; }

int64_t mlgru_train_blocks(int64_t B, int64_t T, int64_t d) {
  return B * mlgru_train_chunks(T) * ((d + kCh - 1) / kCh);
}

hipError_t launch_mlgru_train_scan(const MlgruTrainArgs& p, float* o, float* h_last, float* states, uint64_t* words,
                                   uint32_t* tickets, hipStream_t stream) {
  const int64_t nchunk = mlgru_train_chunks(p.T);
  const FwdArgs a{p.z, p.lb, p.h0, words, tickets, states, o, h_last, p.B, p.T, p.d, nchunk};
  const dim3 grid(static_cast<unsigned>(mlgru_train_blocks(p.B, p.T, p.d)));
  const bool nt = p.B * p.T * p.d * 16 >= kLastLevelBytes;  // z and o'
  if (nchunk > 1) {
    if (const hipError_t e = clear(words, p.B * nchunk * p.d, tickets, stream); e != hipSuccess) return e;
    if (nt)
      hipLaunchKernelGGL((mlgru_train_fwd_kernel<true, true>), grid, dim3(kThreads), 0, stream, a);
    else
      hipLaunchKernelGGL((mlgru_train_fwd_kernel<true, false>), grid, dim3(kThreads), 0, stream, a);
  } else if (nt) {
    hipLaunchKernelGGL((mlgru_train_fwd_kernel<false, true>), grid, dim3(kThreads), 0, stream, a);
  } else {
    hipLaunchKernelGGL((mlgru_train_fwd_kernel<false, false>), grid, dim3(kThreads), 0, stream, a);
  }
  return hipGetLastError();
}

namespace {
template <typename DT>
hipError_t launch_bwd(const BwdArgs& a, unsigned blocks, hipStream_t stream) {
  const dim3 grid(blocks), block(kThreads);
  const bool nt = a.B * a.T * a.d * static_cast<int64_t>(18 + sizeof(DT)) >= kLastLevelBytes;  // z, do and dz
  if (a.nchunk > 1) {
    if (nt)
      hipLaunchKernelGGL((mlgru_train_bwd_kernel<DT, true, true>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((mlgru_train_bwd_kernel<DT, true, false>), grid, block, 0, stream, a);
  } else if (nt) {
    hipLaunchKernelGGL((mlgru_train_bwd_kernel<DT, false, true>), grid, block, 0, stream, a);
  } else {
    hipLaunchKernelGGL((mlgru_train_bwd_kernel<DT, false, false>), grid, block, 0, stream, a);
  }
  return hipGetLastError();
}
}  // namespace

hipError_t launch_mlgru_scan_bwd(const MlgruTrainArgs& p, const float* states, const void* dout, bool dout_is_f32,
                                 const float* dh_last, uint16_t* dz, float* dh0, uint64_t* words, uint32_t* tickets,
                                 double* dlb_part, hipStream_t stream) {
  const int64_t nchunk = mlgru_train_chunks(p.T);
  const BwdArgs a{p.z, p.lb, states, dout, dh_last, words, tickets, dz, dh0, dlb_part, p.B, p.T, p.d, nchunk};
  if (nchunk > 1) {
    if (const hipError_t e = clear(words, p.B * nchunk * p.d, tickets, stream); e != hipSuccess) return e;
  }
  const unsigned blocks = static_cast<unsigned>(mlgru_train_blocks(p.B, p.T, p.d));
  return dout_is_f32 ? launch_bwd<float>(a, blocks, stream) : launch_bwd<uint16_t>(a, blocks, stream);
}

}  // namespace mmf
