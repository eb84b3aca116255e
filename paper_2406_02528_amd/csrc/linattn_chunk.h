// Linear attention with a decay per head over chunks of tokens.
//
// A pass computes, for the queries q, keys k and values v of B sequences and H
// heads (tokens i = 0 .. T-1, in the order of the pass: forward, or from the
// last token to the first) and l = decay[h],
//   o_i = beta (alpha sum_{s <= i} l^(i-s) (q_i . k_s) v_s + l^i E^T q_i)
// with E [Dk][Dv] the state before token 0, its decay to token 0 included.
// The forward is one pass (q, k, v; E = l S_0, beta = scale); the backward is
// three with the roles exchanged:
//   dq: queries do, keys v, values k,  forward,  E = (l S_0)^T, beta = scale
//   dk: queries v, keys do, values q,  backward, E = dS_last^T, alpha = scale
//   dv: queries k, keys q, values do,  backward, E = dS_last,   alpha = scale
//
// Within a chunk of C tokens the sum over s is two products on the matrix
// cores with the decays between them; the chunk's keys and values then join
// the state, E <- l^C E + alpha sum_s l^(C-s) k_s v_s^T.  Long sequences are
// cut into segments of chunks that run in parallel: a first kernel gives each
// segment's own sum, a second joins them into the states that enter the
// segments, from which the pass itself starts.
//
// A workgroup of four waves holds a state of Dk rows and 64 ET columns (16 ET
// per wave) in the accumulators of its matrix instructions.  The layouts are
// chosen so that neither the state nor the values ever pass through LDS
// (v_mfma_f32_16x16x32_bf16; lane = 16 g + n, g = 0..3, n = 0..15; A: row n,
// B: column n, eight contraction slots j per lane; D: column n, rows 4 g + r):
//   - the state's tile (b, i) has row 4 g + r = entry d = 64 b + 16 g + 4 r + i
//     and column n = entry e = ET n + f of the wave's columns, so that a lane
//     keeps ET neighbouring columns;
//   - as the operand B of q E its slots are d = 64 b + 16 g + 4 (j%4) + 2 p +
//     j/4 (tiles i = 2 p and 2 p + 1 side by side), so a lane's part of a
//     query or key is 16 consecutive entries of its row, in two operands p;
//   - tokens as contraction slots are s = 32 c + 16 (j/4) + 4 g + j%4, which is
//     how the transposed products k q^T leave their rows, two tiles side by
//     side: they go to LDS with 8-byte stores in place;
//   - a lane's part of the values (and of the transposed keys) are 8 tokens
//     with ET (4) neighbouring entries each, transposed in registers.
//
// Numerics: bf16 inputs are exact operands.  fp32 values (fp32 inputs, the
// decayed products, the state, the weighted keys) go to the matrix cores as
// sums of 2 or 3 bf16 parts (2^-16 or 2^-24 relative), with the products of
// parts down to the same size: 3 parts where the result is fp32 (o from fp32
// inputs, states), 2 where it is rounded to bf16.  Sums are fp32; powers of l
// come from fp64.
#pragma once
#include "linattn.h"
#include "mmf_device.h"
#include "row_vec.h"

namespace mmf {
namespace la {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v4f mfma(v4i a, v4i b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// Eight fp32 values as N bf16 parts whose sum they are.
template <int N>
__device__ __forceinline__ void split8(const float* x, v4i (&p)[N]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    float a = x[2 * w], b = x[2 * w + 1];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t u = pack_bf16(a, b);
      p[i][w] = static_cast<int>(u);
      if (i + 1 < N) {
        a -= bf16_lo(u);
        b -= bf16_hi(u);
      }
    }
  }
}

// acc += a b over the parts' products of relative size above 2^(-8 L).
template <int L, int NA, int NB>
__device__ __forceinline__ v4f mma(const v4i (&a)[NA], const v4i (&b)[NB], v4f acc) {
#pragma unroll
  for (int i = NA - 1; i >= 0; --i)
#pragma unroll
    for (int j = NB - 1; j >= 0; --j)
      if (i + j < L) acc = mfma(a[i], b[j], acc);
  return acc;
}

// How an operand's elements are stored: bf16, fp32, or as the pass says.
enum Kind { kBf16, kF32, kEither };

// N (1, 2, 4, 16) consecutive elements at byte offset off, zero past the
// resource; bf16 ones two to a dword.
template <int N>
__device__ __forceinline__ void load_f32(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t (&w)[N]) {
  if constexpr (N == 1) {
    w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0);
  } else if constexpr (N == 2) {
    const Words<2> p = load_stream<2, false>(r, off);
    w[0] = p.w[0];
    w[1] = p.w[1];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const Words<4> p = load_stream<4, false>(r, off + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i + j] = p.w[j];
    }
  }
}
template <int N>
__device__ __forceinline__ void load_bf16(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t (&w)[N]) {
  if constexpr (N == 1) {
    w[0] = __builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0);
  } else {
    uint32_t h[N / 2];
    load_f32<N / 2>(r, off, h);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = h[i];
  }
}
// The element e of what was loaded.
template <int N>
__device__ __forceinline__ float element(const uint32_t (&w)[N], bool f32, int e) {
  if (f32) return __uint_as_float(w[e]);
  if (N == 1) return bf16_lo(w[0]);
  return e & 1 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
}

// Rows of one operand: token i of a chunk and `width` elements of its head.
template <Kind K>
struct Rows {
  __amdgpu_buffer_rsrc_t r;
  uint32_t ld;      // bytes of a row
  int width;
  bool f32_;
  __device__ __forceinline__ bool f32() const { return K == kEither ? f32_ : K == kF32; }
  // `n` rows from row `row`.
  __device__ __forceinline__ void at(const LinattnOperand& x, int64_t row, int n, int64_t h, int w) {
    f32_ = x.is_f32;
    const uint32_t size = f32() ? 4u : 2u;
    ld = static_cast<uint32_t>(x.ld) * size;
    width = w;
    char* const base = const_cast<char*>(static_cast<const char*>(x.p)) + (row * x.ld + h * w) * static_cast<int64_t>(size);
    r = __builtin_amdgcn_make_buffer_rsrc(base, 0, static_cast<int>(static_cast<uint32_t>(n - 1) * ld + w * size), kBufferWord3);
  }
  // Elements d .. d + N - 1 of local row i; `on` false: zeros.
  template <int N>
  __device__ __forceinline__ void load(int i, int d, bool on, uint32_t (&w)[N]) const {
    const uint32_t size = f32() ? 4u : 2u;
    const uint32_t off = on && d < width ? static_cast<uint32_t>(i) * ld + static_cast<uint32_t>(d) * size : 0x80000000u;
    if (f32()) load_f32<N>(r, off, w);
    else load_bf16<N>(r, off, w);
  }
};

// MODE: parts of fp32 values in the products of o.  NKT: parts of the weighted
// keys in the state's.  DK: Dk padded to 64s.  STATE: the segment's own sum
// only (no queries, no o).
template <Kind KQ, Kind KK, Kind KV, bool OF32, int MODE, int NKT, int DK, int ET, int C, bool STATE>
__global__ __launch_bounds__(256) void linattn_chunk_kernel(const LinattnPass p) {
  constexpr int kB = DK / 64;        // 64s of Dk
  constexpr int kT = C / 16;         // tiles of tokens
  constexpr int kS = C / 32;         // contraction steps over tokens
  constexpr int NQ = KQ == kBf16 ? 1 : MODE, NK = KK == kBf16 ? 1 : MODE;
  constexpr int NV = KV == kBf16 ? 1 : STATE ? NKT : MODE;
  constexpr int kQFrags = STATE ? 1 : kT * kB * 2 * NQ;
  constexpr int kKFrags = kB * 4 * kS * NKT;
  constexpr int kPFrags = STATE ? 1 : kT * kS * MODE;
  __shared__ v4i q_lds[kQFrags][kWave];   // [t-tile][64s][p][part]
  __shared__ v4i k_lds[kKFrags][kWave];   // [64s][i][token step][part]
  __shared__ v4i p_lds[kPFrags][kWave];   // [t-tile][token step][part]
  __shared__ float pw[C + 1];             // l^i
  __shared__ int s_bad;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  uint32_t blk = blockIdx.x;
  const uint32_t tile = blk % p.tiles;
  blk /= p.tiles;
  const uint32_t seg = blk % p.nseg;
  const uint32_t bh = blk / p.nseg;
  if (STATE && seg + 1 == p.nseg && !p.join_last) return;  // no segment follows
  const int64_t b = bh / p.H, h = bh % p.H;
  const int e0 = static_cast<int>(tile) * 64 * ET + wave * 16 * ET + ET * n;  // the lane's columns e0 .. e0 + ET - 1
  const bool ewave = static_cast<int>(tile) * 64 * ET + wave * 16 * ET < p.Dv;
  const bool eon = e0 < p.Dv;

  // powers of l: fp64, by squaring (any l, 0 among them)
  if (threadIdx.x <= C) {
    double x = p.decay[h], y = 1.0;
    for (int i = threadIdx.x; i != 0; i >>= 1) {
      if (i & 1) y *= x;
      x *= x;
    }
    pw[threadIdx.x] = static_cast<float>(y);
  }
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();

  const float alpha = p.alpha, beta = p.beta;
  // decays between the rows of a transposed product's tile (keys 4 g + r) and
  // its column (query n), on the diagonal and one tile before it, and of the
  // rows 4 g + r of q E
  float w_diag[4], w_off[4], w_row[4];
  if constexpr (!STATE) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int s = 4 * g + r;
      w_diag[r] = n >= s ? alpha * beta * pw[n >= s ? n - s : 0] : 0.0f;
      w_off[r] = alpha * beta * pw[16 + n - s];
      w_row[r] = beta * pw[s];
    }
  }

  // the state, [64s][i][f]
  v4f st[kB][4][ET];
#pragma unroll
  for (int x = 0; x < kB; ++x)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int f = 0; f < ET; ++f) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v = 0.0f;
          const int d = 64 * x + 16 * g + 4 * r + i, e = e0 + f;
          if (!STATE && eon && d < p.Dk) {
            if (p.joined != nullptr) {
              v = p.joined[((static_cast<int64_t>(bh) * p.nseg + seg) * p.Dk + d) * p.Dv + e];
            } else if (p.s_in != nullptr) {
              v = p.s_in[static_cast<int64_t>(bh) * p.Dk * p.Dv + static_cast<int64_t>(d) * p.in_d + static_cast<int64_t>(e) * p.in_e];
              if (!p.rev) v *= pw[1];
            }
          }
          st[x][i][f][r] = v;
        }
      }

  const int64_t begin = static_cast<int64_t>(seg) * p.seg_tokens;
  const int64_t end = begin + p.seg_tokens < p.T ? begin + p.seg_tokens : p.T;
  int64_t single = begin;  // tokens before this one go one by one
  Rows<KQ> rq;
  Rows<KK> rk;
  Rows<KV> rv;
  for (int64_t i0 = begin; i0 < end;) {
    const int64_t left = end - i0;
    const int tc = i0 < single ? 1 : left < C ? static_cast<int>(left) : C;
    const int64_t row = b * p.T + (p.rev ? p.T - i0 - tc : i0);
    const auto local = [&](int i) { return p.rev ? tc - 1 - i : i; };
    rk.at(p.k, row, tc, h, p.Dk);
    rv.at(p.v, row, tc, h, p.Dv);

    // --- values of the wave's columns, and whether they are all finite
    v4i vf[kS][ET][NV];
    float bad = 0.0f;
    {
      uint32_t w[kS][8][ET];
#pragma unroll
      for (int c = 0; c < kS; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int s = 32 * c + 16 * (j / 4) + 4 * g + j % 4;
          rv.template load<ET>(local(s), e0, s < tc, w[c][j]);
        }
#pragma unroll
      for (int c = 0; c < kS; ++c)
#pragma unroll
        for (int f = 0; f < ET; ++f) {
          float x[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            x[j] = element<ET>(w[c][j], rv.f32(), f);
            bad = fmaf(x[j], 0.0f, bad);
          }
          split8<NV>(x, vf[c][f]);
        }
    }
    if (!STATE && __any(bad != 0.0f) && lane == 0) s_bad = 1;

    // --- weighted transposed keys: token step and 64s by wave
    for (int u = wave; u < kB * kS; u += 4) {
      const int x = u / kS, c = u % kS;
      uint32_t w[8][4];
      float wt[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int s = 32 * c + 16 * (j / 4) + 4 * g + j % 4;
        rk.template load<4>(local(s), 64 * x + 4 * n, s < tc, w[j]);
        // decays to the next chunk's first token, or (the forward's last) to
        // the token itself
        const int to = i0 + tc == p.T && !p.rev ? tc - 1 - s : tc - s;
        wt[j] = alpha * pw[to > 0 ? to : 0];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y[8];
        v4i f[NKT];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = element<4>(w[j], rk.f32(), i) * wt[j];
        split8<NKT>(y, f);
#pragma unroll
        for (int k = 0; k < NKT; ++k) k_lds[((x * 4 + i) * kS + c) * NKT + k][lane] = f[k];
      }
    }

    if constexpr (!STATE) {
      // --- queries: token tile by wave
      rq.at(p.q, row, tc, h, p.Dk);
      v4i kf[kB * 2][NK];   // the wave's own keys
      if (wave < kT) {
        const int t = 16 * wave + n;
#pragma unroll
        for (int x = 0; x < kB; ++x) {
          uint32_t w[16], u[16];
          rq.template load<16>(local(t), 64 * x + 16 * g, t < tc, w);
          rk.template load<16>(local(t), 64 * x + 16 * g, t < tc, u);
#pragma unroll
          for (int pr = 0; pr < 2; ++pr) {
            float y[8], z[8];
            v4i f[NQ];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              y[j] = element<16>(w, rq.f32(), 4 * (j % 4) + 2 * pr + j / 4);
              z[j] = element<16>(u, rk.f32(), 4 * (j % 4) + 2 * pr + j / 4);
            }
            split8<NQ>(y, f);
            split8<NK>(z, kf[x * 2 + pr]);
#pragma unroll
            for (int k = 0; k < NQ; ++k) q_lds[((wave * kB + x) * 2 + pr) * NQ + k][lane] = f[k];
          }
        }
      }
      __syncthreads();
      if (tc > 1 && __builtin_amdgcn_readfirstlane(s_bad) != 0) {  // a value that is not finite reaches no token before it
        single = i0 + tc;
        __syncthreads();
        if (threadIdx.x == 0) s_bad = 0;
        __syncthreads();
        continue;
      }

      const auto query = [&](int t, int kb, v4i (&f)[NQ]) {
#pragma unroll
        for (int k = 0; k < NQ; ++k) f[k] = q_lds[(t * kB * 2 + kb) * NQ + k][lane];
      };
      // --- keys x queries, decayed: rows of the wave's token tile
      if (wave < kT) {
        float wx = 1.0f;
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          if (t < wave) {
            if (t == wave - 1 && (wave & 1)) {  // the half of its operand that no tile fills
#pragma unroll
              for (int k = 0; k < MODE; ++k)
                reinterpret_cast<uint2*>(&p_lds[(t * kS + wave / 2) * MODE + k][lane])[1] = make_uint2(0u, 0u);
            }
            continue;
          }
          v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int kb = 0; kb < kB * 2; ++kb) {
            v4i f[NQ];
            query(t, kb, f);
            acc = mma<MODE>(kf[kb], f, acc);
          }
          float y[4];
          if (t == wave) {
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = n >= 4 * g + r ? acc[r] * w_diag[r] : 0.0f;
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = acc[r] * (w_off[r] * wx);
            wx *= pw[16];
          }
#pragma unroll
          for (int k = 0; k < MODE; ++k) {
            const uint2 u = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
            reinterpret_cast<uint2*>(&p_lds[(t * kS + wave / 2) * MODE + k][lane])[wave & 1] = u;
            y[0] -= bf16_lo(u.x);
            y[1] -= bf16_hi(u.x);
            y[2] -= bf16_lo(u.y);
            y[3] -= bf16_hi(u.y);
          }
        }
      }
      // --- queries x state
      v4f o[kT][ET];
      if (ewave) {
#pragma unroll
        for (int t = 0; t < kT; ++t)
#pragma unroll
          for (int f = 0; f < ET; ++f) o[t][f] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int x = 0; x < kB; ++x)
#pragma unroll
          for (int pr = 0; pr < 2; ++pr) {
            v4i sf[ET][MODE];
#pragma unroll
            for (int f = 0; f < ET; ++f) {
              float y[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) y[j] = st[x][2 * pr + j / 4][f][j % 4];
              split8<MODE>(y, sf[f]);
            }
#pragma unroll
            for (int t = 0; t < kT; ++t) {
              v4i q[NQ];
              query(t, x * 2 + pr, q);
#pragma unroll
              for (int f = 0; f < ET; ++f) o[t][f] = mma<MODE>(q, sf[f], o[t][f]);
            }
          }
        float wx = 1.0f;
#pragma unroll
        for (int t = 0; t < kT; ++t) {
#pragma unroll
          for (int f = 0; f < ET; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[t][f][r] *= w_row[r] * wx;
          wx *= pw[16];
        }
      }
      __syncthreads();
      if (threadIdx.x == 0) s_bad = 0;
      if (ewave) {
        // --- products x values
#pragma unroll
        for (int t = 0; t < kT; ++t)
#pragma unroll
          for (int c = 0; c < kS; ++c) {
            if (2 * c > t) continue;
            v4i f[MODE];
#pragma unroll
            for (int k = 0; k < MODE; ++k) f[k] = p_lds[(t * kS + c) * MODE + k][lane];
#pragma unroll
            for (int e = 0; e < ET; ++e) o[t][e] = mma<MODE>(f, vf[c][e], o[t][e]);
          }
        // --- store
        if (eon) {
#pragma unroll
          for (int t = 0; t < kT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int i = 16 * t + 4 * g + r;
              if (i < tc) {
                const int64_t at = (row + local(i)) * p.ldo + h * p.Dv + e0;
                if constexpr (OF32) {
                  float* const y = static_cast<float*>(p.o) + at;
                  if constexpr (ET == 2) *reinterpret_cast<float2*>(y) = make_float2(o[t][0][r], o[t][1][r]);
                  else *y = o[t][0][r];
                } else {
                  uint16_t* const y = static_cast<uint16_t*>(p.o) + at;
                  if constexpr (ET == 2) *reinterpret_cast<uint32_t*>(y) = pack_bf16(o[t][0][r], o[t][1][r]);
                  else *y = static_cast<uint16_t>(pack_bf16(o[t][0][r], 0.0f));
                }
              }
            }
        }
      }
    } else {
      __syncthreads();
    }

    // --- keys x values into the state
    if (ewave) {
      const float w = pw[i0 + tc == p.T && !p.rev ? tc - 1 : tc];
#pragma unroll
      for (int x = 0; x < kB; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
          for (int f = 0; f < ET; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r) st[x][i][f][r] *= w;
#pragma unroll
          for (int c = 0; c < kS; ++c) {
            v4i k[NKT];
#pragma unroll
            for (int y = 0; y < NKT; ++y) k[y] = k_lds[((x * 4 + i) * kS + c) * NKT + y][lane];
#pragma unroll
            for (int f = 0; f < ET; ++f) st[x][i][f] = mma<NKT>(k, vf[c][f], st[x][i][f]);
          }
        }
    }
    __syncthreads();
    i0 += tc;
  }

  // the segment's own sum, or the state after the last token
  float* out = nullptr;
  int64_t od = p.Dv, oe = 1;
  if (STATE) {
    out = p.joined + (static_cast<int64_t>(bh) * p.nseg + seg) * p.Dk * p.Dv;
  } else if (p.s_out != nullptr && seg + 1 == p.nseg) {
    out = p.s_out + static_cast<int64_t>(bh) * p.Dk * p.Dv;
    od = p.in_d;
    oe = p.in_e;
  }
  if (out != nullptr && eon) {
#pragma unroll
    for (int x = 0; x < kB; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int f = 0; f < ET; ++f)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int d = 64 * x + 16 * g + 4 * r + i;
            if (d < p.Dk) out[d * od + (e0 + f) * oe] = st[x][i][f][r];
          }
  }
}

constexpr int chunk_tokens(int DK) { return DK == 256 ? 32 : 64; }

template <Kind KQ, Kind KK, Kind KV, bool OF32, int MODE, int NKT, bool STATE>
hipError_t launch_pass(const LinattnPass& p, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(p.B * p.H * p.nseg * p.tiles));
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, p);
    return hipGetLastError();
  };
#define MMF_DIMS(DK)                                                                                          \
  return p.et == 1 ? go(linattn_chunk_kernel<KQ, KK, KV, OF32, MODE, NKT, DK, 1, chunk_tokens(DK), STATE>)    \
                   : go(linattn_chunk_kernel<KQ, KK, KV, OF32, MODE, NKT, DK, 2, chunk_tokens(DK), STATE>)
  if (p.Dk <= 64) MMF_DIMS(64);
  if (p.Dk <= 128) MMF_DIMS(128);
  MMF_DIMS(256);
#undef MMF_DIMS
}

}  // namespace la
}  // namespace mmf
