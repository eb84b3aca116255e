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
// A workgroup of eight waves holds a state of Dk rows and 64 ET columns in the
// accumulators of its matrix instructions: 16 ET columns per wave and, of each
// four neighbouring rows, two (waves 0-3 and 4-7).  q E of a wave is then a
// part of the sum; each wave finishes half of the token tiles with the other
// half's part from LDS.  A chunk's rows are loaded while the chunk before is
// worked on.  The layouts are chosen so that neither the state nor the values
// ever pass through LDS (v_mfma_f32_16x16x32_bf16; lane = 16 g + n, g = 0..3, n
// = 0..15; A: row n, B: column n, eight contraction slots j per lane; D: column
// n, rows 4 g + r):
//   - the state's tile (x, i) has row m = entry d = 64 x + 4 pi(m) + i (pi a
//     permutation of 16, below) and column n = entry e = ET n + f of the wave's
//     columns, so that a lane keeps ET neighbouring columns;
//   - as the operand B of q E its slots are the rows m = 4 g + j%4 of tiles i =
//     2 h + j/4 (side by side: h = 0 waves 0-3, 1 waves 4-7), so a lane's part of a
//     query or key is four times four entries of its row, in two operands h; pi
//     puts the four lanes g of a row side by side in each load (16 bytes of fp32:
//     d = 16 r + 4 g + i, of bf16: d = 8 g + 4 (r%2) + 32 (r/2) + i), where 16
//     entries in a row per lane would have each load touch four times the lines;
//   - tokens as contraction slots are s = 32 c + 16 (j/4) + 4 g + j%4, which is
//     how the transposed products k q^T leave their rows, two tiles side by
//     side: they go to LDS with 8-byte stores in place;
//   - a lane's part of the values (and of the transposed keys) are 8 (4) tokens
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
typedef unsigned int v2u __attribute__((ext_vector_type(2)));
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
template <int N, int W>
__device__ __forceinline__ void load_bf16(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t (&w)[W]) {
  if constexpr (N == 1) {
    w[0] = __builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0);
  } else {
    uint32_t h[N / 2];
    load_f32<N / 2>(r, off, h);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = h[i];
  }
}
// Rows of one operand in a chunk.  A row past the chunk's tokens has an offset
// past the resource (forward: above it; backward, where token i is row tc - 1 -
// i: below 0, which is far above it), so it reads as zero with no mask; so
// has a column past the head's width (kOff, which no token's step reaches:
// 64 rows take at most 2^29 bytes).
constexpr uint32_t kOff = 0x80000000u;
template <Kind K>
struct Rows {
  __amdgpu_buffer_rsrc_t r;
  uint32_t base;    // of token 0
  int step;         // from a token to the next
  int width;
  bool f32_;
  __device__ __forceinline__ bool f32() const { return K == kEither ? f32_ : K == kF32; }
  // `tc` rows from row `row` of head h, whose entries are `w`.
  __device__ __forceinline__ void at(const LinattnOperand& x, int64_t row, int tc, int64_t h, int w, bool rev) {
    f32_ = x.is_f32;
    const int size = f32() ? 4 : 2, ld = static_cast<int>(x.ld) * size;
    width = w;
    step = rev ? -ld : ld;
    base = rev ? static_cast<uint32_t>((tc - 1) * ld) : 0u;
    char* const p = const_cast<char*>(static_cast<const char*>(x.p)) + (row * x.ld + h * w) * size;
    r = __builtin_amdgcn_make_buffer_rsrc(p, 0, (tc - 1) * ld + w * size, kBufferWord3);
  }
  // A lane's offset: of token i and column d.  Not a constant of the loop for
  // the compiler, which would keep an offset in registers for every load.
  __device__ __forceinline__ uint32_t lane(int i, int d) const {
    uint32_t o = d < width ? base + static_cast<uint32_t>(i * step + d * (f32() ? 4 : 2)) : kOff;
    asm volatile("" : "+v"(o));
    return o;
  }
  // N elements, i tokens behind the lane's.
  template <int N, int W>
  __device__ __forceinline__ void load(uint32_t lane, int i, uint32_t (&w)[W]) const {
    const uint32_t off = lane + static_cast<uint32_t>(i * step);
    if constexpr (K != kBf16) {
      if (f32()) {
        load_f32<N>(r, off, w);
        return;
      }
    }
    if constexpr (K != kF32) load_bf16<N>(r, off, w);
  }
};

// pi: in fours of fp32 (FOURS) or eights of bf16, see above.
template <bool FOURS>
__device__ __forceinline__ int pi(int m) {
  const int g = m >> 2, r = m & 3;
  return FOURS ? g + 4 * r : 2 * g + (r & 1) + 8 * (r >> 1);
}
// A lane's 16 entries of the 64 from d0 of the token at its offset: rows 4 g + r
// of tile i at w's element 4 r + i.
template <bool FOURS, Kind K, int W>
__device__ __forceinline__ void load_entries(const Rows<K>& x, int token, int d0, int g, uint32_t (&w)[W]) {
  constexpr int kRun = FOURS ? 4 : 8;   // entries side by side
#pragma unroll
  for (int c = 0; c < 16 / kRun; ++c) {
    const uint32_t o = x.lane(token, d0 + kRun * g + 4 * kRun * c);
    if constexpr (K == kBf16) {
      uint32_t h[kRun / 2];
      load_f32<kRun / 2>(x.r, o, h);
#pragma unroll
      for (int i = 0; i < kRun / 2; ++i) w[kRun / 2 * c + i] = h[i];
    } else {
      uint32_t h[kRun];
      if (x.f32()) {
        load_f32<kRun>(x.r, o, h);
#pragma unroll
        for (int i = 0; i < kRun; ++i) w[kRun * c + i] = h[i];
      } else if constexpr (K == kEither) {
        load_f32<kRun / 2>(x.r, o, reinterpret_cast<uint32_t(&)[kRun / 2]>(h));
#pragma unroll
        for (int i = 0; i < kRun / 2; ++i) w[kRun / 2 * c + i] = h[i];
      }
    }
  }
}

// Dwords that N elements of a kind take in registers.
template <Kind K, int N>
constexpr int kDwords = K == kBf16 && N > 1 ? N / 2 : N;

// Eight elements as operand parts: of bf16 elements the bits themselves, two
// (word, half) each.
template <Kind K, int NP, typename At>
__device__ __forceinline__ void operand(At&& at, v4i (&f)[NP]) {
  if constexpr (K == kBf16) {
    static_assert(NP == 1, "bf16 operands are exact");
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const auto a = at(2 * w), b = at(2 * w + 1);
      const uint32_t sel = (a.half ? 0x0302u : 0x0100u) | ((b.half ? 0x0706u : 0x0504u) << 16);
      f[0][w] = static_cast<int>(__builtin_amdgcn_perm(b.word, a.word, sel));
    }
  } else {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = at(j).value();
    split8<NP>(x, f);
  }
}
struct Element {
  uint32_t word;
  bool half, f32;
  __device__ __forceinline__ float value() const { return f32 ? __uint_as_float(word) : half ? bf16_hi(word) : bf16_lo(word); }
};
template <int N>
__device__ __forceinline__ Element element(const uint32_t (&w)[N], bool f32, int e) {
  const uint32_t whole = w[e], pair = w[e / 2];
  return {f32 ? whole : pair, !f32 && (e & 1) != 0, f32};
}
// Whether any of N elements of several tokens is not finite: 0 in `bad` else.
template <int count, int N>
__device__ __forceinline__ void look(const uint32_t (&w)[N], bool f32, uint32_t& bad) {
  typedef unsigned short v2us __attribute__((ext_vector_type(2)));
  // the largest of the magnitudes (bf16: of both halves), as integers
  if (f32) {
#pragma unroll
    for (int i = 0; i < count; ++i) bad = max(bad, (w[i] & 0x7FFFFFFFu) >> 16);
  } else {
    constexpr int words = count > 1 ? count / 2 : 1;
#pragma unroll
    for (int i = 0; i < words; ++i) {
      const uint32_t v = count > 1 ? w[i] & 0x7FFF7FFFu : w[i] & 0x7FFFu;
      bad = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2us, bad), __builtin_bit_cast(v2us, v)));
    }
  }
}
__device__ __forceinline__ bool not_finite(uint32_t bad) { return (bad & 0xFFFFu) >= 0x7F80u || (bad >> 16) >= 0x7F80u; }

// MODE: parts of fp32 values in the products of o.  NKT: parts of the weighted
// keys in the state's.  DK: Dk padded to 64s.  STATE: the segment's own sum
// only (no queries, no o).
template <Kind KQ, Kind KK, Kind KV, bool OF32, int MODE, int NKT, int DK, int ET, int C, bool STATE>
__global__ __launch_bounds__(512) void linattn_chunk_kernel(const LinattnPass p) {
  constexpr int kX = DK / 64;        // 64s of Dk
  constexpr int kT = C / 16;         // tiles of tokens
  constexpr int kS = C / 32;         // contraction steps over tokens
  constexpr bool kFours = KQ == kF32 && KK == kF32;
  constexpr int kOwn = kT / 2;       // token tiles that a wave finishes
  constexpr int kPer = 8 / kT;       // waves per tile of keys
  constexpr bool kEarly = STATE || KV == kBf16;   // registers hold the next rows from the start of a chunk
  constexpr int NQ = KQ == kBf16 ? 1 : MODE, NK = KK == kBf16 ? 1 : MODE;
  constexpr int NV = KV == kBf16 ? 1 : STATE ? NKT : MODE;
  __shared__ v4i q_lds[STATE ? 1 : kT * kX * 2 * NQ][kWave];   // [token tile][64s][h][part]
  __shared__ v4i k_lds[STATE ? 2 : 1][kX * 4 * kS * NKT][kWave];   // [in turn][64s][i][token step][part]
  __shared__ v4i p_lds[STATE ? 1 : kT * kS * MODE][kWave];     // [token tile][token step][part]
  __shared__ v4f o_lds[STATE ? 1 : 8 * kOwn * ET][kWave];      // [receiving wave][own tile][f]
  __shared__ float pw[C + 1];                                  // l^i
  __shared__ int s_bad[2];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = wave >> 2, ew = wave & 3;
  const int n = lane & 15, g = lane >> 4;
  uint32_t blk = blockIdx.x;
  const uint32_t tile = blk % p.tiles;
  blk /= p.tiles;
  const uint32_t seg = blk % p.nseg;
  const uint32_t bh = blk / p.nseg;
  if (STATE && seg + 1 == p.nseg && !p.join_last) return;  // no segment follows
  const int64_t b = bh / p.H, h = bh % p.H;
  const int ebase = static_cast<int>(tile) * 64 * ET + ew * 16 * ET;
  const int e0 = ebase + ET * n;     // the lane's columns e0 .. e0 + ET - 1
  const bool ewave = ebase < p.Dv;
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
  if (threadIdx.x < 2) s_bad[threadIdx.x] = 0;

  const int64_t begin = static_cast<int64_t>(seg) * p.seg_tokens;
  const int64_t end = begin + p.seg_tokens < p.T ? begin + p.seg_tokens : p.T;
  int64_t single = begin;  // tokens before this one go one by one
  const auto tokens_at = [&](int64_t i) {
    const int64_t left = end - i;
    return i < single ? 1 : left < C ? static_cast<int>(left) : C;
  };

  // --- a chunk's rows: the wave's values; 4 tokens x 4 entries of the keys for
  // the state; queries and keys of a token tile
  constexpr int kKItems = kX * kS * 2;
  const bool has_k = wave < kKItems;
  const int kx = wave / (2 * kS), kc = wave / 2 % kS, kj = wave & 1;
  const int qi = kT * kX == 8 ? wave : kT * kX == 4 ? wave - 4 : wave >= 6 ? -1 : wave - 4;   // few: waves 4-7
  const bool has_q = qi >= 0;
  const int qt = qi / kX, qx = qi % kX;
  const int ps = wave % kT, pt = wave / kT;         // the wave's keys, and its first query tile behind them
  const bool has_p = ps + pt < kT;
  uint32_t wv[kS][8][kDwords<KV, ET>], wk[4][kDwords<KK, 4>], wq[kDwords<KQ, 16>], wn[kX][kDwords<KK, 16>];
  Rows<KQ> rq;
  Rows<KK> rk;
  Rows<KV> rv;
  const auto first_row = [&](int64_t i0, int tc) { return b * p.T + (p.rev ? p.T - i0 - tc : i0); };
  const auto load_most = [&](int64_t i0, int tc) {
    const int64_t row = first_row(i0, tc);
    rk.at(p.k, row, tc, h, p.Dk, p.rev);
    rv.at(p.v, row, tc, h, p.Dv, p.rev);
    const uint32_t vo = rv.lane(4 * g, e0);
#pragma unroll
    for (int c = 0; c < kS; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) rv.template load<ET>(vo, 32 * c + 16 * (j / 4) + j % 4, wv[c][j]);
    if (has_k) {
      const uint32_t ko = rk.lane(32 * kc + 16 * kj + 4 * g, 64 * kx + 4 * pi<kFours>(n));
#pragma unroll
      for (int r = 0; r < 4; ++r) rk.template load<4>(ko, r, wk[r]);
    }
    if constexpr (!STATE) {
      if (has_q) {
        rq.at(p.q, row, tc, h, p.Dk, p.rev);
        load_entries<kFours>(rq, 16 * qt + n, 64 * qx, g, wq);
      }
    }
  };
  const auto load_keys = [&](int64_t i0, int tc) {
    if constexpr (!STATE) {
      if (has_p) {
        rk.at(p.k, first_row(i0, tc), tc, h, p.Dk, p.rev);
#pragma unroll
        for (int x = 0; x < kX; ++x) load_entries<kFours>(rk, 16 * ps + n, 64 * x, g, wn[x]);
      }
    }
  };
  load_most(begin, tokens_at(begin));
  load_keys(begin, tokens_at(begin));

  // the state, [64s][i - 2 half][f]
  v4f st[kX][2][ET];
  const float first = p.rev || p.joined != nullptr ? 1.0f : p.decay[h];
#pragma unroll
  for (int x = 0; x < kX; ++x)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int f = 0; f < ET; ++f) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v = 0.0f;
          const int d = 64 * x + 4 * pi<kFours>(4 * g + r) + 2 * half + i, e = e0 + f;
          if (!STATE && eon && d < p.Dk) {
            if (p.joined != nullptr) {
              v = p.joined[((static_cast<int64_t>(bh) * p.nseg + seg) * p.Dk + d) * p.Dv + e];
            } else if (p.s_in != nullptr) {
              v = p.s_in[static_cast<int64_t>(bh) * p.Dk * p.Dv + static_cast<int64_t>(d) * p.in_d + static_cast<int64_t>(e) * p.in_e];
              v *= first;
            }
          }
          st[x][i][f][r] = v;
        }
      }
  lds_barrier();

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

  // --- a chunk's rows, as loaded, into operands: values in registers, keys and
  // queries in LDS
  v4i vf[kS][ET][NV];
  const auto stage = [&](int64_t i0, int tc, int flag) {
    const bool last = i0 + tc == p.T && !p.rev;  // the state behind the last token itself
    // values of the wave's columns, and whether they are all finite
    uint32_t bad = 0;
#pragma unroll
    for (int c = 0; c < kS; ++c) {
#pragma unroll
      for (int f = 0; f < ET; ++f) operand<KV>([&](int j) { return element(wv[c][j], rv.f32(), f); }, vf[c][f]);
      if constexpr (!STATE) {
#pragma unroll
        for (int j = 0; j < 8; ++j) look<ET>(wv[c][j], rv.f32(), bad);
      }
    }
    if (!STATE && __any(not_finite(bad)) && lane == 0) s_bad[flag] = 1;
    // weighted transposed keys: decays to the next chunk's first token, or to
    // the last one
    if (has_k) {
      float wt[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int to = tc - (32 * kc + 16 * kj + 4 * g + r) - (last ? 1 : 0);
        wt[r] = alpha * pw[to > 0 ? to : 0];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = element(wk[r], rk.f32(), i).value() * wt[r];
#pragma unroll
        for (int k = 0; k < NKT; ++k) {
          const uint2 u = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
          reinterpret_cast<uint2*>(&k_lds[STATE ? flag : 0][((kx * 4 + i) * kS + kc) * NKT + k][lane])[kj] = u;
          y[0] -= bf16_lo(u.x);
          y[1] -= bf16_hi(u.x);
          y[2] -= bf16_lo(u.y);
          y[3] -= bf16_hi(u.y);
        }
      }
    }
    if constexpr (!STATE) {
      if (has_q) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          v4i f[NQ];
          operand<KQ>([&](int j) { return element(wq, rq.f32(), 4 * (j % 4) + 2 * hh + j / 4); }, f);
#pragma unroll
          for (int k = 0; k < NQ; ++k) q_lds[((qt * kX + qx) * 2 + hh) * NQ + k][lane] = f[k];
        }
      }
    }
  };
  // the rows of the chunk at i0, where there is one
  const auto load = [&](int64_t i0) {
    if (i0 < end) load_most(i0, tokens_at(i0));
  };

  // Two barriers per chunk: the products of staged operands lie between them
  // (keys x queries, queries x state, the state's update), what follows from
  // other waves' products (products x values) and the next chunk's staging
  // behind them.  Whether a chunk's values are finite is told in two flags in
  // turn: one is cleared while the other is read.
  int64_t i0 = begin;
  int tc = tokens_at(i0), flag = 0;
  stage(i0, tc, flag);
  for (;;) {
    const int64_t next = i0 + tc;
    if (kEarly) load(next);
    lds_barrier();
    const bool last = next == p.T && !p.rev;

    v4f o[kOwn][ET];
    if constexpr (!STATE) {
      const bool redo = tc > 1 && __builtin_amdgcn_readfirstlane(s_bad[flag]) != 0;
      if (threadIdx.x == 0) s_bad[flag ^ 1] = 0;
      if (redo) {  // a value that is not finite reaches no token before it
        single = next;
        lds_barrier();
        tc = 1;
        flag ^= 1;
        load_most(i0, 1);
        load_keys(i0, 1);
        stage(i0, 1, flag);
        continue;
      }
      const auto query = [&](int t, int x, int hh, v4i (&f)[NQ]) {
#pragma unroll
        for (int k = 0; k < NQ; ++k) f[k] = q_lds[((t * kX + x) * 2 + hh) * NQ + k][lane];
      };
      // --- keys x queries, decayed
      constexpr int kU = (kT + kPer - 1) / kPer;
      if (has_p) {
        v4f acc[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) acc[u] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int x = 0; x < kX; ++x)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            v4i kf[NK];
            operand<KK>([&](int j) { return element(wn[x], rk.f32(), 4 * (j % 4) + 2 * hh + j / 4); }, kf);
#pragma unroll
            for (int u = 0; u < kU; ++u) {
              const int t = ps + pt + u * kPer;
              if (t >= kT) continue;
              v4i f[NQ];
              query(t, x, hh, f);
              acc[u] = mma<MODE>(kf, f, acc[u]);
            }
          }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int t = ps + pt + u * kPer;
          if (t >= kT) continue;
          float y[4];
          if (t == ps) {
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = n >= 4 * g + r ? acc[u][r] * w_diag[r] : 0.0f;
          } else {
            const float wx = pw[16 * (t - ps - 1)];
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = acc[u][r] * (w_off[r] * wx);
          }
#pragma unroll
          for (int k = 0; k < MODE; ++k) {
            const uint2 v = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
            reinterpret_cast<uint2*>(&p_lds[(t * kS + ps / 2) * MODE + k][lane])[ps & 1] = v;
            y[0] -= bf16_lo(v.x);
            y[1] -= bf16_hi(v.x);
            y[2] -= bf16_lo(v.y);
            y[3] -= bf16_hi(v.y);
          }
        }
      }
      if ((ps & 1) && pt == 1) {  // the half of an operand that no tile fills
#pragma unroll
        for (int k = 0; k < MODE; ++k)
          reinterpret_cast<uint2*>(&p_lds[((ps - 1) * kS + ps / 2) * MODE + k][lane])[1] = make_uint2(0u, 0u);
      }
      if (kEarly && next < end) load_keys(next, tokens_at(next));

      // --- queries x the wave's half of the state; what other waves finish
      if (ewave) {
        v4f a[kT][ET];
#pragma unroll
        for (int t = 0; t < kT; ++t)
#pragma unroll
          for (int f = 0; f < ET; ++f) a[t][f] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int x = 0; x < kX; ++x) {
          v4i sf[ET][MODE];
#pragma unroll
          for (int f = 0; f < ET; ++f) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = st[x][j / 4][f][j % 4];
            split8<MODE>(y, sf[f]);
          }
#pragma unroll
          for (int t = 0; t < kT; ++t) {
            v4i q[NQ];
            query(t, x, half, q);
#pragma unroll
            for (int f = 0; f < ET; ++f) a[t][f] = mma<MODE>(q, sf[f], a[t][f]);
          }
        }
        // tiles 0 and 3 (of 4) or 0 (of 2) are finished by waves 0-3
#pragma unroll
        for (int u = 0; u < kOwn; ++u)
#pragma unroll
          for (int f = 0; f < ET; ++f) {
            const int t0 = kT == 4 ? 3 * u : u, t1 = kT == 4 ? 1 + u : 1;
            o[u][f] = half ? a[t1][f] : a[t0][f];
            o_lds[((wave ^ 4) * kOwn + u) * ET + f][lane] = half ? a[t0][f] : a[t1][f];
          }
      }
      // the next chunk's rows, in the registers that the sums over all tiles had
      if (!kEarly) load(next);
    }

    // --- keys x values into the state
    if (ewave) {
      const float w = pw[last ? tc - 1 : tc];
#pragma unroll
      for (int x = 0; x < kX; ++x)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int f = 0; f < ET; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r) st[x][i][f][r] *= w;
#pragma unroll
          for (int c = 0; c < kS; ++c) {
            v4i k[NKT];
#pragma unroll
            for (int y = 0; y < NKT; ++y) k[y] = k_lds[STATE ? flag : 0][((x * 4 + 2 * half + i) * kS + c) * NKT + y][lane];
#pragma unroll
            for (int f = 0; f < ET; ++f) st[x][i][f] = mma<NKT>(k, vf[c][f], st[x][i][f]);
          }
        }
    }

    if constexpr (!STATE) {
      if (!kEarly && next < end) load_keys(next, tokens_at(next));
      lds_barrier();
      if (ewave) {
#pragma unroll
        for (int u = 0; u < kOwn; ++u) {
          const int t = kT == 4 ? (half ? 1 + u : 3 * u) : half;
          const float wx = pw[16 * t];
#pragma unroll
          for (int f = 0; f < ET; ++f) {
            const v4f more = o_lds[(wave * kOwn + u) * ET + f][lane];
#pragma unroll
            for (int r = 0; r < 4; ++r) o[u][f][r] = (o[u][f][r] + more[r]) * (w_row[r] * wx);
          }
          // --- products x values
#pragma unroll
          for (int c = 0; c < kS; ++c) {
            if (2 * c > t) continue;
            v4i f[MODE];
#pragma unroll
            for (int k = 0; k < MODE; ++k) f[k] = p_lds[(t * kS + c) * MODE + k][lane];
#pragma unroll
            for (int e = 0; e < ET; ++e) o[u][e] = mma<MODE>(f, vf[c][e], o[u][e]);
          }
        }
        // --- store
        const int size = OF32 ? 4 : 2, ld = static_cast<int>(p.ldo) * size;
        const auto ro = __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(p.o) + (first_row(i0, tc) * p.ldo + h * p.Dv) * size,
                                                          0, (tc - 1) * ld + p.Dv * size, kBufferWord3);
        const int step = p.rev ? -ld : ld;
        uint32_t at = eon ? static_cast<uint32_t>((p.rev ? (tc - 1) * ld : 0) + 4 * g * step + e0 * size) : kOff;
        asm volatile("" : "+v"(at));
#pragma unroll
        for (int u = 0; u < kOwn; ++u) {
          const int t = kT == 4 ? (half ? 1 + u : 3 * u) : half;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t off = at + static_cast<uint32_t>((16 * t + r) * step);
            if constexpr (OF32) {
              if constexpr (ET == 2)
                __builtin_amdgcn_raw_buffer_store_b64(v2u{__float_as_uint(o[u][0][r]), __float_as_uint(o[u][1][r])}, ro, off, 0, 0);
              else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(o[u][0][r]), ro, off, 0, 0);
            } else {
              if constexpr (ET == 2) __builtin_amdgcn_raw_buffer_store_b32(pack_bf16(o[u][0][r], o[u][1][r]), ro, off, 0, 0);
              else __builtin_amdgcn_raw_buffer_store_b16(static_cast<uint16_t>(pack_bf16(o[u][0][r], 0.0f)), ro, off, 0, 0);
            }
          }
        }
      }
    }
    if (next >= end) break;
    i0 = next;
    tc = tokens_at(i0);
    flag ^= 1;
    stage(i0, tc, flag);
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
    for (int x = 0; x < kX; ++x)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int f = 0; f < ET; ++f)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int d = 64 * x + 4 * pi<kFours>(4 * g + r) + 2 * half + i;
            if (d < p.Dk) out[d * od + (e0 + f) * oe] = st[x][i][f][r];
          }
  }
}

constexpr int chunk_tokens(int DK, Kind K, bool STATE) { return DK == 256 || (K != kBf16 && !STATE) ? 32 : 64; }

template <Kind KQ, Kind KK, Kind KV, bool OF32, int MODE, int NKT, bool STATE>
hipError_t launch_pass(const LinattnPass& p, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(p.B * p.H * p.nseg * p.tiles));
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(512), 0, stream, p);
    return hipGetLastError();
  };
#define MMF_DIMS(DK)                                                                                          \
  return p.et == 1 ? go(linattn_chunk_kernel<KQ, KK, KV, OF32, MODE, NKT, DK, 1, chunk_tokens(DK, KQ, STATE), STATE>)    \
                   : go(linattn_chunk_kernel<KQ, KK, KV, OF32, MODE, NKT, DK, 2, chunk_tokens(DK, KQ, STATE), STATE>)
  if (p.Dk <= 64) MMF_DIMS(64);
  if (p.Dk <= 128) MMF_DIMS(128);
#undef MMF_DIMS
  return go(linattn_chunk_kernel<KQ, KK, KV, OF32, MODE, NKT, 256, 1, chunk_tokens(256, KQ, STATE), STATE>);
}

}  // namespace la
}  // namespace mmf
