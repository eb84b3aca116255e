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
// A workgroup holds a state of Dk rows and 128 (64) columns in the accumulators of
// its matrix instructions, 16 or 32 columns per wave.  A chunk's rows are read
// once, 16 bytes of bf16 per lane and row, a chunk ahead of their use, and go to
// LDS as they are (fp32: as bf16 parts); every operand of the products comes from
// there, along the rows or, by the transposing read, across them.
// With v_mfma_f32_16x16x32_bf16 (lane = 16 g + n, g = 0..3, n = 0..15; A: row n,
// B: column n, eight contraction slots 8 g + j; D: column n, rows 4 g + r):
//   keys x queries  A: keys as rows, B: queries; D: keys 4 g + r of query n, which
//                   LDS takes as rows of queries, 8 bytes per lane
//   state x queries A: the state's columns as rows, B: queries
//   values x products  A: the values' columns as rows (across), B: the products'
//                   rows; D: columns 4 g + r of query n, side by side in memory
//   keys x values   A: the keys' entries as rows (across), B: the decayed
//                   values' columns (across); D: the state
// The state's tile (b, h) has row m = entry d = 32 b + 8 (m / 4) + 4 h + m % 4, so
// that the rows a lane keeps of the two tiles h are the slots d = 32 b + 8 g + j
// of the operand it is for the next chunk: the state never leaves its registers.
// The keys x queries are formed once per workgroup: each wave forming its own in
// registers (keys in the same order) saves a barrier, but took a tenth longer
// (16384 bf16 tokens, 16 heads of 128; a sixth for the three passes of 4 x 2048
// fp32).  Two buffers for bf16 chunks in LDS, and one barrier instead of two,
// gained nothing.
//
// What bounds it is a chunk's chain of loads, splitting, LDS, products and two barriers:
// 2.7 us of bf16, 5.3 of fp32, whose parts take six products for one, where a compute
// unit has one workgroup.  Over many tokens two of them hide a part of each other:
// that forward moves 303 MB in 95 us, 3.2 TB/s, the vector unit two thirds and the
// matrix cores one third busy, after 163 MB in 43 us for the segments' sums.
//
// Numerics: bf16 inputs are exact operands.  fp32 values (fp32 inputs, the
// decayed products, the state, the decayed values) go to the matrix cores as
// sums of three bf16 parts (2^-24 relative), with the products of parts down to
// the same size: six for one.  Also where the result is rounded to bf16, since
// what is left of terms that cancel would else be that of 17 bits (two parts and
// three products: 16384 bf16 130 us where this takes 142, the backward of 4 x 2048
// fp32 219 and 283, of bf16 150 and 172).  Sums are fp32; powers of l come from fp64.
#pragma once
#include "linattn.h"
#include "mmf_device.h"
#include "row_vec.h"

namespace mmf {
namespace la {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
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
// And back.
template <int N>
__device__ __forceinline__ void sum8(const v4i (&p)[N], float* x) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    float a = bf16_lo(p[N - 1][w]), b = bf16_hi(p[N - 1][w]);
#pragma unroll
    for (int i = N - 2; i >= 0; --i) {
      a += bf16_lo(p[i][w]);
      b += bf16_hi(p[i][w]);
    }
    x[2 * w] = a;
    x[2 * w + 1] = b;
  }
}

constexpr int kParts = 3;   // of an fp32 value

// acc += a b over the parts' products of relative size above 2^-24.
template <int NA, int NB>
__device__ __forceinline__ v4f mma(const v4i (&a)[NA], const v4i (&b)[NB], v4f acc) {
#pragma unroll
  for (int i = NA - 1; i >= 0; --i)
#pragma unroll
    for (int j = NB - 1; j >= 0; --j)
      if (i + j < kParts) acc = mfma(a[i], b[j], acc);
  return acc;
}

// Tiles in LDS: rows of W bf16 values in chunks of 16 bytes, chunk q of a row at
// q ^ swizzle(row).  A cycle serves 16 lanes of a 16-byte read, 32 of a transposing
// one, and touches 64 banks: of the lanes 16 g + n along the rows n = 0 .. 3 and 12
// .. 15 of one g with n = 4 .. 11 of the next, whose chunk is the neighbour (or the
// other way round), so the swizzle takes rows 4 apart to 0, 2, 3, 1; across, 8 rows
// at 2 chunks of 16 bytes, or of the keys at half of 4, which takes two cycles.
// Rows 16 apart have the same swizzle, and chunks 4 b apart differ in address bits
// that no other part of the sum reaches: ^ (b << 6).
template <int W>
__device__ __forceinline__ int tile_at(int row, int chunk) {
  const int q = (row >> 3) & 1, low = 2 * (((row >> 2) & 1) ^ q) + q;
  const int f = W == 32 ? low : W == 64 ? 4 * ((row >> 1) & 1) + low : 4 * (row & 3) + low;
  return row * (2 * W) + ((chunk ^ f) << 4);
}
__device__ __forceinline__ v4i tile_read(const char* tile, int at) { return *reinterpret_cast<const v4i*>(tile + at); }
// Across: 4 rows (from lanes 4 k .. 4 k + 3 of 16, each 4 of 16 columns) to 16
// lanes, a column each.
__device__ __forceinline__ v2u tile_turn(const char* tile, int at) {
  typedef __attribute__((address_space(3))) v4s lds_v4s;
  return __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(tile + at)));
}
__device__ __forceinline__ v4i tile_turn8(const char* tile, int at0, int at1) {
  const v2u a = tile_turn(tile, at0), b = tile_turn(tile, at1);
  return v4i{static_cast<int>(a.x), static_cast<int>(a.y), static_cast<int>(b.x), static_cast<int>(b.y)};
}

// How an operand's elements are stored: bf16, fp32, or as the pass says.
enum Kind { kBf16, kF32, kEither };
template <Kind K>
constexpr int kUnitDwords = K == kBf16 ? 4 : 8;   // of 8 elements in registers

template <Kind K>
struct KindOf {
  static constexpr Kind value = K;
};

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
  char* seq;        // the head's entries of the sequence's first row
  // Head h, whose entries are `w`, of the rows from `row` on.  Kept in registers:
  // fetched again for each chunk, the arguments would be waited for each time.
  __device__ __forceinline__ void init(const LinattnOperand& x, int64_t row, int64_t h, int w, bool rev) {
    f32_ = x.is_f32;
    const int size = f32() ? 4 : 2;
    width = w;
    step = static_cast<int>(x.ld) * (rev ? -size : size);
    seq = const_cast<char*>(static_cast<const char*>(x.p)) + (row * x.ld + h * w) * size;
    uint64_t s = reinterpret_cast<uint64_t>(seq);
    asm volatile("" : "+s"(s), "+s"(step), "+s"(width));
    seq = reinterpret_cast<char*>(s);
  }
  // `tc` of them from row `row`.
  __device__ __forceinline__ void at(int64_t row, int tc) {
    const int ld = step < 0 ? -step : step;
    base = step < 0 ? static_cast<uint32_t>((tc - 1) * ld) : 0u;
    r = __builtin_amdgcn_make_buffer_rsrc(seq + row * ld, 0, (tc - 1) * ld + width * (f32() ? 4 : 2), kBufferWord3);
  }
  // Units of 8 elements: those of `threads` threads from token i, column d on,
  // U of them `apart` tokens from each other.
  template <int U>
  __device__ __forceinline__ void load(int i, int d, int apart, uint32_t (&w)[U][kUnitDwords<K>]) const {
    const uint32_t size = f32() ? 4u : 2u;
    const uint32_t o = d < width ? base + static_cast<uint32_t>(i * step) + static_cast<uint32_t>(d) * size : kOff;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t off = o + static_cast<uint32_t>(u * apart * step);
      const Words<4> a = load_stream<4, false>(r, off);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[u][j] = a.w[j];
      if constexpr (K != kBf16) {
        // (of bf16 rows these are not used)
        const Words<4> b = load_stream<4, false>(r, off + 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[u][4 + j] = b.w[j];
      }
    }
  }
};
// A unit's values in fp32.
template <Kind K>
__device__ __forceinline__ void unit_values(const uint32_t (&w)[kUnitDwords<K>], bool f32, float* x) {
  if constexpr (K == kBf16) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j & 1 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float whole = __uint_as_float(w[j]);
      x[j] = whole;
      if constexpr (K == kEither) {
        const uint32_t pair = w[j / 2];
        const float part = j & 1 ? bf16_hi(pair) : bf16_lo(pair);
        x[j] = f32 ? whole : part;
      }
    }
  }
}
// The largest magnitude's upper 16 bits so far, in both halves of `top`.
__device__ __forceinline__ void look_bf16(uint32_t w, uint32_t& top) {
  typedef unsigned short v2us __attribute__((ext_vector_type(2)));
  top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2us, top), __builtin_bit_cast(v2us, w & 0x7FFF7FFFu)));
}
// Of fp32 the largest magnitude's bits: not finite is what its first part is not.
template <Kind K>
__device__ __forceinline__ bool not_finite(uint32_t top) {
  return K == kBf16 ? (top & 0xFFFFu) >= 0x7F80u || (top >> 16) >= 0x7F80u : top >= 0x7F7F8000u;
}

// DK: Dk padded to 64, 128, 256.  WAVES: of CT x 16 columns each.  STATE: the segment's
// own sum only (no queries, no o; the values go to LDS decayed).  Waves per SIMD: what
// leaves each form its registers, so that none spills (bf16, 4 x 2048, 16 heads of 96 x
// 64, backward: 129.9 us; 132.0 where the 4-wave passes had four and the sums six, with
// 8 bytes of scratch each).  For passes a compute unit so holds two workgroups of 8
// waves; of 4 waves four of bf16 (three from 80 key entries on) and two of fp32; of more
// than 128 key entries one of 8 waves, and of fp32, by its LDS, one of any.
template <Kind KQ, Kind KK, Kind KV, bool OF32, int DK, int WAVES, int CT, bool STATE>
__global__ __launch_bounds__(64 * WAVES, STATE && DK <= 128 ? (KK == kBf16 && WAVES == 8 ? 6 : 5) : DK == 256 || CT == 2 ? 2 : DK == 128 && WAVES == 4 ? 3 : 4) void linattn_chunk_kernel(
    const LinattnPasses args) {
  constexpr int C = kLinattnChunk, kThreads = 64 * WAVES, WC = 16 * CT * WAVES;
  constexpr int kB = DK / 32;        // contraction steps over Dk
  constexpr int kT = C / 16;         // tiles of tokens
  constexpr int kS = C / 32;         // contraction steps over tokens
  static_assert(STATE || (kT == 2 && WAVES >= 4), "the products' tiles are a wave's each");
  constexpr int NQ = KQ == kBf16 ? 1 : kParts, NK = KK == kBf16 ? 1 : kParts;
  constexpr int NV = KV == kBf16 && !STATE ? 1 : kParts;
  // A chunk's rows are asked for before the products of the chunk before; of fp32
  // the queries behind them, which leaves the products their registers.
  constexpr bool kEarly = STATE || KQ == kBf16;
  // units of 8 elements per thread (half the threads have one where a chunk has fewer)
  constexpr bool kHalf = C * DK / 8 < kThreads;
  constexpr int kKUnits = kHalf ? 1 : C * DK / 8 / kThreads, kVUnits = C * WC / 8 / kThreads;
  static_assert(kVUnits >= 1 && kThreads % (DK / 8) == 0 && kThreads % (WC / 8) == 0, "whole rows");
  __shared__ __attribute__((aligned(16))) char q_t[STATE ? 1 : NQ][STATE ? 16 : C * DK * 2];
  __shared__ __attribute__((aligned(16))) char k_t[NK][C * DK * 2];
  __shared__ __attribute__((aligned(16))) char v_t[NV][C * WC * 2];
  __shared__ __attribute__((aligned(16))) char p_t[STATE ? 1 : kParts][STATE ? 16 : C * C * 2];
  __shared__ float pr[2 * C + 2];    // l^(C - i); 1 behind i = C
  __shared__ int s_bad[2];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  // 8 workgroups of one pass, then the same 8 of the next: a segment's passes run
  // on one XCD at about the same time and find each other's rows in its L2.
  const uint32_t whole = args.count / 8 * 8;
  const uint32_t unit = blockIdx.x / 8, rest = blockIdx.x - whole * args.n;
  const bool in_whole = blockIdx.x < whole * args.n;
  const uint32_t which = in_whole ? unit % args.n : rest / (args.count - whole);
  const LinattnPass& p = args.p[which];
  uint32_t blk = in_whole ? unit / args.n * 8 + blockIdx.x % 8 : whole + rest % (args.count - whole);
  const uint32_t tile = blk % p.tiles;
  blk /= p.tiles;
  const uint32_t seg = blk % p.nseg;
  const uint32_t bh = blk / p.nseg;
  if (STATE && seg >= p.segs) return;
  const int64_t b = bh / p.H, h = bh % p.H;
  const int c0 = static_cast<int>(tile) * WC, w0 = c0 + 16 * CT * wave;  // first column of the workgroup, of the wave
  const bool ewave = w0 < p.Dv;      // widths are multiples of 16

  const int64_t begin = static_cast<int64_t>(seg) * p.seg_tokens;
  const int64_t end = begin + p.seg_tokens < p.T ? begin + p.seg_tokens : p.T;
  int64_t single = begin;  // tokens before this one go one by one
  const auto tokens_at = [&](int64_t i) {
    const int64_t left = end - i;
    return i < single ? 1 : left < C ? static_cast<int>(left) : C;
  };
  const bool rev = p.rev;
  int64_t T = p.T;
  asm volatile("" : "+s"(T));
  const auto first_row = [&](int64_t i0, int tc) { return rev ? T - i0 - tc : i0; };   // in the sequence

  // --- a chunk's rows into registers
  const int kr = threadIdx.x / (DK / 8), kq = threadIdx.x % (DK / 8);   // row and chunk of the thread's first unit
  const int vr = threadIdx.x / (WC / 8), vq = threadIdx.x % (WC / 8);
  constexpr int kKApart = kThreads / (DK / 8), kVApart = kThreads / (WC / 8);
  const bool k_on = !kHalf || threadIdx.x < C * DK / 8;
  uint32_t wq[STATE ? 1 : kKUnits][kUnitDwords<KQ>], wk[kKUnits][kUnitDwords<KK>], wv[kVUnits][kUnitDwords<KV>];
  Rows<KQ> rq;
  Rows<KK> rk;
  Rows<KV> rv;
  Rows<OF32 ? kF32 : kBf16> ro;      // of the output
  rk.init(p.k, b * T, h, p.Dk, rev);
  rv.init(p.v, b * T, h, p.Dv, rev);
  if constexpr (!STATE) {
    rq.init(p.q, b * T, h, p.Dk, rev);
    ro.init({p.o, p.ldo, OF32}, b * T, h, p.Dv, rev);
  }
  const auto load = [&](int64_t i0, int tc) {
    const int64_t row = first_row(i0, tc);
    rk.at(row, tc);
    rk.load(kr, k_on ? 8 * kq : rk.width, kKApart, wk);
    rv.at(row, tc);
    rv.load(vr, c0 + 8 * vq, kVApart, wv);
  };
  const auto load_queries = [&](int64_t i0, int tc) {
    if constexpr (!STATE) {
      rq.at(first_row(i0, tc), tc);
      rq.load(kr, k_on ? 8 * kq : rq.width, kKApart, wq);
    }
  };
  load(begin, tokens_at(begin));
  load_queries(begin, tokens_at(begin));

  // powers of l: fp64, by squaring (any l, 0 among them)
  for (int i = threadIdx.x; i < 2 * C + 2; i += kThreads) {
    double x = p.decay[h], y = 1.0;
    for (int e = i < C ? C - i : 0; e != 0; e >>= 1) {
      if (e & 1) y *= x;
      x *= x;
    }
    pr[i] = static_cast<float>(y);
  }
  if (threadIdx.x < 2) s_bad[threadIdx.x] = 0;

  // --- the state: st[b][h] rows 8 g + 4 h + r of 32 b, column w0 + n
  v4f st[CT][kB][2];
  const bool given = !STATE && p.e_in != nullptr;
  const auto re = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<float*>(given ? p.e_in + bh * p.e_bh + seg * p.e_seg : nullptr), 0, given ? p.Dk * p.Dv * 4 : 0, kBufferWord3);
  // every tile of the state, as f(tile of columns, x, i)
  const auto each = [&](auto&& f) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int x = 0; x < kB; ++x)
#pragma unroll
        for (int i = 0; i < 2; ++i) f(ct, x, i);
  };
  each([&](int ct, int x, int i) {
    v4f& e = st[ct][x][i];
    if constexpr (STATE) {
      e = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    } else {
      const int d = 32 * x + 8 * g + 4 * i, col = w0 + 16 * ct + n;
      const uint32_t at = col < p.Dv && d < p.Dk ? 4u * static_cast<uint32_t>(d * p.e_d + col * p.e_e) : kOff;
      if (p.e_d == 1) {
        const Words<4> w = load_stream<4, false>(re, at);
#pragma unroll
        for (int r = 0; r < 4; ++r) e[r] = __uint_as_float(w.w[r]);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) e[r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(re, at + 4u * r * p.e_d, 0, 0));
      }
    }
  });
  if (!STATE && p.e_decay) {
    const float l = p.decay[h];
    each([&](int ct, int x, int i) { st[ct][x][i] *= l; });
  }
  lds_barrier();

  float alpha = p.alpha, beta = p.beta;
  asm volatile("" : "+s"(alpha), "+s"(beta));
  // lane's places in the tiles (those with other steps over Dk are taken from
  // them anew for each chunk, not kept in registers)
  const int k_row = tile_at<DK>(n, g);                                        // along: row n, slots 8 g + j
  const int p_row = tile_at<C>(n, g);
  const int t_row = 8 * g + (n >> 2);                                         // across: rows 8 g .. + 3, + 4 .. + 7
  const int k_a0 = tile_at<DK>(t_row, n & 3), k_a1 = tile_at<DK>(t_row + 4, n & 3);
  const int v_a0 = tile_at<WC>(t_row, 2 * CT * wave + ((n & 3) >> 1)) + 8 * (n & 1);  // (the next 16 columns: ^ 32)
  const int v_a1 = tile_at<WC>(t_row + 4, 2 * CT * wave + ((n & 3) >> 1)) + 8 * (n & 1);
  const int ps = wave % kT, pt = ps + wave / kT;   // the wave's tile of keys x queries, if there is one

  // --- a chunk's rows from registers to LDS; whether its values are finite
  const auto stage = [&](int64_t i0, int tc, int flag) {
    const int last = i0 + tc == T && !rev ? 1 : 0;  // the state behind the last token itself
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < kVUnits; ++u) {
      const int at = tile_at<WC>(vr, vq) + u * kVApart * (2 * WC);
      static_assert(kVApart % 16 == 0, "the same swizzle");
      if constexpr (KV == kBf16 && !STATE) {
        const v4i w = {static_cast<int>(wv[u][0]), static_cast<int>(wv[u][1]), static_cast<int>(wv[u][2]), static_cast<int>(wv[u][3])};
        *reinterpret_cast<v4i*>(&v_t[0][at]) = w;
#pragma unroll
        for (int j = 0; j < 4; ++j) look_bf16(wv[u][j], top);
      } else {
        float x[8];
        unit_values<KV>(wv[u], rv.f32(), x);
        v4i f[NV];
        if constexpr (STATE) {
          const float w = alpha * pr[vr + u * kVApart + C - tc + last];
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] *= w;
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
        }
        split8<NV>(x, f);
#pragma unroll
        for (int k = 0; k < NV; ++k) *reinterpret_cast<v4i*>(&v_t[k][at]) = f[k];
      }
    }
    if (!STATE && __any(not_finite<KV>(top)) && lane == 0) s_bad[flag] = 1;
    const auto put = [&](auto kind, const auto& w, bool f32, auto& t) {
      constexpr Kind K = decltype(kind)::value;
      constexpr int N = sizeof(t) / sizeof(t[0]);
#pragma unroll
      for (int u = 0; u < kKUnits; ++u) {
        const int at = tile_at<DK>(kr + u * kKApart, kq);
        v4i f[N];
        if constexpr (K == kBf16) {
          f[0] = v4i{static_cast<int>(w[u][0]), static_cast<int>(w[u][1]), static_cast<int>(w[u][2]), static_cast<int>(w[u][3])};
        } else {
          float x[8];
          unit_values<K>(w[u], f32, x);
          split8<N>(x, f);
        }
#pragma unroll
        for (int k = 0; k < N; ++k)
          if (k_on) *reinterpret_cast<v4i*>(&t[k][at]) = f[k];
      }
    };
    put(KindOf<KK>{}, wk, rk.f32(), k_t);
    if constexpr (!STATE) put(KindOf<KQ>{}, wq, rq.f32(), q_t);
  };

  // Two barriers per chunk: the products of staged operands lie between them
  // (keys x queries, state x queries, the state's update), what needs other
  // waves' products (values x products) and the next chunk's staging behind
  // them.  Whether a chunk's values are finite is told in two flags in turn:
  // one is cleared while the other is read.
  int64_t i0 = begin;
  int tc = tokens_at(i0), flag = 0;
  stage(i0, tc, flag);
  // The state is there before the loop: a wait for it inside would be one for the
  // next chunk's loads, in every chunk.
  if constexpr (!STATE) each([&](int ct, int x, int i) { asm volatile("" : "+v"(st[ct][x][i])); });
  while (true) {
    const int64_t next = i0 + tc;
    if (next < end) {
      load(next, tokens_at(next));
      if (kEarly) load_queries(next, tokens_at(next));
    }
    lds_barrier();
    const bool last = next == T && !rev;

    int k_row_ = k_row, k_a0_ = k_a0, k_a1_ = k_a1;
    asm volatile("" : "+v"(k_row_), "+v"(k_a0_), "+v"(k_a1_));
    v4f o[STATE ? 1 : CT][kT];
    v4i vf[CT][kS][NV];
    if constexpr (!STATE) {
      const bool redo = tc > 1 && __builtin_amdgcn_readfirstlane(s_bad[flag]) != 0;
      if (threadIdx.x == 0) s_bad[flag ^ 1] = 0;
      if (redo) {  // a value that is not finite reaches no token before it
        single = next;
        lds_barrier();
        tc = 1;
        flag ^= 1;
        load(i0, 1);
        load_queries(i0, 1);
        stage(i0, 1, flag);
        continue;
      }
      const auto query = [&](int t, int x, v4i (&f)[NQ]) {
#pragma unroll
        for (int k = 0; k < NQ; ++k) f[k] = tile_read(q_t[k], (k_row_ ^ (x << 6)) + t * 16 * (2 * DK));
      };
      // --- keys x queries, decayed
      if (pt < kT) {
        v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int x = 0; x < kB; ++x) {
          v4i kf[NK], f[NQ];
#pragma unroll
          for (int k = 0; k < NK; ++k) kf[k] = tile_read(k_t[k], (k_row_ ^ (x << 6)) + ps * 16 * (2 * DK));
          query(pt, x, f);
          acc = mma(kf, f, acc);
        }
        // decay from key 16 ps + 4 g + r to query 16 pt + n; none from later keys
        const float* const w = &pr[C - 16 * (pt - ps) - n + 4 * g];
        float y[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          y[r] = acc[r] * (alpha * beta * w[r]);
          if (pt == ps && n < 4 * g + r) y[r] = 0.0f;
        }
        const int at = tile_at<C>(n, 2 * ps + (g >> 1)) + pt * 16 * (2 * C) + 8 * (g & 1);
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
          const uint2 v = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
          *reinterpret_cast<uint2*>(&p_t[k][at]) = v;
          y[0] -= bf16_lo(v.x);
          y[1] -= bf16_hi(v.x);
          y[2] -= bf16_lo(v.y);
          y[3] -= bf16_hi(v.y);
        }
      }
      if (ps == 1 && pt == kT) {  // the half of an operand that no tile fills
        const int at = tile_at<C>(n, 2 + (g >> 1)) + 8 * (g & 1);
#pragma unroll
        for (int k = 0; k < kParts; ++k) *reinterpret_cast<uint2*>(&p_t[k][at]) = make_uint2(0u, 0u);
      }
      // --- state x queries
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int t = 0; t < kT; ++t) o[ct][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
      if (ewave) {
#pragma unroll
        for (int x = 0; x < kB; ++x) {
          v4i sf[CT][kParts];
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = st[ct][x][j / 4][j % 4];
            split8<kParts>(y, sf[ct]);
          }
#pragma unroll
          for (int t = 0; t < kT; ++t) {
            v4i f[NQ];
            query(t, x, f);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) o[ct][t] = mma(sf[ct], f, o[ct][t]);
          }
        }
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          const float w = beta * pr[C - 16 * t - n];
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) o[ct][t] *= w;
        }
      }
    }
    // The state's decay over the chunk, taken by the registers: kept beside them as a
    // factor, values would enter divided by it, and large ones overflow (no less time
    // either: 16384 bf16 145 us both ways, the backward of 4 x 2048 fp32 284 and 287).
    const float decayed = pr[C - tc + (last ? 1 : 0)];
    each([&](int ct, int x, int i) { st[ct][x][i] *= decayed; });

    // --- keys x values into the state
    if (ewave) {
#pragma unroll
      for (int c = 0; c < kS; ++c) {
        // decayed, with the decays to the next chunk's first token or to the last one
        v4i wf[CT][kParts];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
          for (int k = 0; k < NV; ++k)
            vf[ct][c][k] = tile_turn8(v_t[k], (v_a0 ^ (ct << 5)) + c * 32 * (2 * WC), (v_a1 ^ (ct << 5)) + c * 32 * (2 * WC));
          if constexpr (STATE) {
#pragma unroll
            for (int k = 0; k < kParts; ++k) wf[ct][k] = vf[ct][c][k];
          } else {
            const float* const w = &pr[32 * c + 8 * g + C - tc + (last ? 1 : 0)];
            float y[8];
            sum8<NV>(vf[ct][c], y);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] *= alpha * w[j];
            split8<kParts>(y, wf[ct]);
          }
        }
#pragma unroll
        for (int x = 0; x < kB; ++x)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            v4i f[NK];
#pragma unroll
            for (int k = 0; k < NK; ++k)
              f[k] = tile_turn8(k_t[k], (k_a0_ ^ (x << 6)) + 8 * i + c * 32 * (2 * DK), (k_a1_ ^ (x << 6)) + 8 * i + c * 32 * (2 * DK));
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) st[ct][x][i] = mma(f, wf[ct], st[ct][x][i]);
          }
      }
    }

    if (!kEarly && next < end) load_queries(next, tokens_at(next));
    lds_barrier();
    if constexpr (!STATE) {
      if (ewave) {
        // --- values x products
#pragma unroll
        for (int t = 0; t < kT; ++t)
#pragma unroll
          for (int c = 0; c < kS; ++c) {
            if (2 * c > t) continue;
            v4i f[kParts];
#pragma unroll
            for (int k = 0; k < kParts; ++k) f[k] = tile_read(p_t[k], (p_row ^ (c << 6)) + t * 16 * (2 * C));
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) o[ct][t] = mma(vf[ct][c], f, o[ct][t]);
          }
      }
      // --- store: columns w0 + 4 g + r of token 16 t + n.  By every wave, those
      // without columns past the resource: with a branch around the stores the
      // next chunk's staging would wait for them too, not for its loads alone.
      ro.at(first_row(i0, tc), tc);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const int col = w0 + 16 * ct;
        const uint32_t at = col < p.Dv ? ro.base + static_cast<uint32_t>(n * ro.step + (col + 4 * g) * (OF32 ? 4 : 2)) : kOff;
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          const uint32_t off = at + static_cast<uint32_t>(16 * t * ro.step);
          const v4f& y = o[ct][t];
          if constexpr (OF32) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, y), ro.r, off, 0, 0);
          else __builtin_amdgcn_raw_buffer_store_b64(v2u{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])}, ro.r, off, 0, 0);
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
  if (STATE) out = p.s_out + (static_cast<int64_t>(bh) * p.nseg + seg) * p.Dk * p.Dv;
  else if (p.s_out != nullptr && seg + 1 == p.nseg) out = p.s_out + static_cast<int64_t>(bh) * p.Dk * p.Dv;
  if (out != nullptr) {
    const auto rs = __builtin_amdgcn_make_buffer_rsrc(out, 0, p.Dk * p.Dv * 4, kBufferWord3);
    each([&](int ct, int x, int i) {
      const int d = 32 * x + 8 * g + 4 * i, col = w0 + 16 * ct + n;
      const uint32_t at = col < p.Dv && d < p.Dk ? 4u * static_cast<uint32_t>(d * p.Dv + col) : kOff;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(st[ct][x][i][r]), rs, at + 4u * r * p.Dv, 0, 0);
    });
  }
}

// `n` passes of the same number of workgroups, widths in 64s, and waves.
template <Kind KQ, Kind KK, Kind KV, bool OF32, bool STATE>
hipError_t launch_passes(const LinattnPass* p, int n, hipStream_t stream) {
  LinattnPasses ps{};
  for (int i = 0; i < n; ++i) ps.p[i] = p[i];
  ps.n = static_cast<uint32_t>(n);
  ps.count = p->B * p->H * p->nseg * p->tiles;
  const auto go = [&](auto kernel, int waves) {
    hipLaunchKernelGGL(kernel, dim3(ps.count * ps.n), dim3(64 * waves), 0, stream, ps);
    return hipGetLastError();
  };
#define MMF_FORM(DK, WAVES, CT) \
  go(linattn_chunk_kernel<KQ, KK, KV, OF32, DK, WAVES, CT, STATE>, WAVES)
  if (p->Dk > 128) return p->waves == 4 ? MMF_FORM(256, 4, 1) : MMF_FORM(256, 8, 1);
  // 128 columns: parts of fp32 as 32 per wave, so that what a wave reads from LDS
  // serves twice as many (whole calls: 4 x 2048 fp32, backward, 325 -> 292 us; forward
  // 154 -> 131); bf16, with fewer of them, as 16 per wave (4 x 2048, backward, 175 us,
  // 32 per wave 182; 16384 146, 149)
  if constexpr (STATE || KQ == kBf16) {
    if (p->Dk > 64) return p->waves == 4 ? MMF_FORM(128, 4, 1) : MMF_FORM(128, 8, 1);
    return p->waves == 4 ? MMF_FORM(64, 4, 1) : MMF_FORM(64, 8, 1);
  } else {
    if (p->Dk > 64) return p->waves == 4 ? MMF_FORM(128, 4, 1) : MMF_FORM(128, 4, 2);
    return p->waves == 4 ? MMF_FORM(64, 4, 1) : MMF_FORM(64, 4, 2);
  }
#undef MMF_FORM
}

}  // namespace la
}  // namespace mmf
