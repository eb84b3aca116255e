// A step of beam search: the n best of W beams x V tokens, and the beams'
// states reordered after them.
//
//   score(w, v) = scores[w] + z[w][v] - ln sum_v exp z[w][v]
// in the order of falling scores, then rising beams, falling logits, rising
// tokens.  A done beam's row is taken as 0 at `end` and -inf elsewhere, without
// being read: it goes on as itself.  NaN logits count as -inf.
//
// Within a row the order is that of the logits, so a first kernel keeps the n
// best logits of each piece of a row, sorted, with the piece's maximum and its
// sum of exponentials (one pass over the logits); a second merges the lists of
// a row (equal logits: the piece with the lower tokens first), then those of
// the beams by their scores, in fp64 (scores next to each other are told apart,
// and a tie is a tie of equal inputs).
//
// The n best of a piece: of the 64 lanes' own maxima, the n-th largest is at
// most the piece's n-th largest logit, so only what reaches the largest such
// bound of the four waves goes to LDS (of the logits that are equal to it, the
// first n of each wave), where each counts those before it.  The smallest of the
// waves' n/4-th largest is such a bound too, which for evenly spread logits leaves
// little more than n (50000 fp32, n = 64: 66 -> 33 us; for n = 4 its search costs
// more than it saves, 9.3 -> 9.7); the first one limits the list whatever they are.
//
// 32 x 8 rows of 50000 bf16: 17 us for the pieces, bound by the vector unit (about
// 25 instructions for 64 logits), 8 for the merging, bound by its steps in line.
// Reordering those beams' states of 1 MB each, two layers: 118 us, 5.2 TB/s.
#include "beam.h"
#include "mmf_device.h"
#include "row_vec.h"

namespace mmf {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr double kLog2e = 1.4426950408889634074;

// A logit as a number whose order is its own; 0: none.
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);  // -0 is 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
// With its token: higher logits, then lower tokens first.
__device__ __forceinline__ uint64_t key_of(uint32_t o, int token) {
  return (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~token);
}
__device__ __forceinline__ int token_of(uint64_t key) { return static_cast<int>(~static_cast<uint32_t>(key)); }

struct Stat {
  double sum;    // of exp(z - max); of an infinite maximum: how many have it
  float max;
  float pad;
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
  return static_cast<uint32_t>(dpp_i32<CTRL>(static_cast<int>(v)));
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = max(v, dpp_u32<kDppXor1>(v));
  v = max(v, dpp_u32<kDppXor2>(v));
  v = max(v, dpp_u32<kDppHalfMirror>(v));
  v = max(v, dpp_u32<kDppMirror>(v));
  const auto at = [&](int lane) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), lane)); };
  return max(max(at(0), at(16)), max(at(32), at(48)));
}

// The largest x that at least n lanes' values reach; LOW: the lowest bit in
// which values differ (all below it are those of a bf16 logit's order).
template <int LOW>
__device__ __forceinline__ uint32_t nth_largest(uint32_t v, int n) {
  uint32_t x = 0;
#pragma unroll
  for (int bit = 31; bit >= LOW; --bit) {
    const uint32_t t = x | (1u << bit);
    if (__popcll(__ballot(v >= t)) >= n) x = t;
  }
  return x;
}

struct Scratch {
  uint64_t* keys;  // [rows][pieces][n], sorted; 0: none
  Stat* stats;     // [rows][pieces]
  int pieces, piece;
};

constexpr int kFew = 8;
// Candidates of a piece that LDS holds, and those that are ranked by counting
// (n = 32 of 64 rows of 32000: 30 us; one after the other, for any number, 46).
constexpr int list_size(int vals, int n) { return kWaves * ((n - 1) * vals + n); }
constexpr int kCounted = 1024;

template <typename T, int VALS>
__global__ __launch_bounds__(kThreads) void beam_piece_kernel(const BeamSelectArgs a, const Scratch s) {
  extern __shared__ uint64_t s_list[];
  __shared__ float s_max[kWaves];
  __shared__ double s_sum[kWaves];
  __shared__ uint32_t s_bound[kWaves], s_part[kWaves];
  __shared__ uint64_t s_key[kWaves];
  __shared__ int s_count;
  const int piece = blockIdx.x % s.pieces;
  const int64_t row = blockIdx.x / s.pieces;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int begin = piece * s.piece, end = min(begin + s.piece, a.V);
  const bool done = a.done != nullptr && a.done[row] != 0;
  // no branches: all loads in flight at once (a done row's read nothing)
  const auto z = row_rsrc(static_cast<const T*>(a.logits) + row * a.V + begin, end - begin, !done);
  uint32_t w[VALS];
#pragma unroll
  for (int i = 0; i < VALS; ++i) {
    const uint32_t at = (i * kThreads + threadIdx.x) * sizeof(T);
    if constexpr (sizeof(T) == 4) w[i] = __builtin_amdgcn_raw_buffer_load_b32(z, at, 0, 0);
    else w[i] = static_cast<uint32_t>(__builtin_amdgcn_raw_buffer_load_b16(z, at, 0, 0)) << 16;
  }
  float v[VALS];   // NaN, and what is behind the piece's end, as -inf
#pragma unroll
  for (int i = 0; i < VALS; ++i) {
    const int t = begin + i * kThreads + threadIdx.x;
    v[i] = t < end && !done ? __uint_as_float(w[i]) : -__builtin_inff();
    if (done && t == a.end && t < end) v[i] = 0.0f;   // (threads behind the end stand on the next piece's tokens)
  }
  if (threadIdx.x == 0) s_count = 0;
  float m = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < VALS; ++i) {
    v[i] = fmaxf(v[i], -__builtin_inff());
    m = fmaxf(m, v[i]);
  }
  // the lane's largest, where it has a logit at all.  A bf16 logit differs from
  // the others in the upper half only: the lower is 0, or of negative ones all ones
  const uint32_t top = begin + static_cast<int>(threadIdx.x) < end ? order_of(m) : 0u;
  m = wave_max_f32(m);
  const auto reached_by = [&](int n) {
    const uint32_t x = nth_largest<sizeof(T) == 4 ? 0 : 16>(top, n);
    return sizeof(T) == 2 && x != 0 && (x >> 31) == 0 ? x | 0xFFFFu : x;
  };
  const uint32_t bound_w = reached_by(a.n), part_w = a.n > kFew ? reached_by((a.n + kWaves - 1) / kWaves) : 0u;
  if (lane == 0) {
    s_max[wave] = m;
    s_bound[wave] = bound_w;
    s_part[wave] = part_w;
  }
  __syncthreads();
  m = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
  const uint32_t bound_o = max(max(max(s_bound[0], s_bound[1]), max(s_bound[2], s_bound[3])),
                               min(min(s_part[0], s_part[1]), min(s_part[2], s_part[3])));
  const float bound = bound_o != 0 ? logit_of(bound_o) : -__builtin_inff();

  // what reaches the bound; all of a piece that no wave has n lanes of
  int equal = 0;  // of the wave's, so far
#pragma unroll
  for (int i = 0; i < VALS; ++i) {
    if (__ballot(v[i] >= bound) == 0) continue;
    const int t = begin + i * kThreads + threadIdx.x;
    const uint64_t same = __ballot(v[i] == bound && t < end);
    const uint64_t below = same & ((uint64_t(1) << lane) - 1);
    const bool take = t < end && (v[i] > bound || (((same >> lane) & 1) != 0 && equal + __popcll(below) < a.n));
    equal += __popcll(same);
    const uint64_t mask = __ballot(take);
    if (mask != 0) {
      int at = 0;
      if (lane == 0) at = atomicAdd(&s_count, __popcll(mask));  // their order in the list does not matter
      at = __builtin_amdgcn_readfirstlane(at) + __popcll(mask & ((uint64_t(1) << lane) - 1));
      if (take) s_list[at] = key_of(order_of(v[i]), t);
    }
  }
  float e = 0.0f;
  if (__builtin_fabsf(m) < __builtin_inff()) {
#pragma unroll
    for (int i = 0; i < VALS; ++i) e += __builtin_amdgcn_exp2f((v[i] - m) * static_cast<float>(kLog2e));
  } else {
#pragma unroll
    for (int i = 0; i < VALS; ++i) e += v[i] == m ? 1.0f : 0.0f;
  }
  // what is behind the piece's end is -inf: nothing, but as many as the piece where all of it is
  const double sum = wave_sum_f64(e);
  if (lane == 0) s_sum[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) s.stats[row * s.pieces + piece] = {(s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]), m, 0.0f};
  const int count = s_count;
  uint64_t* const out = s.keys + (row * s.pieces + piece) * a.n;
  if (count <= kCounted) {
    for (int j = threadIdx.x; j < count; j += kThreads) {
      const uint64_t k = s_list[j];
      int before = 0;
      for (int i = 0; i < count; ++i) before += s_list[i] > k;
      if (before < a.n) out[before] = k;
    }
    if (threadIdx.x < a.n && static_cast<int>(threadIdx.x) >= count) out[threadIdx.x] = 0;
    return;
  }
  uint64_t last = ~uint64_t(0);  // many: one after the other
  for (int j = 0; j < a.n; ++j) {
    uint64_t best = 0;
    for (int i = threadIdx.x; i < count; i += kThreads) {
      const uint64_t k = s_list[i];
      if (k < last && k > best) best = k;
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) {
      const uint64_t k = __shfl_xor(best, x);
      best = k > best ? k : best;
    }
    if (lane == 0) s_key[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) best = s_key[w] > best ? s_key[w] : best;
    if (threadIdx.x == 0) out[j] = best;
    last = best;
    __syncthreads();
  }
}

// A score as a number whose order is its own.
__device__ __forceinline__ uint64_t order_of(double s) {
  const uint64_t b = __builtin_bit_cast(uint64_t, s + 0.0);
  return b >> 63 ? ~b : b | (uint64_t(1) << 63);
}

constexpr int kFinalWaves = 16;
constexpr int kStaged = 6144;   // keys of a batch's lists that LDS holds (64 beams of 1000 tokens, n = 64: 86 us, from memory 106)
constexpr int kRanked = 128;    // candidates of a batch that are ranked by counting (8 x 16: 17.8 us, merged 18.5; 16 x 16: 23.8, 20.8)

// A wave merges the lists of a row (a lane per piece); the beams' are then ranked
// by counting, or, of many, merged by wave 0 (a lane per beam).
__global__ __launch_bounds__(kFinalWaves* kWave) void beam_final_kernel(const BeamSelectArgs a, const Scratch s, bool staged) {
  extern __shared__ uint64_t s_dyn[];           // [W][n] merged; the lists where they are staged, then [W][n] scores
  __shared__ double s_score[kBeamMax];          // of each beam
  __shared__ double s_log[kBeamMax];            // ln of its sum of exponentials
  __shared__ float s_max[kBeamMax];
  const int64_t b = blockIdx.x;
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = s.pieces * a.n;
  const uint64_t* lists = s.keys + b * a.W * per;
  if (staged) {
    uint64_t* const l = s_dyn + a.W * a.n;
    for (int i = threadIdx.x; i < a.W * per; i += blockDim.x) l[i] = lists[i];
    lists = l;
  }
  for (int w = wave; w < a.W; w += waves) {
    Stat st{0.0, -__builtin_inff(), 0.0f};
    if (lane < s.pieces) st = s.stats[(b * a.W + w) * s.pieces + lane];
    const float m = wave_max_f32(st.max);
    double sum = 0.0;
    if (lane < s.pieces) sum = st.max == m ? st.sum : st.sum * exp(static_cast<double>(st.max) - m);
    sum = wave_sum_f64(sum);
    if (lane == 0) {
      const float c = a.scores[b * a.W + w];
      // scores that are no number, and rows in which no token is possible
      const bool none = !(c < __builtin_inff()) || m == -__builtin_inff();
      s_score[w] = none ? -__builtin_inf() : static_cast<double>(c);
      s_log[w] = none ? 0.0 : log(sum);
      s_max[w] = m;
    }
  }
  __syncthreads();
  for (int w = wave; w < a.W; w += waves) {
    const uint64_t* const l = lists + w * per + lane * a.n;
    int at = 0;
    uint64_t head = lane < s.pieces ? l[0] : 0;
    for (int j = 0; j < a.n; ++j) {
      const uint32_t o = static_cast<uint32_t>(head >> 32), best = wave_max_u32(o);
      const int from = __ffsll(__ballot(o == best)) - 1;  // of equal logits the lowest tokens
      if (lane == from) {
        s_dyn[w * a.n + j] = head;
        ++at;
        head = head != 0 && at < a.n ? l[at] : 0;
      }
    }
  }
  __syncthreads();
  // --- the scores, and the n best of them
  uint64_t* const order = s_dyn + a.W * a.n;   // in place of the lists
  const int all = a.W * a.n;
  const auto score_of = [&](uint64_t key, int w) {
    const float z = logit_of(static_cast<uint32_t>(key >> 32)), m = s_max[w];
    const double d = z == m ? 0.0 : static_cast<double>(z) - m;
    return s_score[w] + (d - s_log[w]);
  };
  const auto put = [&](int j, uint64_t key, int w, double score) {
    const int64_t out = b * a.n + j;
    const int token = token_of(key);
    a.new_scores[out] = static_cast<float>(score);
    a.tokens[out] = token;
    a.parents[out] = w;
    if (a.new_done != nullptr) a.new_done[out] = token == a.end || (a.done != nullptr && a.done[b * a.W + w] != 0);
  };
  for (int i = threadIdx.x; i < all; i += blockDim.x) order[i] = s_dyn[i] != 0 ? order_of(score_of(s_dyn[i], i / a.n)) : 0;
  __syncthreads();
  if (all <= kRanked) {  // each counts those before it: higher scores, and equal ones of lower beams or places
    for (int i = threadIdx.x; i < all; i += blockDim.x) {
      const uint64_t o = order[i];
      int before = 0;
      for (int k = 0; k < all; ++k) before += order[k] > o || (order[k] == o && k < i);
      if (before < a.n) put(before, s_dyn[i], i / a.n, score_of(s_dyn[i], i / a.n));
    }
    return;
  }
  if (wave != 0) return;
  int at = 0;
  uint64_t o = lane < a.W ? order[lane * a.n] : 0;
  for (int j = 0; j < a.n; ++j) {
    const uint32_t hi = static_cast<uint32_t>(o >> 32), best_hi = wave_max_u32(hi);
    const uint32_t lo = hi == best_hi ? static_cast<uint32_t>(o) : 0u, best_lo = wave_max_u32(lo);
    const int from = __ffsll(__ballot(hi == best_hi && lo == best_lo)) - 1;  // of equal scores the lowest beam
    if (lane == from) {
      const uint64_t key = s_dyn[lane * a.n + at];
      put(j, key, lane, score_of(key, lane));
      ++at;
      o = at < a.n ? order[lane * a.n + at] : 0;
    }
  }
}

// ---------------------------------------------------------------------------
// Reordering.  A thread holds a column of 16 (or 4) bytes of all rows of a
// batch that change, so that the rows can change in place.
// ---------------------------------------------------------------------------
constexpr int kSet = 128;
struct Set {
  const char* src[kSet];
  char* dst[kSet];
  int64_t row[kSet];       // bytes
  uint32_t first[kSet];    // first workgroup of each array
  uint32_t cols[kSet];     // workgroups per batch
  int n;
};

// Every row goes through a buffer resource of its own, of size 0 where it stays:
// no branch, so all loads are in flight at once (branches for every row made
// the compiler lay out a path for every set of rows, in 242 registers).
template <int WORDS, int MAXW, bool NT>
__global__ __launch_bounds__(kThreads) void beam_reorder_kernel(const Set s, const int32_t* __restrict__ parents, int W) {
  int lo = 0, hi = s.n - 1;  // the last array whose first workgroup is at most this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (s.first[mid] <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const uint32_t blk = blockIdx.x - s.first[lo];
  const int64_t b = blk / s.cols[lo];
  const uint32_t col = ((blk % s.cols[lo]) * kThreads + threadIdx.x) * (4u * WORDS);
  const int64_t row = s.row[lo];
  const char* const src = s.src[lo] + b * W * row;
  char* const dst = s.dst[lo] + b * W * row;
  const bool moved = src != dst;
  const int32_t* const p = parents + b * W;
  constexpr int kPolicy = NT ? kNontemporal : 0;
  typedef unsigned int vec __attribute__((ext_vector_type(WORDS == 4 ? 4 : 2)));
  vec v[MAXW];
  const auto from = [&](int j) {
    const int f = j < W ? __builtin_amdgcn_readfirstlane(p[j]) : j;
    return f < 0 || f >= W ? j : f;
  };
  const auto rsrc = [&](const char* base, int j, int f) {
    const bool on = j < W && (f != j || moved);
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, on ? static_cast<int>(row) : 0, kBufferWord3);
  };
#pragma unroll
  for (int j = 0; j < MAXW; ++j) {
    const int f = from(j);
    const auto r = rsrc(src + f * row, j, f);
    if constexpr (WORDS == 4) v[j] = __builtin_amdgcn_raw_buffer_load_b128(r, col, 0, kPolicy);
    else v[j][0] = __builtin_amdgcn_raw_buffer_load_b32(r, col, 0, kPolicy);
  }
#pragma unroll
  for (int j = 0; j < MAXW; ++j) {
    const auto r = rsrc(dst + j * row, j, from(j));
    if constexpr (WORDS == 4) __builtin_amdgcn_raw_buffer_store_b128(v[j], r, col, 0, kPolicy);
    else __builtin_amdgcn_raw_buffer_store_b32(v[j][0], r, col, 0, kPolicy);
  }
}

// Logits per thread: few where there are few rows, as long as a wave holds a
// row's pieces (4 rows of 32000 fp32: 8.9 us, with 16 per thread 9.2; 32 rows 12.8
// and 12.5, 256 rows of 50000 38 and 24).
constexpr int kMaxPieces = kWave;
int vals_of(int64_t rows, int V) {
  const int64_t small = (V + 4 * kThreads - 1) / (4 * kThreads);
  return small <= kMaxPieces && rows * small <= 512 ? 4 : 16;
}
int pieces_of(int64_t rows, int V) {
  const int piece = vals_of(rows, V) * kThreads;
  return (V + piece - 1) / piece;
}
static_assert(kBeamMaxV <= kMaxPieces * 16 * kThreads, "a lane per piece");

}  // namespace

size_t beam_select_bytes(int64_t B, int W, int V, int n) {
  const int64_t pieces = B * W * pieces_of(B * W, V);
  return static_cast<size_t>(pieces) * (sizeof(Stat) + sizeof(uint64_t) * n);
}

hipError_t launch_beam_select(const BeamSelectArgs& a, void* scratch, hipStream_t stream) {
  const int64_t rows = a.B * a.W;
  const int vals = vals_of(rows, a.V);
  Scratch s;
  s.pieces = pieces_of(rows, a.V);
  s.piece = (a.V + s.pieces - 1) / s.pieces;
  s.stats = static_cast<Stat*>(scratch);
  s.keys = reinterpret_cast<uint64_t*>(s.stats + rows * s.pieces);
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(rows * s.pieces)), dim3(kThreads),
                       list_size(vals, a.n) * sizeof(uint64_t), stream, a, s);
    return hipGetLastError();
  };
  const hipError_t e = a.is_f32 ? vals == 4 ? go(beam_piece_kernel<float, 4>) : go(beam_piece_kernel<float, 16>)
                       : vals == 4 ? go(beam_piece_kernel<uint16_t, 4>) : go(beam_piece_kernel<uint16_t, 16>);
  if (e != hipSuccess) return e;
  const int total = a.W * s.pieces * a.n;
  const bool staged = total <= kStaged;
  hipLaunchKernelGGL(beam_final_kernel, dim3(static_cast<uint32_t>(a.B)),
                     dim3(kWave * (a.W < kFinalWaves ? a.W : kFinalWaves)),
                     (a.W * a.n + (staged && s.pieces > 1 ? total : a.W * a.n)) * sizeof(uint64_t), stream, a, s, staged);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(const BeamReorderArgs& a, hipStream_t stream) {
  const int unit = a.W <= 16 ? 16 : 4;    // of 64 rows 16 bytes each would take 256 registers
  const int64_t most = int64_t(1) << 23;  // workgroups per launch
  int64_t bytes = 0;
  for (int64_t i = 0; i < a.count; ++i) bytes += a.row_bytes[i] * a.B * a.W;
  // streams pass the caches where the arrays fill the last of them (32 x 8 beams of
  // two states of 1 MB 149 -> 135 us; 8 x 8, 134 MB: 27, nontemporal 35)
  const bool nt = bytes >= kLastLevelBytes;
  int64_t done = 0;
  while (done < a.count) {
    Set s{};
    int64_t groups = 0;
    for (; done < a.count; ++done) {
      const int64_t cols = (a.row_bytes[done] / unit + kThreads - 1) / kThreads;
      if (cols == 0) continue;
      if (s.n == kSet || (s.n > 0 && groups + cols * a.B > most)) break;
      s.src[s.n] = static_cast<const char*>(a.src[done]);
      s.dst[s.n] = static_cast<char*>(a.dst[done]);
      s.row[s.n] = a.row_bytes[done];
      s.first[s.n] = static_cast<uint32_t>(groups);
      s.cols[s.n] = static_cast<uint32_t>(cols);
      groups += cols * a.B;
      ++s.n;
    }
    if (groups == 0) break;
    const auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(groups)), dim3(kThreads), 0, stream, s, a.parents, a.W);
      return hipGetLastError();
    };
    const hipError_t e = a.W <= 4    ? nt ? go(beam_reorder_kernel<4, 4, true>) : go(beam_reorder_kernel<4, 4, false>)
                         : a.W <= 8  ? nt ? go(beam_reorder_kernel<4, 8, true>) : go(beam_reorder_kernel<4, 8, false>)
                         : a.W <= 16 ? go(beam_reorder_kernel<4, 16, false>)
                                     : go(beam_reorder_kernel<1, 64, false>);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mmf
