// A step of beam search: the n best of W beams x V tokens, and the beams'
// states reordered after them.
//
//   score(w, v) = scores[w] + z[w][v] - ln sum_v exp z[w][v]
// in the order of falling scores, then rising beams, falling logits, rising
// tokens.  A done beam's row is taken as 0 at `end` and -inf elsewhere, without
// being read: it goes on as itself.  NaN logits count as -inf.
//
// Within a row the order is that of the logits, so a first kernel keeps the n
// best logits of each piece of a row, with the piece's maximum and its sum of
// exponentials (one pass over the logits); a second computes the scores of
// what is left, in fp64 (scores next to each other are told apart, and a tie
// is a tie of equal inputs), and takes the n best.
#include "beam.h"
#include "mmf_device.h"
#include "row_vec.h"

namespace mmf {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr double kLog2e = 1.4426950408889634074;
constexpr int kVals = 16;                      // logits per thread
constexpr int kPiece = kThreads * kVals;       // logits per piece at most

// A logit and its token, as a number whose order is theirs (higher logit, then
// lower token); 0: none.
__device__ __forceinline__ uint64_t key_of(float z, int token) {
  const uint32_t b = __float_as_uint(z + 0.0f);  // -0 is 0
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~token);
}
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t o = static_cast<uint32_t>(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ int token_of(uint64_t key) { return static_cast<int>(~static_cast<uint32_t>(key)); }

struct Stat {
  double sum;    // of exp(z - max); of an infinite maximum: how many have it
  float max;
  float pad;
};

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int x = 1; x < kWave; x *= 2) {
    const uint64_t o = __shfl_xor(v, x);
    v = o > v ? o : v;
  }
  return v;
}

struct Scratch {
  uint64_t* keys;  // [rows][pieces][n]
  Stat* stats;     // [rows][pieces]
  int pieces, piece;
};

template <typename T>
__global__ __launch_bounds__(kThreads) void beam_piece_kernel(const BeamSelectArgs a, const Scratch s) {
  __shared__ float s_max[kWaves];
  __shared__ double s_sum[kWaves];
  __shared__ uint64_t s_key[kWaves];
  const int piece = blockIdx.x % s.pieces;
  const int64_t row = blockIdx.x / s.pieces;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int begin = piece * s.piece, end = min(begin + s.piece, a.V);
  const bool done = a.done != nullptr && a.done[row] != 0;
  const T* const z = static_cast<const T*>(a.logits) + row * a.V;
  float v[kVals];
#pragma unroll
  for (int i = 0; i < kVals; ++i) {
    const int t = begin + i * kThreads + threadIdx.x;
    float x = -__builtin_inff();
    if (done) {
      if (t == a.end) x = 0.0f;
    } else if (t < end) {
      if constexpr (sizeof(T) == 4) x = z[t];
      else x = bf16_to_f32(z[t]);
      if (x != x) x = -__builtin_inff();
    }
    v[i] = x;
  }
  float m = v[0];
#pragma unroll
  for (int i = 1; i < kVals; ++i) m = fmaxf(m, v[i]);
  m = wave_max_f32(m);
  if (lane == 0) s_max[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
  float e = 0.0f;
#pragma unroll
  for (int i = 0; i < kVals; ++i)
    e += v[i] == m ? 1.0f : __builtin_amdgcn_exp2f((v[i] - m) * static_cast<float>(kLog2e));
  const double sum = wave_sum_f64(e);
  if (lane == 0) s_sum[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) s.stats[row * s.pieces + piece] = {(s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]), m, 0.0f};
  // the n best, one after the other
  uint64_t last = ~uint64_t(0);
  for (int j = 0; j < a.n; ++j) {
    uint64_t best = 0;
#pragma unroll
    for (int i = 0; i < kVals; ++i) {
      const int t = begin + i * kThreads + threadIdx.x;
      const uint64_t k = t < end ? key_of(v[i], t) : 0;
      if (k < last && k > best) best = k;
    }
    best = wave_max(best);
    if (lane == 0) s_key[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) best = s_key[w] > best ? s_key[w] : best;
    if (threadIdx.x == 0) s.keys[(row * s.pieces + piece) * a.n + j] = best;
    last = best;
    __syncthreads();
  }
}

struct Candidate {
  double score;
  uint64_t key;
  int beam;      // -1: none
};
__device__ __forceinline__ bool before(const Candidate& a, const Candidate& b) {
  if (b.beam < 0) return a.beam >= 0;
  if (a.beam < 0) return false;
  if (a.score != b.score) return a.score > b.score;
  if (a.beam != b.beam) return a.beam < b.beam;
  return a.key > b.key;
}

__global__ __launch_bounds__(kThreads) void beam_final_kernel(const BeamSelectArgs a, const Scratch s) {
  __shared__ double s_score[kBeamMax];   // of each beam
  __shared__ double s_log[kBeamMax];     // ln of its sum of exponentials
  __shared__ float s_max[kBeamMax];
  __shared__ Candidate s_best[kWaves];
  const int64_t b = blockIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (threadIdx.x < a.W) {
    const Stat* const st = s.stats + (b * a.W + threadIdx.x) * s.pieces;
    float m = -__builtin_inff();
    for (int p = 0; p < s.pieces; ++p) m = fmaxf(m, st[p].max);
    double sum = 0.0;
    for (int p = 0; p < s.pieces; ++p) sum += st[p].max == m ? st[p].sum : st[p].sum * exp(static_cast<double>(st[p].max) - m);
    const float c = a.scores[b * a.W + threadIdx.x];
    // scores that are no number, and rows in which no token is possible
    const bool none = !(c < __builtin_inff()) || m == -__builtin_inff();
    s_score[threadIdx.x] = none ? -__builtin_inf() : static_cast<double>(c);
    s_log[threadIdx.x] = none ? 0.0 : log(sum);
    s_max[threadIdx.x] = m;
  }
  __syncthreads();
  const int per = s.pieces * a.n, total = a.W * per;
  const uint64_t* const keys = s.keys + b * total;
  const auto candidate = [&](int i) {
    Candidate c{0.0, keys[i], i / per};
    if (c.key == 0) {
      c.beam = -1;
    } else {
      const float z = logit_of(c.key), m = s_max[c.beam];
      const double d = z == m ? 0.0 : static_cast<double>(z) - m;
      c.score = s_score[c.beam] + (d - s_log[c.beam]);
    }
    return c;
  };
  Candidate last{__builtin_inf(), ~uint64_t(0), 0};
  for (int j = 0; j < a.n; ++j) {
    Candidate best{0.0, 0, -1};
    for (int i = threadIdx.x; i < total; i += kThreads) {
      const Candidate c = candidate(i);
      if (before(last, c) && before(c, best)) best = c;
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) {
      const Candidate o{__shfl_xor(best.score, x), __shfl_xor(best.key, x), __shfl_xor(best.beam, x)};
      if (before(o, best)) best = o;
    }
    if (lane == 0) s_best[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (before(s_best[w], best)) best = s_best[w];
    if (threadIdx.x == 0) {
      const int64_t at = b * a.n + j;
      const int token = token_of(best.key);
      a.new_scores[at] = static_cast<float>(best.score);
      a.tokens[at] = token;
      a.parents[at] = best.beam;
      if (a.new_done != nullptr)
        a.new_done[at] = token == a.end || (a.done != nullptr && a.done[b * a.W + best.beam] != 0);
    }
    last = best;
    __syncthreads();
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

template <typename U, int MAXW>
__global__ __launch_bounds__(kThreads) void beam_reorder_kernel(const Set s, const int32_t* __restrict__ parents, int W) {
  int lo = 0, hi = s.n - 1;  // the last array whose first workgroup is at most this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (s.first[mid] <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const uint32_t blk = blockIdx.x - s.first[lo];
  const int64_t b = blk / s.cols[lo];
  const int64_t col = (static_cast<int64_t>(blk % s.cols[lo]) * kThreads + threadIdx.x) * sizeof(U);
  const int64_t row = s.row[lo];
  if (col >= row) return;
  const char* const src = s.src[lo] + b * W * row + col;
  char* const dst = s.dst[lo] + b * W * row + col;
  const bool moved = src != dst;
  const int32_t* const p = parents + b * W;
  U v[MAXW];
#pragma unroll
  for (int j = 0; j < MAXW; ++j) {
    if (j >= W) break;
    int from = p[j];
    if (from < 0 || from >= W) from = j;
    if (from != j || moved) v[j] = *reinterpret_cast<const U*>(src + from * row);
  }
#pragma unroll
  for (int j = 0; j < MAXW; ++j) {
    if (j >= W) break;
    const int from = p[j];
    if ((from != j && from >= 0 && from < W) || moved) *reinterpret_cast<U*>(dst + j * row) = v[j];
  }
}

int pieces_of(int V) { return (V + kPiece - 1) / kPiece; }

}  // namespace

size_t beam_select_bytes(int64_t B, int W, int V, int n) {
  const int64_t pieces = B * W * pieces_of(V);
  return static_cast<size_t>(pieces) * (sizeof(Stat) + sizeof(uint64_t) * n);
}

hipError_t launch_beam_select(const BeamSelectArgs& a, void* scratch, hipStream_t stream) {
  Scratch s;
  s.pieces = pieces_of(a.V);
  s.piece = (a.V + s.pieces - 1) / s.pieces;
  s.stats = static_cast<Stat*>(scratch);
  s.keys = reinterpret_cast<uint64_t*>(s.stats + a.B * a.W * s.pieces);
  const dim3 grid(static_cast<uint32_t>(a.B * a.W * s.pieces));
  if (a.is_f32) hipLaunchKernelGGL(beam_piece_kernel<float>, grid, dim3(kThreads), 0, stream, a, s);
  else hipLaunchKernelGGL(beam_piece_kernel<uint16_t>, grid, dim3(kThreads), 0, stream, a, s);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL(beam_final_kernel, dim3(static_cast<uint32_t>(a.B)), dim3(kThreads), 0, stream, a, s);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(const BeamReorderArgs& a, hipStream_t stream) {
  const int unit = a.W <= 16 ? 16 : 4;
  const int64_t most = int64_t(1) << 23;  // workgroups per launch
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
    const hipError_t e = a.W <= 4    ? go(beam_reorder_kernel<uint4, 4>)
                         : a.W <= 8  ? go(beam_reorder_kernel<uint4, 8>)
                         : a.W <= 16 ? go(beam_reorder_kernel<uint4, 16>)
                                     : go(beam_reorder_kernel<uint32_t, 64>);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mmf
