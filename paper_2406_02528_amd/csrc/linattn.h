// Internal launchers of the linear attention kernels.  Shapes are validated by
// the C-ABI layer before any of these is called.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mmf {

// Linear attention with a decay per head (linattn_step.hip, linattn_chunk.hip):
// B sequences of T tokens, H heads, rows of qkv = q [H][dk] | k [H][dk] | v
// [H][dv]; o [B*T][H][dv] in the type of qkv; s0, s_last [B][H][dk][dv]
// (nullptr: 0, not stored; may be the same array).
constexpr int kLinattnMaxDim = 256;
constexpr int kLinattnChunk = 32;   // tokens of a chunk
struct LinattnArgs {
  const void* qkv;
  bool is_f32;
  const float* decay;
  float scale;
  const float* s0;
  void* o;
  float* s_last;
  int64_t B, T, H;
  int dk, dv;
};
hipError_t launch_linattn_step(const LinattnArgs& a, hipStream_t stream);

// A pass over chunks (linattn_chunk.h).  Operands: the first row of a segment
// of the stacked rows, `ld` elements from one row to the next, head h at h
// times its width.
struct LinattnOperand {
  const void* p;
  int64_t ld;
  bool is_f32;
};
struct LinattnPass {
  LinattnOperand q, k, v;
  void* o;
  int64_t ldo;
  const float* decay;
  float alpha, beta;
  bool rev;
  // the state that enters segment `seg` of state bh: entry (d, e) at e_in[bh
  // e_bh + seg e_seg + d e_d + e e_e] (nullptr: 0), times the decay if e_decay
  const float* e_in;
  int64_t e_bh, e_seg;
  int e_d, e_e;
  bool e_decay;
  // the state behind the last token (nullptr: not stored); of a pass for
  // states alone the segments' own sums [B H][nseg][Dk][Dv], those of segments
  // below `segs`
  float* s_out;
  uint32_t segs;
  uint32_t B, H;
  int64_t T;
  int Dk, Dv;
  uint32_t nseg, tiles;   // segments; workgroups per state
  int waves;              // of a workgroup, for 16 columns each: 4 or 8
  int64_t seg_tokens;
};
// Up to three passes of one kernel in a launch, `count` workgroups each.
struct LinattnPasses {
  LinattnPass p[3];
  uint32_t n, count;
};
// Of at least one token (as the launches).
size_t linattn_chunk_bytes(int64_t B, int64_t T, int64_t H, int dk, int dv);
hipError_t launch_linattn_chunk(const LinattnArgs& a, float* joined, hipStream_t stream);
// Backward: dqkv bf16; s0, ds_last, ds0 may be nullptr, ds0 may be ds_last.
struct LinattnBwdArgs {
  const void* qkv;
  bool is_f32;
  const float* decay;
  float scale;
  const float* s0;
  const void* dout;
  bool do_is_f32;
  const float* ds_last;
  uint16_t* dqkv;
  float* ds0;
  int64_t B, T, H;
  int dk, dv;
};
size_t linattn_bwd_bytes(int64_t B, int64_t T, int64_t H, int dk, int dv);
hipError_t launch_linattn_bwd(const LinattnBwdArgs& a, float* joined, hipStream_t stream);

}  // namespace mmf
