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
// times its width.  The state s_in, s_out (nullptr: 0, not stored) has strides
// in_d and in_e within a head's Dk Dv entries.
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
  const float* s_in;
  float* s_out;
  int64_t in_d, in_e;
  uint32_t B, H;
  int64_t T;
  int Dk, Dv;
  // from linattn_plan
  uint32_t nseg, tiles;
  int et;
  int64_t seg_tokens;
  float* joined;   // [B H][nseg][Dk][Dv]; nullptr: one segment, from s_in
  bool join_last;  // the joining gives s_out (the last segment's own sum too)
};
// How a pass is cut: columns of the state per workgroup (64 et) and tokens per
// segment.
struct LinattnPlan {
  uint32_t nseg, tiles;
  int et;
  int64_t seg_tokens;
  size_t joined_bytes;
};
LinattnPlan linattn_plan(int64_t B, int64_t T, int64_t H, int Dk, int Dv);
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
