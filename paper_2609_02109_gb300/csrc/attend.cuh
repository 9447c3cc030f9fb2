// One pass of linear attention, which its forward call and its gradients have in common.
//
// With D[t][s] = the product of the factors of steps s + 1..t (0 behind a trace's end; t >= s), a pass computes
//   out_i = sum over j of alpha D (x_i . y_j) z_j  +  what the state brings:  x_i S times the factors from there to i,
// where S gathers y_j z_j^T, forward in time (j <= i) or in reverse (j >= i):
//   forward:  o  = pass(q, k, v)      dq = pass(do, v, k), on the transposed states of the forward call
//   reverse:  dv = pass(k, q, do)     dk = pass(v, do, q), on the transposed states of dv's pass
// Where k or v stand, missing samples' rows are read as zeros (y and z forward, x in reverse); in reverse their results
// are zeros whatever the state and y hold.  No other condition on missing samples is needed.
#pragma once

#include "mf_ops.cuh"

namespace mf {

struct AttendSeq {
  const void* p;
  int64_t sb, st, sh;
};

struct AttendPass {
  AttendSeq x, y, z, out;      // (out.p is written)
  const uint8_t* marks;
  int64_t marks_sb, marks_st;
  const float* log_decay;
  // the states that segments start from, [batch][heads][state_segs][dx][dz] (or [dz][dx]); NULL: zeros
  const float* state;
  int state_segs;
  bool state_t;
  float* final_state;          // [batch][heads][dx][dz] behind the last segment; NULL: not wanted
  float* save;                 // [batch][heads][dx][dz]: the state at the start (calls of one segment); NULL: not wanted
  // a pass for segments' own states alone: [batch][heads][segs][dx][dz], and the samples of each, or -1 where a trace
  // begins in it
  float* local;
  float* seen;
  int64_t time;
  int heads, dx, dz;
  int chunks, segs, seg_chunks;
  float alpha, alpha_row, alpha_src;
  bool reverse;
  bool few_warps;              // scan_columns
  uint32_t tries;              // of each bounded wait
  uint32_t* status;
};

// The logarithm of a head's factor; finite, so that no samples leave exactly 1.  (NaN stays.)
__device__ __forceinline__ float finite_log(float l) { return l < -1e30f ? -1e30f : l > 1e30f ? 1e30f : l; }
constexpr float kLog2e = 1.4426950408889634f;

// The third root of 2^e, for e > 0: three factors that are float32s, of one that may be none.  (Beyond 2^360 nothing but 0
// stays in range.  A NaN stays.)
__device__ __forceinline__ float third_root(float e) { return exp2f((e > 360.f ? 360.f : e) * (1.f / 3.f)); }

// What is left of a state after some samples (fewer than none: nothing at all).  A factor near 1 that is rounded to fp32
// would be off the same way in every chunk of a long memory (2000 samples by chunks of 32: 1.7e-6 of the state), so it
// is kept as what is lost, and the state goes through one rounding a chunk.  Where a memory has grown by a factor that is no
// float32 (beyond()), the state has to be grown() first: what is nothing stays nothing.
struct Remains {
  float factor, lost, third = 0.f;
  __device__ __forceinline__ Remains(float log_decay, float samples) {
    factor = samples < 0.f ? -1.f : exp2f(log_decay * kLog2e * samples);
    lost = samples < 0.f ? 0.f : expm1f(log_decay * samples);
    if (lost > 3.4028235e38f) {
      third = third_root(log_decay * kLog2e * samples);
      factor = 1.f;
      lost = 0.f;
    }
  }
  __device__ __forceinline__ bool beyond() const { return third > 0.f; }
  __device__ __forceinline__ float grown(float state) const { return state * third * third * third; }
  __device__ __forceinline__ float operator()(float state, float more) const {
    return factor < 0.f ? more : factor >= 0.5f ? state + fmaf(state, lost, more) : fmaf(state, factor, more);
  }
};

// A pass step by step on the CUDA cores; segments of whole kAttendScanChunk steps.
constexpr int kAttendScanChunk = 64;
// Columns of a warp, whose lanes hold all rows of x.  A lane's values are the more the fewer loads from shared memory a
// product takes; where there are few heads and steps (`few_warps`) narrower warps keep more of the GPU busy.
inline int scan_columns(int dx, int dz, bool few_warps) {
  if (dx <= 16) return dz <= 16 ? 16 : 32;
  if (dx <= 64) return few_warps || dz <= 8 ? 8 : dz <= 16 ? 16 : 32;
  return few_warps || dz <= 8 ? 8 : 16;
}
// Warps of an SM, by the registers that the rows take.  (16 x 16 x 86400 with marks: 343 us a call with 16, 354 with 20, 378 with 24.)
__host__ __device__ constexpr int scan_warps(int dx) { return dx <= 32 ? 16 : 8; }
mf_status attend_scan(int type, const AttendPass& p, int64_t rows, cudaStream_t s);
mf_status attend_scan_bf16(const AttendPass& p, int64_t rows, cudaStream_t s);
mf_status attend_scan_f16(const AttendPass& p, int64_t rows, cudaStream_t s);

// A tensor-core pass over chunks of kAttendTcChunk steps (bf16, fp16).
constexpr int kAttendTcChunk = 128;
mf_status attend_tc(int type, const AttendPass& p, int64_t rows, cudaStream_t s);

}  // namespace mf
