// Sums of squares that neither overflow nor underflow in fp32.
#pragma once

#include "mf_ops.cuh"

namespace mf {

// Squares in three ranges, so that none overflows or underflows in fp32: small values scaled by 2^96, large ones by
// 2^-90.  No sum of 2^40 squares, the most that a matrix (or a set of tensors) has, passes 2^120.
struct Squares {
  float mid = 0.f, small = 0.f, large = 0.f;
  __device__ __forceinline__ void add(float v) {
    const float m = fabsf(v);
    if (m < 0x1p-62f) small = fmaf(v * 0x1p96f, v * 0x1p96f, small);
    else if (m > 0x1p40f) large = fmaf(v * 0x1p-90f, v * 0x1p-90f, large);
    else mid = fmaf(v, v, mid);  // (NaN too)
  }
  __device__ __forceinline__ void add(const Squares& q) {
    mid += q.mid;
    small += q.small;
    large += q.large;
  }
};
__device__ __forceinline__ Squares warp_sum(Squares q) {
  for (int w = 16; w > 0; w >>= 1) {
    q.mid += __shfl_xor_sync(0xffffffffu, q.mid, w);
    q.small += __shfl_xor_sync(0xffffffffu, q.small, w);
    q.large += __shfl_xor_sync(0xffffffffu, q.large, w);
  }
  return q;
}

// The block's sum of squares, in every thread of its first warp.
__device__ __forceinline__ Squares block_sum(Squares q, Squares* part) {
  q = warp_sum(q);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = q;
  __syncthreads();
  q = Squares{};
  if (threadIdx.x < blockDim.x / 32) q = part[threadIdx.x];
  return threadIdx.x < 32 ? warp_sum(q) : q;
}

// The square root of the sum; infinite where that is no float32.
__device__ __forceinline__ float norm_of(const Squares& q) {
  if (q.large > 0.f) return sqrtf(fmaf(q.mid * 0x1p-90f, 0x1p-90f, q.large)) * 0x1p90f;
  if (q.mid < 0x1p-70f) return sqrtf(fmaf(q.mid * 0x1p96f, 0x1p96f, q.small)) * 0x1p-96f;
  return sqrtf(fmaf(q.small * 0x1p-96f, 0x1p-96f, q.mid));
}

}  // namespace mf
