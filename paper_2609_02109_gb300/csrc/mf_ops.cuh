// Internal declarations of the training operators (see the operators' section of include/mf.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "mf_internal.cuh"

namespace mf {

// Steps between the states that a forward recurrence saves for its gradient.
constexpr int kRecurSave = 16;

// wait_test: mf_debug_operators_wait_test's polls.
mf_status recur_forward(const mf_recurrence_args& p, void* work, uint32_t wait_test, cudaStream_t s);
mf_status recur_backward(const mf_recurrence_grad_args& p, void* work, uint32_t wait_test, cudaStream_t s);
// Scratch bytes of a call with these sizes.
mf_status recur_work(int type, int64_t batch, int64_t time, int64_t dim, bool backward, uint64_t* bytes);

// The largest |a s + b s^3 + c s^5| of 0 <= s <= top: at the end or where the derivative, quadratic in s^2, is zero.
double orth_largest(const mf_orthogonalize_args& p, double top);
mf_status orth_work(const mf_orthogonalize_args& p, uint64_t* bytes);
mf_status orth_run(const mf_orthogonalize_args& p, void* work, uint32_t wait_test, cudaStream_t s);

// Arithmetic is in fp32; a value is rounded to its tensor's type once, to nearest.
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32(float v) { return v; }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }

}  // namespace mf
