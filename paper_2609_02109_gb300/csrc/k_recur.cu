// Gated linear recurrence over sequences (the operators' section of include/mf.h).
#include "mf_ops.cuh"

namespace mf {
namespace {

struct Seq {
  void* p;
  int64_t sb, st;
};
Seq seq(const mf_seq& t) { return {t.d_ptr, t.stride_batch, t.stride_time}; }

struct Fwd {
  int64_t batch, time, dim;
  Seq x, z, h;
  const uint8_t* marks;
  int64_t mb, mt;
  const float* h0;
  float *last, *saved;
};
struct Bwd {
  int64_t batch, time, dim;
  Seq x, z, dh, dx, dz;
  const uint8_t* marks;
  int64_t mb, mt;
  const float *saved, *dlast;
  float* dh0;
};

// The gate f = 1 / (1 + e^-z) and 1 - f = e^-z / (1 + e^-z), both without cancellation; z below
// -80 counts as -80 (f is then about 1e-35) so that e^-z stays finite.
__device__ __forceinline__ void gate(float z, float& f, float& g) {
  if (z != z) { f = g = z; return; }
  const float e = expf(-fmaxf(z, -80.f));
  f = 1.f / (1.f + e);
  g = e * f;
}

// One thread a channel, step after step.
template <typename T>
__global__ void __launch_bounds__(256) k_recur_fwd(const Fwd a) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= a.batch * a.dim) return;
  const int64_t b = i / a.dim, c = i % a.dim;
  const T* x = (const T*)a.x.p + b * a.x.sb + c;
  const T* z = (const T*)a.z.p + b * a.z.sb + c;
  T* h = (T*)a.h.p + b * a.h.sb + c;
  const int64_t nseg = (a.time + kRecurSave - 1) / kRecurSave;
  float s = a.h0 ? a.h0[i] : 0.f;
  for (int64_t t = 0; t < a.time; ++t) {
    if (a.saved && t % kRecurSave == 0) a.saved[(b * nseg + t / kRecurSave) * a.dim + c] = s;
    const int m = a.marks ? a.marks[b * a.mb + t * a.mt] : MF_MARK_SAMPLE;
    if (m != MF_MARK_MISSING) {
      float f, g;
      gate(to_f32(z[t * a.z.st]), f, g);
      const float in = g * to_f32(x[t * a.x.st]);
      s = m == MF_MARK_FIRST ? in : fmaf(f, s, in);
    }
    h[t * a.h.st] = from_f32<T>(s);
  }
  if (a.last) a.last[i] = s;
}

template <typename T>
__global__ void __launch_bounds__(256) k_recur_bwd(const Bwd a) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= a.batch * a.dim) return;
  const int64_t b = i / a.dim, c = i % a.dim;
  const T* x = (const T*)a.x.p + b * a.x.sb + c;
  const T* z = (const T*)a.z.p + b * a.z.sb + c;
  const T* dh = (const T*)a.dh.p + b * a.dh.sb + c;
  T* dx = (T*)a.dx.p + b * a.dx.sb + c;
  T* dz = (T*)a.dz.p + b * a.dz.sb + c;
  const int64_t nseg = (a.time + kRecurSave - 1) / kRecurSave;
  float l = a.dlast ? a.dlast[i] : 0.f;
  for (int64_t seg = nseg - 1; seg >= 0; --seg) {
    const int64_t t0 = seg * kRecurSave;
    const int len = (int)min((int64_t)kRecurSave, a.time - t0);
    float before[kRecurSave];
    float s = a.saved[(b * nseg + seg) * a.dim + c];
    for (int j = 0; j < len; ++j) {
      const int64_t t = t0 + j;
      const int m = a.marks ? a.marks[b * a.mb + t * a.mt] : MF_MARK_SAMPLE;
      before[j] = m == MF_MARK_FIRST ? 0.f : s;
      if (m == MF_MARK_MISSING) continue;
      float f, g;
      gate(to_f32(z[t * a.z.st]), f, g);
      const float in = g * to_f32(x[t * a.x.st]);
      s = m == MF_MARK_FIRST ? in : fmaf(f, s, in);
    }
    for (int j = len - 1; j >= 0; --j) {
      const int64_t t = t0 + j;
      const int m = a.marks ? a.marks[b * a.mb + t * a.mt] : MF_MARK_SAMPLE;
      l += to_f32(dh[t * a.dh.st]);
      float gx = 0.f, gz = 0.f;
      if (m != MF_MARK_MISSING) {
        float f, g;
        gate(to_f32(z[t * a.z.st]), f, g);
        gx = g * l;
        gz = l * (before[j] - to_f32(x[t * a.x.st])) * (f * g);
        l = m == MF_MARK_FIRST ? 0.f : f * l;
      }
      dx[t * a.dx.st] = from_f32<T>(gx);
      dz[t * a.dz.st] = from_f32<T>(gz);
    }
  }
  if (a.dh0) a.dh0[i] = l;
}

}  // namespace

mf_status recur_work(int, int64_t, int64_t, int64_t, bool, uint64_t* bytes) {
  *bytes = 0;
  return MF_OK;
}

mf_status recur_forward(const mf_recurrence_args& p, void*, cudaStream_t s) {
  const Fwd a{p.batch, p.time, p.dim, seq(p.x), seq(p.z), seq(p.h), p.d_marks, p.marks_stride_batch, p.marks_stride_time,
              p.d_h0, p.d_last, p.d_saved};
  const unsigned grid = (unsigned)((p.batch * p.dim + 255) / 256);
  if (p.type == MF_TYPE_F32) k_recur_fwd<float><<<grid, 256, 0, s>>>(a);
  else if (p.type == MF_TYPE_BF16) k_recur_fwd<__nv_bfloat16><<<grid, 256, 0, s>>>(a);
  else k_recur_fwd<__half><<<grid, 256, 0, s>>>(a);
  MF_CUDA(cudaGetLastError());
  return MF_OK;
}

mf_status recur_backward(const mf_recurrence_grad_args& p, void*, cudaStream_t s) {
  const Bwd a{p.batch, p.time, p.dim, seq(p.x), seq(p.z), seq(p.dh), seq(p.dx), seq(p.dz), p.d_marks, p.marks_stride_batch,
              p.marks_stride_time, p.d_saved, p.d_dlast, p.d_dh0};
  const unsigned grid = (unsigned)((p.batch * p.dim + 255) / 256);
  if (p.type == MF_TYPE_F32) k_recur_bwd<float><<<grid, 256, 0, s>>>(a);
  else if (p.type == MF_TYPE_BF16) k_recur_bwd<__nv_bfloat16><<<grid, 256, 0, s>>>(a);
  else k_recur_bwd<__half><<<grid, 256, 0, s>>>(a);
  MF_CUDA(cudaGetLastError());
  return MF_OK;
}

}  // namespace mf
