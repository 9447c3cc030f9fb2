// C ABI of the training operators: argument checks, then the kernels' host sides.  Messages allocate, so each entry
// point ends exceptions in MF_ENOMEM.
#include <cmath>
#include <string>

#include "mf_ops.cuh"

namespace mf {
namespace {

mf_status refuse(const char* where, const std::string& msg) {
  set_error(std::string(where) + ": " + msg);
  return MF_EINVAL;
}

int type_size(int type) { return type == MF_TYPE_F32 ? 4 : 2; }
bool known_type(int type) { return type == MF_TYPE_F32 || type == MF_TYPE_BF16 || type == MF_TYPE_F16; }
bool aligned(const void* p, int to) { return ((uintptr_t)p & (uintptr_t)(to - 1)) == 0; }

thread_local uint32_t t_wait_test = 0;
__device__ uint32_t g_operators_status;  // (zero when the module is loaded: nothing to set, in no stream's order)

constexpr int64_t kMaxSize = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxRows = int64_t(1) << 38;  // channels of all sequences (launch sizes)
constexpr int64_t kMaxStride = int64_t(1) << 56;

// Whether two axes (counts n1, n2; strides s1, s2) of rows of `width` elements never meet.
bool apart(int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t width) {
  if (n1 > 1 && n2 > 1 && s1 > s2) return apart(n2, s2, n1, s1, width);
  if (n1 <= 1) return n2 <= 1 || s2 >= width;
  if (s1 < width) return false;
  return n2 <= 1 || s2 >= (n1 - 1) * s1 + width;
}

std::string check_sizes(int32_t type, int64_t batch, int64_t time, int64_t dim) {
  if (!known_type(type)) return "unknown type";
  if (batch < 0 || time < 0 || dim < 0) return "a size is negative";
  if (batch > kMaxSize || time > kMaxSize || dim > kMaxSize) return "a size is 2^31 or more";
  if (batch > kMaxRows / (dim > 0 ? dim : 1)) return "batch * dim is too large";
  if (batch && time && dim && batch * dim > kMaxStride / time) return "batch * time * dim is too large";
  return "";
}

std::string check_seq(const mf_seq& t, const char* name, int32_t type, int64_t batch, int64_t time, int64_t dim, bool out) {
  if (!batch || !time || !dim) return "";
  if (!t.d_ptr) return std::string(name) + " is NULL";
  if (!aligned(t.d_ptr, type_size(type))) return std::string(name) + " is not aligned to its type";
  if (t.stride_batch < 0 || t.stride_time < 0 || t.stride_batch > kMaxStride / batch || t.stride_time > kMaxStride / time)
    return std::string(name) + ": a stride is out of range";
  if (out && !apart(time, t.stride_time, batch, t.stride_batch, dim)) return std::string(name) + " overlaps itself";
  return "";
}

std::string check_marks(const uint8_t* marks, int64_t sb, int64_t st, int64_t batch, int64_t time) {
  if (!marks || !batch || !time) return "";
  if (sb < 0 || st < 0 || sb > kMaxStride / batch || st > kMaxStride / time) return "marks: a stride is out of range";
  return "";
}

std::string check_work(const void* work, uint64_t bytes, uint64_t need) {
  if (!need) return "";
  if (!work) return "d_work is NULL";
  if (!aligned(work, 16)) return "d_work is not 16-byte aligned";
  if (bytes < need) return "d_work is too small: " + std::to_string(need) + " bytes are needed";
  return "";
}

}  // namespace
}  // namespace mf

using namespace mf;

extern "C" {

mf_status mf_recurrence_sizes(int32_t type, int64_t batch, int64_t time, int64_t dim, uint64_t* saved_floats,
                              uint64_t* forward_bytes, uint64_t* backward_bytes) try {
  const char* me = "mf_recurrence_sizes";
  const std::string bad = check_sizes(type, batch, time, dim);
  if (!bad.empty()) return refuse(me, bad);
  if (saved_floats) *saved_floats = (uint64_t)batch * (uint64_t)((time + kRecurSave - 1) / kRecurSave) * (uint64_t)dim;
  mf_status st = MF_OK;
  if (forward_bytes) st = recur_work(type, batch, time, dim, false, forward_bytes);
  if (st == MF_OK && backward_bytes) st = recur_work(type, batch, time, dim, true, backward_bytes);
  return st;
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_recurrence_forward(const mf_recurrence_args* p, void* d_work, uint64_t work_bytes, void* stream) try {
  const char* me = "mf_recurrence_forward";
  if (!p) return refuse(me, "arguments are NULL");
  std::string bad = check_sizes(p->type, p->batch, p->time, p->dim);
  if (bad.empty()) bad = check_seq(p->x, "x", p->type, p->batch, p->time, p->dim, false);
  if (bad.empty()) bad = check_seq(p->z, "z", p->type, p->batch, p->time, p->dim, false);
  if (bad.empty()) bad = check_seq(p->h, "h", p->type, p->batch, p->time, p->dim, true);
  if (bad.empty()) bad = check_marks(p->d_marks, p->marks_stride_batch, p->marks_stride_time, p->batch, p->time);
  if (bad.empty() && !(aligned(p->d_h0, 4) && aligned(p->d_last, 4) && aligned(p->d_saved, 4) && aligned(p->d_status, 4)))
    bad = "a pointer is not aligned to its type";
  if (!bad.empty()) return refuse(me, bad);
  uint64_t need = 0;
  const mf_status st = recur_work(p->type, p->batch, p->time, p->dim, false, &need);
  if (st != MF_OK) return st;
  bad = check_work(d_work, work_bytes, need);
  if (!bad.empty()) return refuse(me, bad);
  if (!p->batch || !p->dim) return MF_OK;
  return recur_forward(*p, d_work, t_wait_test, (cudaStream_t)stream);
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_recurrence_backward(const mf_recurrence_grad_args* p, void* d_work, uint64_t work_bytes, void* stream) try {
  const char* me = "mf_recurrence_backward";
  if (!p) return refuse(me, "arguments are NULL");
  std::string bad = check_sizes(p->type, p->batch, p->time, p->dim);
  const struct { const mf_seq* t; const char* name; bool out; } seqs[5] = {
      {&p->x, "x", false}, {&p->z, "z", false}, {&p->dh, "dh", false}, {&p->dx, "dx", true}, {&p->dz, "dz", true}};
  for (const auto& q : seqs)
    if (bad.empty()) bad = check_seq(*q.t, q.name, p->type, p->batch, p->time, p->dim, q.out);
  if (bad.empty()) bad = check_marks(p->d_marks, p->marks_stride_batch, p->marks_stride_time, p->batch, p->time);
  if (bad.empty() && p->batch && p->time && p->dim && !p->d_saved) bad = "d_saved is NULL";
  if (bad.empty() && !(aligned(p->d_saved, 4) && aligned(p->d_dlast, 4) && aligned(p->d_dh0, 4) && aligned(p->d_status, 4)))
    bad = "a pointer is not aligned to its type";
  if (!bad.empty()) return refuse(me, bad);
  uint64_t need = 0;
  const mf_status st = recur_work(p->type, p->batch, p->time, p->dim, true, &need);
  if (st != MF_OK) return st;
  bad = check_work(d_work, work_bytes, need);
  if (!bad.empty()) return refuse(me, bad);
  if (!p->batch || !p->dim) return MF_OK;
  return recur_backward(*p, d_work, t_wait_test, (cudaStream_t)stream);
} catch (...) {
  return MF_ENOMEM;
}

// The arguments that a workspace depends on and the polynomial; "" if they are fine.
static std::string check_orth(const mf_orthogonalize_args* p) {
  if (!known_type(p->type)) return "unknown type";
  if (p->batch < 0 || p->rows < 0 || p->cols < 0) return "a size is negative";
  if (p->batch > kMaxSize || p->rows > (1 << 20) || p->cols > (1 << 20)) return "a size is too large";
  if (p->rows && p->cols && p->batch > kMaxStride / 64 / (p->rows * p->cols)) return "the batch is too large";
  if (p->steps < 0 || p->steps > MF_ORTH_MAX_STEPS) return "steps must be in 0..32";
  if (!std::isfinite(p->a) || !std::isfinite(p->b) || !std::isfinite(p->c)) return "a, b and c must be finite";
  if (!std::isfinite(p->eps) || p->eps < 0.f) return "eps must be finite and not negative";
  double top = 1.0;  // of the singular values
  for (int s = 0; s < p->steps; ++s) {
    top = orth_largest(*p, top);
    if (!(top <= 4.0)) return "these coefficients let singular values grow past 4";
  }
  return "";
}

mf_status mf_orthogonalize_workspace(const mf_orthogonalize_args* p, uint64_t* bytes) try {
  const char* me = "mf_orthogonalize_workspace";
  if (!p || !bytes) return refuse(me, "NULL argument");
  const std::string bad = check_orth(p);
  if (!bad.empty()) return refuse(me, bad);
  *bytes = 0;
  if (!p->batch || !p->rows || !p->cols) return MF_OK;
  return orth_work(*p, bytes);
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_orthogonalize(const mf_orthogonalize_args* p, void* d_work, uint64_t work_bytes, void* stream) try {
  const char* me = "mf_orthogonalize";
  if (!p) return refuse(me, "arguments are NULL");
  std::string bad = check_orth(p);
  if (!bad.empty()) return refuse(me, bad);
  if (!p->batch || !p->rows || !p->cols) return MF_OK;
  const int size = type_size(p->type);
  if (!p->d_g || !p->d_out) return refuse(me, "a required pointer is NULL");
  if (!aligned(p->d_g, size) || !aligned(p->d_out, size) || !aligned(p->d_status, 4))
    return refuse(me, "a pointer is not aligned to its type");
  if (p->g_stride_batch < 0 || p->g_stride_row < 0 || p->g_stride_batch > kMaxStride / p->batch ||
      p->g_stride_row > kMaxStride / p->rows || p->out_stride_batch < 0 || p->out_stride_row < 0 ||
      p->out_stride_batch > kMaxStride / p->batch || p->out_stride_row > kMaxStride / p->rows)
    return refuse(me, "a stride is out of range");
  if (!apart(p->rows, p->out_stride_row, p->batch, p->out_stride_batch, p->cols)) return refuse(me, "out overlaps itself");
  uint64_t need = 0;
  const mf_status st = orth_work(*p, &need);
  if (st != MF_OK) return st;
  bad = check_work(d_work, work_bytes, need);
  if (!bad.empty()) return refuse(me, bad);
  return orth_run(*p, d_work, t_wait_test, (cudaStream_t)stream);
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_operators_status(uint32_t** d_word) try {
  if (!d_word) return refuse("mf_operators_status", "NULL argument");
  // (the lookup may load the module, which a stream capture of this thread would forbid although it takes no part in it)
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
  MF_CUDA(cudaThreadExchangeStreamCaptureMode(&mode));
  const cudaError_t e = cudaGetSymbolAddress((void**)d_word, g_operators_status);
  MF_CUDA(cudaThreadExchangeStreamCaptureMode(&mode));
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "cudaGetSymbolAddress");
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_debug_operators_wait_test(uint32_t polls) {
  t_wait_test = polls < 4096 ? polls : 4096;
  return MF_OK;
}

}  // extern "C"
