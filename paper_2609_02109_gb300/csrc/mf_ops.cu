// C ABI of the training operators: argument checks, then the kernels' host sides.  Messages allocate, so each entry
// point ends exceptions in MF_ENOMEM.
#include <algorithm>
#include <cmath>
#include <string>
#include <vector>

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

// The same of three axes.
bool apart(int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t n3, int64_t s3, int64_t width) {
  std::pair<int64_t, int64_t> axis[3] = {{s1, n1}, {s2, n2}, {s3, n3}};
  std::sort(axis, axis + 3);
  for (const auto& a : axis) {
    if (a.second <= 1) continue;
    if (a.first < width) return false;
    width += (a.second - 1) * a.first;
  }
  return true;
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

std::string check_heads(const mf_heads& t, const char* name, int32_t type, int64_t batch, int64_t time, int64_t heads, int64_t dim,
                        bool out) {
  if (!batch || !time || !heads || !dim) return "";
  if (!t.d_ptr) return std::string(name) + " is NULL";
  if (!aligned(t.d_ptr, type_size(type))) return std::string(name) + " is not aligned to its type";
  if (t.stride_batch < 0 || t.stride_time < 0 || t.stride_head < 0 || t.stride_batch > kMaxStride / batch ||
      t.stride_time > kMaxStride / time || t.stride_head > kMaxStride / heads)
    return std::string(name) + ": a stride is out of range";
  if (out && !apart(batch, t.stride_batch, time, t.stride_time, heads, t.stride_head, dim)) return std::string(name) + " overlaps itself";
  return "";
}

std::string check_attend_sizes(int32_t type, int64_t batch, int64_t time, int64_t heads, int64_t dk, int64_t dv) {
  if (!known_type(type)) return "unknown type";
  if (batch < 0 || time < 0 || heads < 0 || dk < 0 || dv < 0) return "a size is negative";
  if (batch > kMaxSize || time > kMaxSize || heads > kMaxSize) return "a size is 2^31 or more";
  if (dk > MF_ATTEND_MAX_DIM || dv > MF_ATTEND_MAX_DIM) return "dim_k and dim_v must be at most " + std::to_string(MF_ATTEND_MAX_DIM);
  if (heads && batch > kMaxSize / heads) return "batch * heads is too large";
  return "";
}

// One of the rows axes: [rows][dim] with a stride.
std::string check_rows(const void* p, const char* name, int32_t type, int64_t rows, int64_t dim, int64_t stride, bool out) {
  if (!rows || !dim) return "";
  if (!p) return std::string(name) + " is NULL";
  if (!aligned(p, type_size(type))) return std::string(name) + " is not aligned to its type";
  if (stride < 0 || stride > kMaxStride / rows) return std::string(name) + ": a stride is out of range";
  if (out && rows > 1 && stride < dim) return std::string(name) + " overlaps itself";
  return "";
}

std::string check_embed(int32_t type, int32_t id_bits, int64_t rows, int64_t dim, int64_t tokens, const void* ids, float scale,
                        const void* status) {
  if (!known_type(type)) return "unknown type";
  if (id_bits != 32 && id_bits != 64) return "id_bits must be 32 or 64";
  if (rows < 0 || dim < 0 || tokens < 0) return "a size is negative";
  if (rows > kMaxSize || dim > kMaxSize || tokens > kMaxSize) return "a size is 2^31 or more";
  if (dim && (rows > (kMaxStride >> 16) / dim || tokens > (kMaxStride >> 16) / dim)) return "rows * dim or tokens * dim is too large";
  if (!std::isfinite(scale)) return "scale must be finite";
  if (tokens && dim && !ids) return "ids is NULL";
  if (!aligned(ids, id_bits / 8) || !aligned(status, 4)) return "a pointer is not aligned to its type";
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

mf_status mf_linear_attention_sizes(int32_t type, int64_t batch, int64_t time, int64_t heads, int64_t dim_k, int64_t dim_v,
                                    uint64_t* saved_floats, uint64_t* forward_bytes, uint64_t* backward_bytes) try {
  const std::string bad = check_attend_sizes(type, batch, time, heads, dim_k, dim_v);
  if (!bad.empty()) return refuse("mf_linear_attention_sizes", bad);
  return attend_sizes(type, batch, time, heads, dim_k, dim_v, saved_floats, forward_bytes, backward_bytes);
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_linear_attention_forward(const mf_linear_attention_args* p, void* d_work, uint64_t work_bytes, void* stream) try {
  const char* me = "mf_linear_attention_forward";
  if (!p) return refuse(me, "arguments are NULL");
  std::string bad = check_attend_sizes(p->type, p->batch, p->time, p->heads, p->dim_k, p->dim_v);
  const struct { const mf_heads* t; const char* name; int64_t dim; bool out; } seqs[4] = {
      {&p->q, "q", p->dim_k, false}, {&p->k, "k", p->dim_k, false}, {&p->v, "v", p->dim_v, false}, {&p->o, "o", p->dim_v, true}};
  for (const auto& q : seqs)
    if (bad.empty()) bad = check_heads(*q.t, q.name, p->type, p->batch, p->time, p->heads, q.dim, q.out);
  if (bad.empty()) bad = check_marks(p->d_marks, p->marks_stride_batch, p->marks_stride_time, p->batch, p->time);
  if (bad.empty() && !std::isfinite(p->scale)) bad = "scale must be finite";
  if (bad.empty() && p->batch && p->heads && !p->d_log_decay) bad = "log_decay is NULL";
  if (bad.empty() && !(aligned(p->d_log_decay, 4) && aligned(p->d_state, 4) && aligned(p->d_last, 4) && aligned(p->d_saved, 4) &&
                       aligned(p->d_status, 4)))
    bad = "a pointer is not aligned to its type";
  if (!bad.empty()) return refuse(me, bad);
  if (!p->batch || !p->heads) return MF_OK;
  uint64_t need = 0;
  const mf_status st = attend_sizes(p->type, p->batch, p->time, p->heads, p->dim_k, p->dim_v, nullptr, &need, nullptr);
  if (st != MF_OK) return st;
  bad = check_work(d_work, work_bytes, need);
  if (!bad.empty()) return refuse(me, bad);
  return attend_forward(*p, d_work, t_wait_test, (cudaStream_t)stream);
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_linear_attention_backward(const mf_linear_attention_grad_args* p, void* d_work, uint64_t work_bytes, void* stream) try {
  const char* me = "mf_linear_attention_backward";
  if (!p) return refuse(me, "arguments are NULL");
  std::string bad = check_attend_sizes(p->type, p->batch, p->time, p->heads, p->dim_k, p->dim_v);
  const struct { const mf_heads* t; const char* name; int64_t dim; bool out; } seqs[7] = {
      {&p->q, "q", p->dim_k, false},     {&p->k, "k", p->dim_k, false}, {&p->v, "v", p->dim_v, false},
      {&p->dout, "dout", p->dim_v, false}, {&p->dq, "dq", p->dim_k, true}, {&p->dk, "dk", p->dim_k, true},
      {&p->dv, "dv", p->dim_v, true}};
  for (const auto& q : seqs)
    if (bad.empty()) bad = check_heads(*q.t, q.name, p->type, p->batch, p->time, p->heads, q.dim, q.out);
  if (bad.empty()) bad = check_marks(p->d_marks, p->marks_stride_batch, p->marks_stride_time, p->batch, p->time);
  if (bad.empty() && !std::isfinite(p->scale)) bad = "scale must be finite";
  if (bad.empty() && p->batch && p->heads && !p->d_log_decay) bad = "log_decay is NULL";
  if (bad.empty() && p->batch && p->heads && p->dim_k && p->dim_v && !p->d_saved) bad = "d_saved is NULL";
  if (bad.empty() && !(aligned(p->d_log_decay, 4) && aligned(p->d_saved, 4) && aligned(p->d_dlast, 4) && aligned(p->d_dstate, 4) &&
                       aligned(p->d_status, 4)))
    bad = "a pointer is not aligned to its type";
  if (!bad.empty()) return refuse(me, bad);
  if (!p->batch || !p->heads) return MF_OK;
  uint64_t need = 0;
  const mf_status st = attend_sizes(p->type, p->batch, p->time, p->heads, p->dim_k, p->dim_v, nullptr, nullptr, &need);
  if (st != MF_OK) return st;
  bad = check_work(d_work, work_bytes, need);
  if (!bad.empty()) return refuse(me, bad);
  return attend_backward(*p, d_work, t_wait_test, (cudaStream_t)stream);
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_embedding_forward(const mf_embedding_args* p, void* stream) try {
  const char* me = "mf_embedding_forward";
  if (!p) return refuse(me, "arguments are NULL");
  std::string bad = check_embed(p->type, p->id_bits, p->rows, p->dim, p->tokens, p->d_ids, p->scale, p->d_status);
  if (bad.empty()) bad = check_rows(p->d_table, "table", p->type, p->tokens ? p->rows : 0, p->dim, p->table_stride, false);
  if (bad.empty()) bad = check_rows(p->d_out, "out", p->type, p->tokens, p->dim, p->out_stride, true);
  if (!bad.empty()) return refuse(me, bad);
  if (!p->tokens || !p->dim) return MF_OK;
  return embed_forward(*p, (cudaStream_t)stream);
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_embedding_workspace(const mf_embedding_grad_args* p, uint64_t* bytes) try {
  const char* me = "mf_embedding_workspace";
  if (!p || !bytes) return refuse(me, "NULL argument");
  const std::string bad = check_embed(p->type, p->id_bits, p->rows, p->dim, 0, nullptr, p->scale, nullptr);
  if (!bad.empty()) return refuse(me, bad);
  if (p->tokens < 0 || p->tokens > kMaxSize || (p->dim && p->tokens > (kMaxStride >> 16) / p->dim))
    return refuse(me, "tokens is out of range");
  *bytes = p->rows && p->dim ? embed_work(*p) : 0;
  return MF_OK;
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_embedding_backward(const mf_embedding_grad_args* p, void* d_work, uint64_t work_bytes, void* stream) try {
  const char* me = "mf_embedding_backward";
  if (!p) return refuse(me, "arguments are NULL");
  std::string bad = check_embed(p->type, p->id_bits, p->rows, p->dim, p->tokens, p->d_ids, p->scale, p->d_status);
  if (bad.empty()) bad = check_rows(p->d_dout, "dout", p->type, p->rows ? p->tokens : 0, p->dim, p->dout_stride, false);
  if (bad.empty()) bad = check_rows(p->d_dtable, "dtable", p->type, p->rows, p->dim, p->dtable_stride, true);
  if (!bad.empty()) return refuse(me, bad);
  if (!p->rows || !p->dim) return MF_OK;
  bad = check_work(d_work, work_bytes, embed_work(*p));
  if (!bad.empty()) return refuse(me, bad);
  return embed_backward(*p, d_work, (cudaStream_t)stream);
} catch (...) {
  return MF_ENOMEM;
}

// Whether an output meets another tensor's memory; a tensor's own input may be its output.
static bool clip_overlaps(const mf_clip_args* p) {
  struct Range {
    uintptr_t lo, hi;
    bool out;
  };
  std::vector<Range> r;
  r.reserve((size_t)p->count);
  bool sorted = true;
  for (int64_t i = 0; i < p->count; ++i) {
    if (!p->sizes[i]) continue;
    const uintptr_t bytes = (uintptr_t)p->sizes[i] * (uintptr_t)type_size(p->types[i]);
    const uintptr_t o = (uintptr_t)p->d_out[i], in = (uintptr_t)p->d_in[i];
    sorted = sorted && (r.empty() || r.back().hi <= o);
    r.push_back({o, o + bytes, true});
    if (in != o) {
      sorted = sorted && r.back().hi <= in;
      r.push_back({in, in + bytes, false});
    }
  }
  if (sorted) return false;
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
  uintptr_t any = 0, out = 0;  // the ends of all ranges, and of the outputs', so far
  for (const Range& a : r) {
    if (a.lo < (a.out ? any : out)) return true;
    any = std::max(any, a.hi);
    if (a.out) out = std::max(out, a.hi);
  }
  return false;
}

static std::string check_clip(const mf_clip_args* p) {
  if (p->count < 0 || p->count > kMaxSize) return "count is out of range";
  if (p->count && (!p->sizes || !p->types)) return "sizes or types is NULL";
  constexpr int64_t most = int64_t(1) << 40;
  int64_t all = 0;
  for (int64_t i = 0; i < p->count; ++i) {
    if (!known_type(p->types[i])) return "unknown type";
    if (p->sizes[i] < 0 || p->sizes[i] >= most) return "a size is out of range";
    all += p->sizes[i];
    if (all >= most) return "the tensors are too large together";
  }
  return "";
}

mf_status mf_clip_workspace(const mf_clip_args* p, uint64_t* bytes) try {
  const char* me = "mf_clip_workspace";
  if (!p || !bytes) return refuse(me, "NULL argument");
  const std::string bad = check_clip(p);
  if (!bad.empty()) return refuse(me, bad);
  *bytes = clip_work(*p);
  return MF_OK;
} catch (...) {
  return MF_ENOMEM;
}

mf_status mf_clip_gradients(const mf_clip_args* p, void* d_work, uint64_t work_bytes, void* stream) try {
  const char* me = "mf_clip_gradients";
  if (!p) return refuse(me, "arguments are NULL");
  std::string bad = check_clip(p);
  if (bad.empty() && p->count && (!p->d_in || !p->d_out)) bad = "d_in or d_out is NULL";
  if (bad.empty() && !(p->max_norm >= 0.f)) bad = "max_norm must not be negative or NaN";
  if (bad.empty() && !(std::isfinite(p->eps) && p->eps >= 0.f)) bad = "eps must be finite and not negative";
  if (bad.empty() && !aligned(p->d_norm, 4)) bad = "a pointer is not aligned to its type";
  for (int64_t i = 0; bad.empty() && i < p->count; ++i) {
    if (!p->sizes[i]) continue;
    if (!p->d_in[i] || !p->d_out[i]) bad = "a tensor is NULL";
    else if (!aligned(p->d_in[i], type_size(p->types[i])) || !aligned(p->d_out[i], type_size(p->types[i])))
      bad = "a tensor is not aligned to its type";
  }
  if (bad.empty() && clip_overlaps(p)) bad = "an output overlaps another tensor";
  if (bad.empty()) bad = check_work(d_work, work_bytes, clip_work(*p));
  if (!bad.empty()) return refuse(me, bad);
  return clip_run(*p, d_work, (cudaStream_t)stream);
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
