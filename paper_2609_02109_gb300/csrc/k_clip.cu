// The norm of many tensors together, and the tensors scaled so that it stays within a bound (the operators' section of
// include/mf.h).
//
// Bound by memory: every value is read for the norm, and read again and written where it is scaled.  Tensors come as
// descriptors in the launches' arguments (no copy that a captured call would have to keep alive), kGroup a launch, cut
// into chunks; a block sums the chunks b, b + blocks, ..., so that equal calls add in an equal order.  Each block of the
// second launch adds all blocks' sums up by itself, in order, and scales its chunks from the last to the first: what was
// read last is in L2 still.  Few values are one launch: a cluster of blocks that exchange their sums.
//
// Measured on 24 bf16 tensors of 381 M values (763 MB read, then read and written): squares 125 us (6.1 TB/s; with the
// ranges of squares.cuh for every value 216), scaling 260 (5.9 TB/s), 411 a call.  Holding what fits on chip between the
// passes (30 MB of shared memory and the L2) would save about a tenth.
#include <algorithm>
#include <cmath>
#include <vector>

#include <cooperative_groups.h>

#include "mf_ops.cuh"
#include "squares.cuh"

namespace mf {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kChunk = 16384;  // values
constexpr int kGroup = 1000;                   // descriptors of a launch (32 bytes each, of 32764 bytes of arguments)

struct Tensor {
  const void* in;
  void* out;
  int64_t n;
  uint32_t type, first;  // first: chunks of the launch's tensors before
};
template <int N>
struct Group {
  int count, chunks;
  float max_norm, eps;
  Squares* part;   // of this launch's blocks
  int parts;       // of all launches' blocks
  float* norm;
  Tensor t[N];
};
using Many = Group<kGroup>;
static_assert(sizeof(Many) <= 32700, "a launch's arguments");
// A call of so few chunks and values is one launch of one cluster.
constexpr int kFew = 8, kFewChunks = 128;
constexpr int64_t kFewValues = 524288;
using Few = Group<kFewChunks>;

// Where a tensor's values [lo, hi) lie: up to `head` before the first 16-byte boundary, then whole vectors to `tail`.
template <typename T>
__device__ __forceinline__ void cut(const T* p, int64_t lo, int64_t hi, int64_t* head, int64_t* tail) {
  constexpr int kPer = 16 / sizeof(T);
  const int64_t off = (int64_t)(((uintptr_t)(p + lo) & 15) / sizeof(T));
  *head = min(hi, off ? lo + kPer - off : lo);
  *tail = *head + (hi - *head) / kPer * kPer;
}

// Squares in plain fp32, and the largest magnitude: three instructions a value.
struct Plain {
  float sum[4] = {}, top = 0.f;
  template <typename T>
  __device__ __forceinline__ void add(const uint4& w) {
    const T* v = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int k = 0; k < (int)(16 / sizeof(T)); ++k) {
      const float f = to_f32(v[k]);
      top = fmaxf(top, fabsf(f));
      sum[k & 3] = fmaf(f, f, sum[k & 3]);
    }
  }
  // Whether the sum is one of squares.cuh's middle range: no value passes it, so no sum of 2^40 squares overflows, and
  // what underflowed (below 2^-62 each, at most 2^10 values) is below 2^-34 of it.
  __device__ __forceinline__ bool fine() const { return top <= 0x1p40f && (top > 0x1p-40f || top == 0.f) && total() < 0x1p120f; }
  __device__ __forceinline__ float total() const { return (sum[0] + sum[1]) + (sum[2] + sum[3]); }
};

// The squares of values [lo, hi), over the block's threads.
template <typename T>
__device__ __forceinline__ void add_squares(const T* p, int64_t lo, int64_t hi, Squares& q) {
  int64_t head, tail;
  cut(p, lo, hi, &head, &tail);
  const uint4* const v = reinterpret_cast<const uint4*>(p + head);
  const int vectors = (int)((tail - head) * sizeof(T) / 16);
  Plain plain;
  int i = threadIdx.x;
  for (; i + 3 * (int)blockDim.x < vectors; i += 4 * blockDim.x) {
    uint4 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = v[i + j * blockDim.x];
#pragma unroll
    for (int j = 0; j < 4; ++j) plain.add<T>(w[j]);
  }
  for (; i < vectors; i += blockDim.x) plain.add<T>(v[i]);
  if (plain.fine()) {
    q.mid += plain.total();
  } else {  // (very small or large values, infinities, NaN: once more, in ranges)
#pragma unroll 1
    for (i = threadIdx.x; i < vectors; i += blockDim.x) {
      const uint4 w = v[i];
      const T* const u = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int k = 0; k < (int)(16 / sizeof(T)); ++k) q.add(to_f32(u[k]));
    }
  }
  for (int64_t k = lo + threadIdx.x; k < head; k += blockDim.x) q.add(to_f32(p[k]));
  for (int64_t k = tail + threadIdx.x; k < hi; k += blockDim.x) q.add(to_f32(p[k]));
}

template <typename T>
__device__ __forceinline__ uint4 scaled(const uint4& w, float f) {
  uint4 r;
  const T* v = reinterpret_cast<const T*>(&w);
  T* o = reinterpret_cast<T*>(&r);
#pragma unroll
  for (int k = 0; k < (int)(16 / sizeof(T)); ++k) o[k] = from_f32<T>(to_f32(v[k]) * f);
  return r;
}

template <typename T>
__device__ __forceinline__ void scale_values(const T* in, T* out, int64_t lo, int64_t hi, float f) {
  if (((uintptr_t)in ^ (uintptr_t)out) & 15) {  // vectors of one would not be vectors of the other
    for (int64_t k = lo + threadIdx.x; k < hi; k += blockDim.x) out[k] = from_f32<T>(to_f32(in[k]) * f);
    return;
  }
  int64_t head, tail;
  cut(in, lo, hi, &head, &tail);
  const uint4* const v = reinterpret_cast<const uint4*>(in + head);
  uint4* const o = reinterpret_cast<uint4*>(out + head);
  const int vectors = (int)((tail - head) * sizeof(T) / 16);
  int i = threadIdx.x;
  for (; i + 3 * (int)blockDim.x < vectors; i += 4 * blockDim.x) {
    uint4 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = v[i + j * blockDim.x];
#pragma unroll
    for (int j = 0; j < 4; ++j) o[i + j * blockDim.x] = scaled<T>(w[j], f);
  }
  for (; i < vectors; i += blockDim.x) o[i] = scaled<T>(v[i], f);
  for (int64_t k = lo + threadIdx.x; k < head; k += blockDim.x) out[k] = from_f32<T>(to_f32(in[k]) * f);
  for (int64_t k = tail + threadIdx.x; k < hi; k += blockDim.x) out[k] = from_f32<T>(to_f32(in[k]) * f);
}

__device__ __forceinline__ void add_any(const Tensor& t, int64_t lo, int64_t hi, Squares& q) {
  if (t.type == MF_TYPE_F32) add_squares((const float*)t.in, lo, hi, q);
  else if (t.type == MF_TYPE_BF16) add_squares((const __nv_bfloat16*)t.in, lo, hi, q);
  else add_squares((const __half*)t.in, lo, hi, q);
}
__device__ __forceinline__ void scale_any(const Tensor& t, int64_t lo, int64_t hi, float f) {
  if (t.type == MF_TYPE_F32) scale_values((const float*)t.in, (float*)t.out, lo, hi, f);
  else if (t.type == MF_TYPE_BF16) scale_values((const __nv_bfloat16*)t.in, (__nv_bfloat16*)t.out, lo, hi, f);
  else scale_values((const __half*)t.in, (__half*)t.out, lo, hi, f);
}

// The tensor that holds the launch's chunk c: the last whose first chunk is not behind it.  (Empty ones have no chunk.)
template <int N>
__device__ __forceinline__ const Tensor& tensor_of(const Group<N>& g, int c) {
  int lo = 0, hi = g.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if ((int)g.t[mid].first <= c) lo = mid;
    else hi = mid;
  }
  return g.t[lo];
}

// The norm is finite where all values are and it is a float32: then the factor is min(1, max_norm / (norm + eps)), else 1.
__device__ __forceinline__ float factor_of(float norm, float max_norm, float eps) {
  const float f = max_norm / (norm + eps);
  return isfinite(norm) && f < 1.f ? f : 1.f;
}

__global__ void __launch_bounds__(kThreads) k_clip_squares(const __grid_constant__ Many g) {
  __shared__ Squares s_part[kThreads / 32];
  Squares q;
  for (int c = blockIdx.x; c < g.chunks; c += gridDim.x) {
    const Tensor& t = tensor_of(g, c);
    const int64_t lo = (int64_t)(c - (int)t.first) * kChunk;
    Squares chunk;  // (sums of sums: a long one would lose bits)
    add_any(t, lo, min(t.n, lo + kChunk), chunk);
    q.add(chunk);
  }
  q = block_sum(q, s_part);
  if (threadIdx.x == 0) g.part[blockIdx.x] = q;
}

// (g.part: all launches' sums.)
__global__ void __launch_bounds__(kThreads) k_clip_scale(const __grid_constant__ Many g) {
  __shared__ Squares s_part[kThreads / 32];
  __shared__ float s_factor;
  Squares q;
#pragma unroll 4
  for (int i = threadIdx.x; i < g.parts; i += kThreads) q.add(g.part[i]);
  q = block_sum(q, s_part);
  if (threadIdx.x == 0) {
    const float norm = norm_of(q);
    s_factor = factor_of(norm, g.max_norm, g.eps);
    if (blockIdx.x == 0 && g.norm) *g.norm = norm;
  }
  __syncthreads();
  const float f = s_factor;
  for (int c = g.chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
    const Tensor& t = tensor_of(g, c);
    if (f == 1.f && t.in == t.out) continue;
    const int64_t lo = (int64_t)(c - (int)t.first) * kChunk;
    scale_any(t, lo, min(t.n, lo + kChunk), f);
  }
}

__global__ void __launch_bounds__(kThreads) k_clip_few(const __grid_constant__ Few g) {
  __shared__ Squares s_part[kThreads / 32], s_block;
  __shared__ float s_factor;
  const cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank();
  Squares q;
  for (int c = rank; c < g.chunks; c += kFew) {
    const Tensor& t = tensor_of(g, c);
    const int64_t lo = (int64_t)(c - (int)t.first) * kChunk;
    add_any(t, lo, min(t.n, lo + kChunk), q);
  }
  q = block_sum(q, s_part);
  if (threadIdx.x == 0) s_block = q;
  cluster.sync();
  if (threadIdx.x == 0) {
    q = Squares{};
    for (int r = 0; r < kFew; ++r) q.add(*cluster.map_shared_rank(&s_block, r));
    const float norm = norm_of(q);
    s_factor = factor_of(norm, g.max_norm, g.eps);
    if (rank == 0 && g.norm) *g.norm = norm;
  }
  cluster.sync();
  const float f = s_factor;
  for (int c = rank; c < g.chunks; c += kFew) {
    const Tensor& t = tensor_of(g, c);
    if (f == 1.f && t.in == t.out) continue;
    const int64_t lo = (int64_t)(c - (int)t.first) * kChunk;
    scale_any(t, lo, min(t.n, lo + kChunk), f);
  }
}

// Blocks of a launch: four an SM, all its threads, with four loads of 16 bytes in flight each.
int blocks_of(int chunks) { return std::min(chunks, 152 * 4); }

// The tensors from `at` on that a launch takes; at moves behind them.
template <int N>
void take_group(const mf_clip_args& p, int64_t* at, Group<N>* g) {
  g->count = 0;
  int64_t chunks = 0;
  for (; *at < p.count && g->count < N; ++*at) {
    const int64_t n = p.sizes[*at], c = (n + kChunk - 1) / kChunk;
    if (!n) continue;
    if (chunks + c > 0x3FFFFFFF) break;
    g->t[g->count++] = {p.d_in[*at], p.d_out[*at], n, (uint32_t)p.types[*at], (uint32_t)chunks};
    chunks += c;
  }
  g->chunks = (int)chunks;
}

}  // namespace

// Launches' blocks in all, for p.sizes.
int64_t clip_parts(const mf_clip_args& p) {
  int64_t parts = 0, at = 0;
  while (at < p.count) {
    int64_t chunks = 0;
    for (int n = 0; at < p.count && n < kGroup; ++at) {
      const int64_t c = (p.sizes[at] + kChunk - 1) / kChunk;
      if (!c) continue;
      if (chunks + c > 0x3FFFFFFF) break;
      chunks += c;
      ++n;
    }
    parts += blocks_of((int)chunks);
  }
  return parts;
}
// Whether a call is one cluster's: so few values take longer to launch than to read.
bool clip_few(const mf_clip_args& p) {
  int64_t values = 0, chunks = 0;
  for (int64_t i = 0; i < p.count; ++i) {
    values += p.sizes[i];
    chunks += (p.sizes[i] + kChunk - 1) / kChunk;
    if (values > kFewValues || chunks > kFewChunks) return false;
  }
  return true;
}
uint64_t clip_work(const mf_clip_args& p) { return clip_few(p) ? 0 : (uint64_t)clip_parts(p) * sizeof(Squares); }

mf_status clip_run(const mf_clip_args& p, void* work, cudaStream_t s) {
  int64_t at = 0;
  if (clip_few(p)) {
    Few g;
    g.max_norm = p.max_norm;
    g.eps = p.eps;
    g.norm = p.d_norm;
    take_group(p, &at, &g);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(kFew);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = kFew;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    MF_CUDA(cudaLaunchKernelEx(&cfg, k_clip_few, g));
    return MF_OK;
  }
  Many g;
  g.max_norm = p.max_norm;
  g.eps = p.eps;
  g.norm = p.d_norm;
  g.part = (Squares*)work;
  g.parts = (int)clip_parts(p);
  std::vector<int64_t> starts;  // the launches' first tensors
  while (at < p.count) {
    const int64_t here = at;
    take_group(p, &at, &g);
    if (!g.count) break;  // (only empty tensors were left)
    const int blocks = blocks_of(g.chunks);
    k_clip_squares<<<blocks, kThreads, 0, s>>>(g);
    MF_CUDA(cudaGetLastError());
    g.part += blocks;
    starts.push_back(here);
  }
  g.part = (Squares*)work;
  // the last launch's tensors first: they were read last
  for (size_t k = starts.size(); k-- > 0;) {
    at = starts[k];
    take_group(p, &at, &g);
    k_clip_scale<<<blocks_of(g.chunks), kThreads, 0, s>>>(g);
    MF_CUDA(cudaGetLastError());
    g.norm = nullptr;
  }
  return MF_OK;
}

}  // namespace mf
