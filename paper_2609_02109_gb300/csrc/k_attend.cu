// Linear attention with a decay for each head (the operators' section of include/mf.h; the passes are in attend.cuh): the
// kernel for single tokens, the passes on the CUDA cores, and the host side.
#include <algorithm>

#include "attend.cuh"

namespace mf {
namespace {

// ------------------------------------------------------------------------------------------
// A few steps, one by one
// ------------------------------------------------------------------------------------------

struct FewArgs {
  AttendSeq q, k, v, o;
  const uint8_t* marks;
  int64_t marks_sb, marks_st;
  const float* log_decay;
  const float* state;
  float* last;
  int time, heads, dk, dv;
  float scale;
};

// A block holds a head's state in registers: V columns of a row a thread, in as many row groups as 256 threads make.
// Bound by memory where there are many heads: the state is read and written once, all of a thread's loads in flight.
template <typename T, int V>
__global__ void __launch_bounds__(256) k_attend_few(const FewArgs a) {
  constexpr int kRows = V == 4 ? 16 : 64;
  __shared__ float s_q[128], s_k[128], s_v[128], s_sum[256 * V];
  const int b = blockIdx.x / a.heads, h = blockIdx.x - b * a.heads;
  const int groups = (a.dv + V - 1) / V, per = 256 / groups;  // threads of a row; rows side by side
  const int r0 = threadIdx.x / groups, c = (threadIdx.x - r0 * groups) * V;
  const int64_t at = (int64_t)blockIdx.x * a.dk * a.dv;
  float s[kRows][V];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = r0 + i * per;
#pragma unroll
    for (int k = 0; k < V; ++k) s[i][k] = 0.f;
    if (a.state && r0 < per && r < a.dk) {
      if constexpr (V == 4) *(float4*)s[i] = *(const float4*)(a.state + at + (int64_t)r * a.dv + c);
      else s[i][0] = a.state[at + (int64_t)r * a.dv + c];
    }
  }
  const Remains left(finite_log(a.log_decay[h]), 1.f);
  for (int t = 0; t < a.time; ++t) {
    const int mark = a.marks ? a.marks[b * a.marks_sb + t * a.marks_st] : MF_MARK_SAMPLE;
    if (threadIdx.x < 128) {
      const int i = threadIdx.x;
      const int64_t qo = b * a.q.sb + t * a.q.st + h * a.q.sh, ko = b * a.k.sb + t * a.k.st + h * a.k.sh;
      s_q[i] = i < a.dk ? to_f32(((const T*)a.q.p)[qo + i]) : 0.f;
      s_k[i] = i < a.dk && mark != MF_MARK_MISSING ? to_f32(((const T*)a.k.p)[ko + i]) : 0.f;
    } else {
      const int i = threadIdx.x - 128;
      const int64_t vo = b * a.v.sb + t * a.v.st + h * a.v.sh;
      s_v[i] = i < a.dv && mark != MF_MARK_MISSING ? to_f32(((const T*)a.v.p)[vo + i]) : 0.f;
    }
    __syncthreads();
    float sum[V] = {}, v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = c + k < 128 ? s_v[c + k] : 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = r0 + i * per;
      if (r0 >= per || r >= a.dk) break;
      const float key = s_k[r], query = s_q[r];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (mark == MF_MARK_FIRST) s[i][k] = key * v[k];
        else if (mark != MF_MARK_MISSING) s[i][k] = left(s[i][k], key * v[k]);
        sum[k] = fmaf(query, s[i][k], sum[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) s_sum[threadIdx.x * V + k] = sum[k];
    __syncthreads();
    if (threadIdx.x < a.dv) {
      const int stride = groups * V;  // of a row group's sums
      float total = 0.f;
      for (int g = 0; g < per; ++g) total += s_sum[g * stride + threadIdx.x];
      ((T*)a.o.p)[b * a.o.sb + t * a.o.st + h * a.o.sh + threadIdx.x] = from_f32<T>(total * a.scale);
    }
  }
  if (!a.last) return;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = r0 + i * per;
    if (r0 >= per || r >= a.dk) break;
    if constexpr (V == 4) *(float4*)(a.last + at + (int64_t)r * a.dv + c) = *(const float4*)s[i];
    else a.last[at + (int64_t)r * a.dv + c] = s[i][0];
  }
}

// ------------------------------------------------------------------------------------------
// The passes on the CUDA cores
// ------------------------------------------------------------------------------------------

constexpr int kChunk = 32;
constexpr int kPad = kChunk + 4;

__host__ __device__ inline int up4(int n) { return (n + 3) & ~3; }
// Row strides of x and y: rows one behind the other start four banks apart.
__host__ __device__ inline int stride_x(int dx) {
  const int p = up4(dx);
  return p % 8 ? p : p + 4;
}
__host__ __device__ inline size_t simt_floats(int dx, int dz) {
  const int px = up4(dx), pz = up4(dz);
  return (size_t)2 * kChunk * stride_x(dx) + (size_t)kChunk * pz + (size_t)px * pz + kChunk * kPad;
}
inline int simt_threads(int dx, int dz) {
  const int tiles = up4(dx) / 4 * (up4(dz) / 4);
  return tiles <= 32 ? 32 : tiles <= 96 ? 64 : tiles <= 256 ? 128 : 256;
}

// Rows of a tensor's chunk into shared memory as fp32, zeros outside and where `skip` has a row's bit.  True if a value is
// not finite.
template <typename T>
__device__ __forceinline__ bool load_rows(float* to, int stride, const AttendSeq& q, int64_t base, int64_t lo, int rows, int dim,
                                          uint32_t skip) {
  const int width = up4(dim);
  bool bad = false;
  for (int i = threadIdx.x; i < kChunk * width; i += blockDim.x) {
    const int r = i / width, c = i - r * width;
    float v = 0.f;
    if (r < rows && c < dim && !(skip >> r & 1)) v = to_f32(((const T*)q.p)[base + (lo + r) * q.st + c]);
    bad |= !(fabsf(v) <= 3.4028235e38f);
    to[r * stride + c] = v;
  }
  return bad;
}

// The state's rows k0.., columns c0..: S = what is left of S + sum of alpha w_j y_j z_j, R x R values a thread.  (A step whose
// weight is negative adds nothing, whatever its values.)
template <int R>
__device__ __forceinline__ void update_state(float* s, const float* y, const float* z, const float* w, int px, int pz, int sx,
                                             const Remains& left, float alpha) {
  const int across = (pz + R - 1) / R, tiles = (px + R - 1) / R * across;
  for (int tile = threadIdx.x; tile < tiles; tile += blockDim.x) {
    const int k0 = tile / across * R, c0 = (tile - tile / across * across) * R;
    float acc[R][R] = {};
    for (int j = 0; j < kChunk; ++j) {
      if (w[j] < 0.f) continue;
      const float wj = w[j] * alpha;
      float a[R], b[R];
#pragma unroll
      for (int k = 0; k < R; k += 4) {
        const float4 v = k0 + k < px ? *(const float4*)(y + j * sx + k0 + k) : make_float4(0.f, 0.f, 0.f, 0.f);
        const float4 u = c0 + k < pz ? *(const float4*)(z + j * pz + c0 + k) : make_float4(0.f, 0.f, 0.f, 0.f);
        a[k] = v.x * wj; a[k + 1] = v.y * wj; a[k + 2] = v.z * wj; a[k + 3] = v.w * wj;
        b[k] = u.x; b[k + 1] = u.y; b[k + 2] = u.z; b[k + 3] = u.w;
      }
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int c = 0; c < R; ++c) acc[k][c] = fmaf(a[k], b[c], acc[k][c]);
    }
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int c = 0; c < R; c += 4)
        if (k0 + k < px && c0 + c < pz) {
          float4* const to = (float4*)(s + (k0 + k) * pz + c0 + c);
          const float4 v = *to;
          *to = make_float4(left(v.x, acc[k][c]), left(v.y, acc[k][c + 1]), left(v.z, acc[k][c + 2]), left(v.w, acc[k][c + 3]));
        }
  }
}

// A block: one segment of a head, chunk by chunk, the state in shared memory.  4 x 4 (states: up to 8 x 8) values a thread
// from operands in shared memory; bound by the FMA pipe and shared memory.
template <typename T>
__global__ void __launch_bounds__(256) k_attend_simt(const AttendPass p) {
  extern __shared__ float4 smem4[];
  const int px = up4(p.dx), pz = up4(p.dz), sx = stride_x(p.dx);
  float* const s_x = (float*)smem4;
  float* const s_y = s_x + kChunk * sx;
  float* const s_z = s_y + kChunk * sx;
  float* const s_s = s_z + kChunk * pz;
  float* const s_p = s_s + px * pz;
  __shared__ float s_row[kChunk], s_src[kChunk], s_samples;
  __shared__ int s_seen[kChunk], s_trace[kChunk];
  __shared__ uint32_t s_missing;
  const bool states = p.local != nullptr;
  const int segs = states ? p.segs - 1 : p.segs;
  const int64_t row = blockIdx.x / segs;
  const int seg = (int)(blockIdx.x - row * segs) + (states && p.reverse ? 1 : 0);
  const int64_t b = row / p.heads;
  const int h = (int)(row - b * p.heads);
  const float log_decay = finite_log(p.log_decay[h]), l2 = log_decay * kLog2e;
  const int64_t xo = b * p.x.sb + h * p.x.sh, yo = b * p.y.sb + h * p.y.sh, zo = b * p.z.sb + h * p.z.sh,
                oo = b * p.out.sb + h * p.out.sh;

  const float* const from = states || !p.state ? nullptr : p.state + (row * p.state_segs + (p.state_segs > 1 ? seg : 0)) * p.dx * p.dz;
  for (int i = threadIdx.x; i < px * pz; i += blockDim.x) {
    const int k = i / pz, c = i - k * pz;
    float v = 0.f;
    if (from && k < p.dx && c < p.dz) v = from[p.state_t ? c * p.dx + k : k * p.dz + c];
    s_s[i] = v;
    if (p.save && k < p.dx && c < p.dz) p.save[row * p.dx * p.dz + k * p.dz + c] = v;
  }
  float samples = 0.f;
  const int first = seg * p.seg_chunks, end = min(p.chunks, first + p.seg_chunks);
  for (int n = 0; n < end - first; ++n) {
    const int64_t lo = (int64_t)(p.reverse ? end - 1 - n : first + n) * kChunk;
    const int rows = (int)min((int64_t)kChunk, p.time - lo);
    __syncthreads();
    if (threadIdx.x < 32) {
      // samples seen and traces begun, up to and with each step; what is left of the state before the chunk at each
      // step, and of each step behind the chunk (-1: nothing, a trace begins in between)
      const int i = threadIdx.x;
      const int mark = i >= rows ? MF_MARK_MISSING : p.marks ? p.marks[b * p.marks_sb + (lo + i) * p.marks_st] : MF_MARK_SAMPLE;
      const uint32_t missing = __ballot_sync(0xffffffffu, mark == MF_MARK_MISSING);
      const uint32_t begins = __ballot_sync(0xffffffffu, mark == MF_MARK_FIRST), upto = 0xffffffffu >> (31 - i);
      const int seen = __popc(~missing & upto), trace = __popc(begins & upto);
      const int all = __popc(~missing), traces = __popc(begins);
      s_seen[i] = seen;
      s_trace[i] = trace;
      const float head = trace ? -1.f : exp2f(l2 * (float)seen), tail = trace == traces ? exp2f(l2 * (float)(all - seen)) : -1.f;
      s_row[i] = p.reverse ? tail : head;
      s_src[i] = p.reverse ? head : tail;
      if (i == 31) s_samples = trace ? -1.f : (float)seen;
      if (i == 0) s_missing = missing;
    }
    __syncthreads();
    const uint32_t missing = s_missing;
    if (!states) load_rows<T>(s_x, sx, p.x, xo, lo, rows, p.dx, p.reverse ? missing : 0u);
    load_rows<T>(s_y, sx, p.y, yo, lo, rows, p.dx, p.reverse ? 0u : missing);
    bool bad = load_rows<T>(s_z, pz, p.z, zo, lo, rows, p.dz, p.reverse ? 0u : missing);
    bad = __syncthreads_or(bad);
    if (!states) {
      // the products of x and y, and what is left between their steps
      for (int tile = threadIdx.x; tile < 64; tile += blockDim.x) {
        const int i0 = tile >> 3, j0 = tile & 7;
        float acc[4][4] = {};
        for (int k = 0; k < px; k += 4) {
          float4 u[4], v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            u[r] = *(const float4*)(s_x + (i0 + 8 * r) * sx + k);
            v[r] = *(const float4*)(s_y + (j0 + 8 * r) * sx + k);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c)
              acc[r][c] = fmaf(u[r].w, v[c].w, fmaf(u[r].z, v[c].z, fmaf(u[r].y, v[c].y, fmaf(u[r].x, v[c].x, acc[r][c]))));
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int i = i0 + 8 * r, j = j0 + 8 * c;
            const bool sees = (p.reverse ? j >= i : j <= i) && s_trace[i] == s_trace[j];
            s_p[i * kPad + j] = sees ? acc[r][c] * exp2f(l2 * (float)abs(s_seen[i] - s_seen[j])) * p.alpha : 0.f;
          }
      }
      __syncthreads();
      const int across = pz / 4;
      for (int tile = threadIdx.x; tile < 8 * across; tile += blockDim.x) {
        const int i0 = tile / across, c0 = (tile - i0 * across) * 4;
        float acc[4][4] = {};
        for (int k = 0; k < px; k += 4) {
          float4 u[4], v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            u[r] = *(const float4*)(s_x + (i0 + 8 * r) * sx + k);
            v[r] = *(const float4*)(s_s + (k + r) * pz + c0);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float a[4] = {u[r].x, u[r].y, u[r].z, u[r].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              acc[r][0] = fmaf(a[q], v[q].x, acc[r][0]);
              acc[r][1] = fmaf(a[q], v[q].y, acc[r][1]);
              acc[r][2] = fmaf(a[q], v[q].z, acc[r][2]);
              acc[r][3] = fmaf(a[q], v[q].w, acc[r][3]);
            }
          }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float w = s_row[i0 + 8 * r];
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[r][c] = w < 0.f ? 0.f : acc[r][c] * (w * p.alpha_row);
        }
        for (int j = 0; j < kChunk; j += 4) {
          float4 u[4], v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            u[r] = *(const float4*)(s_p + (i0 + 8 * r) * kPad + j);
            v[r] = *(const float4*)(s_z + (j + r) * pz + c0);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = i0 + 8 * r;
            const float a[4] = {u[r].x, u[r].y, u[r].z, u[r].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              // (no product with what a row does not see where a value is infinite or NaN)
              if (bad && ((p.reverse ? j + q < i : j + q > i) || s_trace[i] != s_trace[j + q])) continue;
              acc[r][0] = fmaf(a[q], v[q].x, acc[r][0]);
              acc[r][1] = fmaf(a[q], v[q].y, acc[r][1]);
              acc[r][2] = fmaf(a[q], v[q].z, acc[r][2]);
              acc[r][3] = fmaf(a[q], v[q].w, acc[r][3]);
            }
          }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (i0 + 8 * r < rows && c0 + c < p.dz)
              ((T*)p.out.p)[oo + (lo + i0 + 8 * r) * p.out.st + c0 + c] = from_f32<T>(acc[r][c]);
      }
      __syncthreads();
    }
    const Remains left(log_decay, s_samples);
    samples = samples < 0.f || s_samples < 0.f ? -1.f : samples + s_samples;
    if (px > 64 && pz > 64) update_state<8>(s_s, s_y, s_z, s_src, px, pz, sx, left, p.alpha_src);
    else update_state<4>(s_s, s_y, s_z, s_src, px, pz, sx, left, p.alpha_src);
  }
  __syncthreads();
  float* to = nullptr;
  if (states) to = p.local + (row * p.segs + seg) * p.dx * p.dz;
  else if (p.final_state && seg == (p.reverse ? 0 : p.segs - 1)) to = p.final_state + row * p.dx * p.dz;
  if (to)
    for (int i = threadIdx.x; i < p.dx * p.dz; i += blockDim.x) {
      const int k = i / p.dz;
      to[i] = s_s[k * pz + i - k * p.dz];
    }
  if (states && threadIdx.x == 0) p.seen[row * p.segs + seg] = samples;
}

// The segments' own states -> the states that they start from, in place.  A thread: a value of the state.
__global__ void __launch_bounds__(256) k_attend_chain(float* local, const float* seen, const float* state, const float* log_decay,
                                                      int64_t row0, int heads, int segs, int values, bool reverse) {
  const int64_t row = blockIdx.y;
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= values) return;
  float now = state ? state[row * values + i] : 0.f;
  float* const at = local + row * segs * values + i;
  const float* const samples = seen + row * segs;
  const float log = finite_log(log_decay[(row0 + row) % heads]);
#pragma unroll 8
  for (int n = 0; n < segs; ++n) {
    const int seg = reverse ? segs - 1 - n : n;
    float* const here = at + (int64_t)seg * values;
    const bool end = n == segs - 1;  // (the last segment's own state is not needed)
    const float own = end ? 0.f : *here;
    *here = now;
    now = Remains(log, end ? 0.f : samples[seg])(now, own);
  }
}

// ------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------

constexpr int kFew = 8;  // steps that pass one by one

struct Plan {
  bool tc;
  int chunk, chunks, segs, seg_chunks;
};

Plan plan_of(int type, int64_t rows, int64_t time, int dk, int dv) {
  Plan p{};
  p.tc = type != MF_TYPE_F32 && time > kFew && dk && dv;
  p.chunk = p.tc ? kAttendTcChunk : kChunk;
  p.chunks = (int)((time + p.chunk - 1) / p.chunk);
  // Blocks that run at a time, and as many segments as make the longest block's way shortest: a segment's chunks once
  // more for its own state (about half of a chunk's work) where there are several.
  int64_t slots = 152;
  if (!p.tc) {
    const size_t smem = simt_floats(dk, dv) * 4 + 2048;
    slots *= std::min<int64_t>(228 * 1024 / (int64_t)(smem + 1024), std::min(32, 2048 / simt_threads(dk, dv)));
  }
  p.segs = 1;
  double best = 1e300;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(p.chunks, 4 * slots / std::max<int64_t>(rows, 1) + 1));
  for (int64_t n = 1; n <= most; n += 1 + n / 16) {
    const int64_t per = (p.chunks + n - 1) / n, segs = per ? (p.chunks + per - 1) / per : 1;
    const double waves = (double)((rows * segs + slots - 1) / slots);
    const double cost = waves * ((double)per * (segs > 1 ? 1.5 : 1.0) + 1.0) + (segs > 1 ? 2.0 + 0.02 * (double)segs : 0.0);
    if (cost < best * 0.999) {
      best = cost;
      p.segs = (int)segs;
      p.seg_chunks = (int)per;
    }
  }
  if (!p.chunks) p.seg_chunks = 0;
  return p;
}

mf_status run_pass(int type, bool tc, const AttendPass& p, int64_t rows, cudaStream_t s) {
  if (tc) return attend_tc(type, p, rows, s);
  const int64_t blocks = rows * (p.local ? p.segs - 1 : p.segs);
  const size_t smem = simt_floats(p.dx, p.dz) * 4;
  auto kernel = type == MF_TYPE_F32 ? k_attend_simt<float> : type == MF_TYPE_BF16 ? k_attend_simt<__nv_bfloat16> : k_attend_simt<__half>;
  MF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  kernel<<<(unsigned)blocks, simt_threads(p.dx, p.dz), smem, s>>>(p);
  MF_CUDA(cudaGetLastError());
  return MF_OK;
}

AttendSeq seq_of(const mf_heads& h) { return {h.d_ptr, h.stride_batch, h.stride_time, h.stride_head}; }

// What the passes of a call have in common.
template <typename Args>
AttendPass pass_of(const Args& a, const Plan& plan, uint32_t wait_test) {
  AttendPass p{};
  p.marks = a.d_marks;
  p.marks_sb = a.marks_stride_batch;
  p.marks_st = a.marks_stride_time;
  p.log_decay = a.d_log_decay;
  p.time = a.time;
  p.heads = (int)a.heads;
  p.chunks = plan.chunks;
  p.segs = plan.segs;
  p.seg_chunks = plan.seg_chunks;
  p.alpha = a.scale;
  p.status = a.d_status;
  p.tries = wait_test;
  return p;
}

mf_status chain(float* local, const float* seen, const float* state, const float* log_decay, int heads, const Plan& plan,
                int64_t rows, int values, bool reverse, cudaStream_t s) {
  const unsigned y = (unsigned)std::min<int64_t>(rows, 32768);
  if (!values) return MF_OK;
  for (int64_t at = 0; at < rows; at += y) {  // (launches of at most 32768 rows)
    const unsigned n = (unsigned)std::min<int64_t>(y, rows - at);
    k_attend_chain<<<dim3((unsigned)((values + 255) / 256), n), 256, 0, s>>>(
        local + at * plan.segs * values, seen + at * plan.segs, state ? state + at * values : nullptr, log_decay, at, heads,
        plan.segs, values, reverse);
    MF_CUDA(cudaGetLastError());
  }
  return MF_OK;
}

uint64_t up256(uint64_t n) { return (n + 255) / 256 * 256; }

}  // namespace

mf_status attend_sizes(int type, int64_t batch, int64_t time, int64_t heads, int64_t dk, int64_t dv, uint64_t* saved,
                       uint64_t* forward, uint64_t* backward) {
  const int64_t rows = batch * heads;
  const Plan plan = plan_of(type, rows, time, (int)dk, (int)dv);
  if (rows > 0x7FFFFFFF / plan.segs) {
    set_error("mf_linear_attention: batch * heads is too large");
    return MF_EINVAL;
  }
  const uint64_t states = (uint64_t)rows * (uint64_t)plan.segs * (uint64_t)(dk * dv);
  const uint64_t work = plan.segs > 1 ? up256(states * 4) + up256((uint64_t)rows * plan.segs * 4) : 0;
  if (saved) *saved = states;
  if (forward) *forward = work;
  if (backward) *backward = work;
  return MF_OK;
}

mf_status attend_forward(const mf_linear_attention_args& a, void* work, uint32_t wait_test, cudaStream_t s) {
  const int64_t rows = a.batch * a.heads;
  const int dk = (int)a.dim_k, dv = (int)a.dim_v;
  const Plan plan = plan_of(a.type, rows, a.time, dk, dv);
  if (a.time <= kFew && dk && dv && plan.segs == 1) {
    if (a.d_saved) {
      const size_t bytes = (size_t)rows * dk * dv * 4;
      if (a.d_state) MF_CUDA(cudaMemcpyAsync(a.d_saved, a.d_state, bytes, cudaMemcpyDeviceToDevice, s));
      else MF_CUDA(cudaMemsetAsync(a.d_saved, 0, bytes, s));
    }
    FewArgs f{seq_of(a.q), seq_of(a.k), seq_of(a.v), seq_of(a.o), a.d_marks, a.marks_stride_batch, a.marks_stride_time,
              a.d_log_decay, a.d_state, a.d_last, (int)a.time, (int)a.heads, dk, dv, a.scale};
    const bool wide = dv % 4 == 0 && (((uintptr_t)a.d_state | (uintptr_t)a.d_last) & 15) == 0;
    auto kernel = a.type == MF_TYPE_F32 ? (wide ? k_attend_few<float, 4> : k_attend_few<float, 1>)
                  : a.type == MF_TYPE_BF16 ? (wide ? k_attend_few<__nv_bfloat16, 4> : k_attend_few<__nv_bfloat16, 1>)
                                           : (wide ? k_attend_few<__half, 4> : k_attend_few<__half, 1>);
    kernel<<<(unsigned)rows, 256, 0, s>>>(f);
    MF_CUDA(cudaGetLastError());
    return MF_OK;
  }
  AttendPass p = pass_of(a, plan, wait_test);
  p.x = seq_of(a.q);
  p.y = seq_of(a.k);
  p.z = seq_of(a.v);
  p.out = seq_of(a.o);
  p.dx = dk;
  p.dz = dv;
  p.alpha_row = a.scale;
  p.alpha_src = 1.f;
  p.state = a.d_state;
  p.state_segs = 1;
  if (plan.segs > 1) {
    const uint64_t states = (uint64_t)rows * plan.segs * (uint64_t)(dk * dv);
    float* const local = a.d_saved ? a.d_saved : (float*)work;
    float* const seen = (float*)((char*)work + up256(states * 4));
    AttendPass own = p;
    own.local = local;
    own.seen = seen;
    mf_status st = run_pass(a.type, plan.tc, own, rows, s);
    if (st == MF_OK) st = chain(local, seen, a.d_state, a.d_log_decay, p.heads, plan, rows, dk * dv, false, s);
    if (st != MF_OK) return st;
    p.state = local;
    p.state_segs = plan.segs;
  } else {
    p.save = a.d_saved;
  }
  p.final_state = a.d_last;
  return run_pass(a.type, plan.tc, p, rows, s);
}

mf_status attend_backward(const mf_linear_attention_grad_args& a, void* work, uint32_t wait_test, cudaStream_t s) {
  const int64_t rows = a.batch * a.heads;
  const int dk = (int)a.dim_k, dv = (int)a.dim_v;
  const Plan plan = plan_of(a.type, rows, a.time, dk, dv);
  const AttendPass common = pass_of(a, plan, wait_test);
  const AttendSeq q = seq_of(a.q), k = seq_of(a.k), v = seq_of(a.v), d = seq_of(a.dout);
  AttendPass p = common;
  p.x = d;
  p.y = v;
  p.z = k;
  p.out = seq_of(a.dq);
  p.dx = dv;
  p.dz = dk;
  p.alpha_row = a.scale;
  p.alpha_src = 1.f;
  p.state = a.d_saved;
  p.state_segs = plan.segs;
  p.state_t = true;
  mf_status st = run_pass(a.type, plan.tc, p, rows, s);
  if (st != MF_OK) return st;

  p = common;
  p.reverse = true;
  p.x = k;
  p.y = q;
  p.z = d;
  p.out = seq_of(a.dv);
  p.dx = dk;
  p.dz = dv;
  p.alpha_row = 1.f;
  p.alpha_src = a.scale;
  p.state = a.d_dlast;
  p.state_segs = 1;
  if (plan.segs > 1) {
    const uint64_t states = (uint64_t)rows * plan.segs * (uint64_t)(dk * dv);
    AttendPass own = p;
    own.local = (float*)work;
    own.seen = (float*)((char*)work + up256(states * 4));
    st = run_pass(a.type, plan.tc, own, rows, s);
    if (st == MF_OK) st = chain(own.local, own.seen, a.d_dlast, a.d_log_decay, p.heads, plan, rows, dk * dv, true, s);
    if (st != MF_OK) return st;
    p.state = own.local;
    p.state_segs = plan.segs;
  }
  p.final_state = a.d_dstate;
  st = run_pass(a.type, plan.tc, p, rows, s);
  if (st != MF_OK) return st;
  p.final_state = nullptr;
  p.x = v;
  p.y = d;
  p.z = q;
  p.out = seq_of(a.dk);
  p.dx = dv;
  p.dz = dk;
  p.state_t = true;
  return run_pass(a.type, plan.tc, p, rows, s);
}

}  // namespace mf
