// Linear attention with a decay for each head (the operators' section of include/mf.h; the passes are in attend.cuh): the
// kernel for single tokens, the chain of segments, and the host side.
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

// One step.  A block passes a head's state once, V columns of a row a thread, kBatch rows at a time: bound by memory (the
// state is read and written once), with 128 KB of loads in flight an SM.  128 x 16 states of 128 x 128: 47 us, 5.7 TB/s
// (with the whole state in a block's registers, one block an SM: 98).
template <typename T, int V>
__global__ void __launch_bounds__(256, V == 4 ? 4 : 6) k_attend_one(const FewArgs a) {
  constexpr int kBatch = 8;
  __shared__ float s_q[128], s_k[128], s_v[128], s_sum[256 * V];
  const int b = blockIdx.x / a.heads, h = blockIdx.x - b * a.heads;
  const int groups = (a.dv + V - 1) / V, per = 256 / groups;  // threads of a row; rows side by side
  const int r0 = threadIdx.x / groups, c = (threadIdx.x - r0 * groups) * V;
  const int64_t at = (int64_t)blockIdx.x * a.dk * a.dv + c;
  const int mark = a.marks ? a.marks[b * a.marks_sb] : MF_MARK_SAMPLE;
  if (threadIdx.x < 128) {
    const int i = threadIdx.x;
    s_q[i] = i < a.dk ? to_f32(((const T*)a.q.p)[b * a.q.sb + h * a.q.sh + i]) : 0.f;
    s_k[i] = i < a.dk && mark != MF_MARK_MISSING ? to_f32(((const T*)a.k.p)[b * a.k.sb + h * a.k.sh + i]) : 0.f;
  } else {
    const int i = threadIdx.x - 128;
    s_v[i] = i < a.dv && mark != MF_MARK_MISSING ? to_f32(((const T*)a.v.p)[b * a.v.sb + h * a.v.sh + i]) : 0.f;
  }
  const Remains left(finite_log(a.log_decay[h]), mark == MF_MARK_FIRST ? -1.f : mark == MF_MARK_MISSING ? 0.f : 1.f);
  const bool still = mark == MF_MARK_MISSING;  // (the state's bits stay)
  __syncthreads();
  float sum[V] = {}, v[V];
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = c + k < 128 ? s_v[c + k] : 0.f;
  for (int r = r0; r0 < per && r < a.dk; r += kBatch * per) {
    float s[kBatch][V];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
#pragma unroll
      for (int k = 0; k < V; ++k) s[i][k] = 0.f;
      if (!a.state || r + i * per >= a.dk) continue;
      const float* const from = a.state + at + (int64_t)(r + i * per) * a.dv;
      if constexpr (V == 4) *(float4*)s[i] = *(const float4*)from;
      else s[i][0] = *from;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (r + i * per >= a.dk) continue;
      const float key = s_k[r + i * per], query = s_q[r + i * per];
      if (left.beyond())
#pragma unroll
        for (int k = 0; k < V; ++k) s[i][k] = left.grown(s[i][k]);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (!still) s[i][k] = left(s[i][k], key * v[k]);
        sum[k] = fmaf(query, s[i][k], sum[k]);
      }
      if (!a.last || (still && a.last == a.state)) continue;
      float* const to = a.last + at + (int64_t)(r + i * per) * a.dv;
      if constexpr (V == 4) *(float4*)to = *(const float4*)s[i];
      else *to = s[i][0];
    }
  }
#pragma unroll
  for (int k = 0; k < V; ++k) s_sum[threadIdx.x * V + k] = sum[k];
  __syncthreads();
  if (threadIdx.x < a.dv) {
    float total = 0.f;
    for (int g = 0; g < per; ++g) total += s_sum[g * groups * V + threadIdx.x];
    ((T*)a.o.p)[b * a.o.sb + h * a.o.sh + threadIdx.x] = from_f32<T>(total * a.scale);
  }
}

// A block holds a head's state in registers: V columns of a row a thread, in as many row groups as 256 threads make.
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
      if (left.beyond() && mark != MF_MARK_MISSING)
#pragma unroll
        for (int k = 0; k < V; ++k) s[i][k] = left.grown(s[i][k]);
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
// Segments
// ------------------------------------------------------------------------------------------

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
  constexpr int kAhead = 8;
  float own[kAhead], seen_here[kAhead];
  auto load = [&](int n0) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {  // (the last segment's own state is not needed)
      const bool in = n0 + k < segs - 1;
      const int seg = reverse ? segs - 1 - n0 - k : n0 + k;
      own[k] = in ? at[(int64_t)seg * values] : 0.f;
      seen_here[k] = in ? samples[seg] : 0.f;
    }
  };
  load(0);
  for (int n0 = 0; n0 < segs; n0 += kAhead) {
    float own_now[kAhead], seen_now[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      own_now[k] = own[k];
      seen_now[k] = seen_here[k];
    }
    load(n0 + kAhead);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (n0 + k >= segs) break;
      at[(int64_t)(reverse ? segs - 1 - n0 - k : n0 + k) * values] = now;
      const Remains left(log, seen_now[k]);
      if (left.beyond()) now = left.grown(now);
      now = left(now, own_now[k]);
    }
  }
}

// ------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------

constexpr int kFew = 8;  // steps that pass one by one

struct Plan {
  bool tc, few_warps;
  int chunk, chunks, segs, seg_chunks;
};

Plan plan_of(int type, int64_t rows, int64_t time, int dk, int dv) {
  Plan p{};
  // Chunks on the tensor cores where they take less time than steps: a chunk of 128 (not full: the same) as much as 90 steps of
  // a warp's columns, of fp16, whose operands are two parts, as 120.  (6264 heads with gradients, us by chunks and by steps:
  // 64 x 64 bf16 1210, and 30 steps 866, 38 1000, 60 1394; fp16 1580, and 38 steps 1002, 60 1400.  128 x 128 bf16 1896, and
  // 12 steps 1964, 19 2718; fp16 2437, and 12 steps 1914, 19 2650.  80 x 72, 19 steps: bf16 1476 and 1663, fp16 2010 and 1618.)
  const int64_t warps_of_step = dk <= 64 ? (dv + 31) / 32 : (dv + 15) / 16;
  p.tc = type != MF_TYPE_F32 && time > kFew && dk && dv && (dk > 32 || dv > 32) &&
         time * warps_of_step > (time + kAttendTcChunk - 1) / kAttendTcChunk * (type == MF_TYPE_BF16 ? 90 : 120);
  p.chunk = p.tc ? kAttendTcChunk : kAttendScanChunk;
  p.chunks = (int)((time + p.chunk - 1) / p.chunk);
  // Blocks (warps) that run at a time, and as many segments as make the longest one's way shortest: a segment's chunks once
  // more for its own state (about half of a chunk's work) where there are several.
  int64_t slots = 152;
  if (!p.tc) {
    slots *= scan_warps(std::max(dk, dv));
    // (segments of 256 steps or more: shorter ones spend their time on states)
    const int64_t warps = rows * std::max<int64_t>(1, time / 256);
    p.few_warps = warps * ((dv + 31) / 32) < 152 * 8;
    rows *= std::max(1, (dv + scan_columns(dk, dv, p.few_warps) - 1) / scan_columns(dk, dv, p.few_warps));
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
  return tc ? attend_tc(type, p, rows, s) : attend_scan(type, p, rows, s);
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
  p.few_warps = plan.few_warps;
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
    const bool one = a.time == 1;
    auto kernel = one ? (a.type == MF_TYPE_F32 ? (wide ? k_attend_one<float, 4> : k_attend_one<float, 1>)
                         : a.type == MF_TYPE_BF16 ? (wide ? k_attend_one<__nv_bfloat16, 4> : k_attend_one<__nv_bfloat16, 1>)
                                                  : (wide ? k_attend_one<__half, 4> : k_attend_one<__half, 1>))
                  : a.type == MF_TYPE_F32 ? (wide ? k_attend_few<float, 4> : k_attend_few<float, 1>)
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
