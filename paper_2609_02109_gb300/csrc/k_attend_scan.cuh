// The passes of linear attention step by step, on the CUDA cores (attend.cuh has the formulas; a translation unit a type): S <- f S + y z^T,
// out = x S, with the state in registers.
//
// A warp takes a segment of a head and some columns of z; a lane holds R rows of x of CC columns of the state (G groups of
// lanes share a column's rows).  A step is one packed multiply-add for every two values of the state and one for every two of the result:
// the decay is taken out of the steps, S' = S f^-n over the n samples of a block of steps, so z comes times f^-n, the result leaves
// times f^n, and the state is brought up to date once a block.  (A decay of more than 2^-2.5 a sample would leave fp32's
// range in a block; there the state is multiplied in each step.)  x and y go through shared memory as fp32, the next block's
// on their way meanwhile.
//
// Bound by the FMA pipe (2 dx dz products a step, 128 a clock and SM: 64 clocks for 64 x 64), for small states by the
// issue of what is around them (16 x 16: 8 of about 25 instructions a step are products).  The form by chunks of 32 steps
// does 32 (dx + dz) + 2 dx dz products a step from operands in shared memory: for 8 x 86400 x 4 x 16 x 16 it took 2300 us.
#pragma once

#include "attend.cuh"

namespace mf {
namespace {

constexpr int kWarps = 4;

__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float2 parts(uint64_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}

// STATES: a pass for the segments' own states.
template <typename T, int R, int CC, int G, bool STATES>
__global__ void __launch_bounds__(32 * kWarps) k_attend_scan(const __grid_constant__ AttendPass p, int64_t units, int blocks) {
  constexpr int kRows = R * G, kLanes = 32 / G, kCols = CC * kLanes;  // of a warp
  constexpr int kSteps = kRows > 64 ? 4 : 8;                          // of a block
  constexpr int kLoads = kSteps * kRows / 32, kZLoads = kSteps * kCols / 32;  // values of x, of y and of z that a lane loads
  __shared__ __align__(16) float s_x[kWarps][STATES ? 1 : kSteps][STATES ? 4 : kRows], s_y[kWarps][kSteps][kRows], s_w[kWarps][2][kSteps];
  __shared__ uint64_t s_z[kWarps][kSteps][kCols];  // (each value twice)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * kWarps + warp;
  if (unit >= units) return;
  const int segs = STATES ? p.segs - 1 : p.segs;
  const int64_t at = unit / blocks, row = at / segs;
  const int block = (int)(unit - at * blocks), seg = (int)(at - row * segs) + (STATES && p.reverse ? 1 : 0);
  const int64_t b = row / p.heads;
  const int h = (int)(row - b * p.heads);
  const T* const x = (const T*)p.x.p + b * p.x.sb + h * p.x.sh;
  const T* const y = (const T*)p.y.p + b * p.y.sb + h * p.y.sh;
  const T* const z = (const T*)p.z.p + b * p.z.sb + h * p.z.sh;
  T* const out = (T*)p.out.p + b * p.out.sb + h * p.out.sh;
  const float log_decay = finite_log(p.log_decay[h]), l2 = log_decay * kLog2e;
  const bool fast = !(fabsf(l2) <= 2.5f);  // (a NaN too)
  const Remains one(log_decay, 1.f);

  const int group = lane / kLanes, r0 = group * R, c0 = block * kCols + (lane - group * kLanes) * CC;
  uint64_t s[CC][R / 2];
  const float* const from = STATES || !p.state ? nullptr : p.state + (row * p.state_segs + (p.state_segs > 1 ? seg : 0)) * p.dx * p.dz;
#pragma unroll
  for (int c = 0; c < CC; ++c)
#pragma unroll
    for (int r = 0; r < R; r += 2) {
      float v[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bool in = r0 + r + k < p.dx && c0 + c < p.dz;
        v[k] = from && in ? from[p.state_t ? (c0 + c) * p.dx + r0 + r + k : (r0 + r + k) * p.dz + c0 + c] : 0.f;
        if (!STATES && p.save && in) p.save[row * p.dx * p.dz + (r0 + r + k) * p.dz + c0 + c] = v[k];
      }
      s[c][r / 2] = pair(v[0], v[1]);
    }

  // Blocks of steps in the pass's order: step `pos` is the pos-th from the segment's first, or, in reverse, from its last.
  const int64_t first = (int64_t)seg * p.seg_chunks * kAttendScanChunk;
  const int64_t length = max((int64_t)0, min(p.time - first, (int64_t)p.seg_chunks * kAttendScanChunk));
  auto time_of = [&](int64_t pos) { return p.reverse ? first + length - 1 - pos : first + pos; };
  float xr[STATES ? 1 : kLoads], yr[kLoads], zr[kZLoads];
  int mark = MF_MARK_MISSING;
  auto load = [&](int64_t n) {
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int i = lane + 32 * k, c = i % kRows;
      const int64_t pos = n + i / kRows, t = time_of(pos);
      const bool in = pos < length && c < p.dx;
      yr[k] = in ? to_f32(y[t * p.y.st + c]) : 0.f;
      if constexpr (!STATES) xr[k] = in ? to_f32(x[t * p.x.st + c]) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < kZLoads; ++k) {
      const int i = lane + 32 * k, c = block * kCols + i % kCols;
      const int64_t pos = n + i / kCols;
      zr[k] = pos < length && c < p.dz ? to_f32(z[time_of(pos) * p.z.st + c]) : 0.f;
    }
    mark = MF_MARK_MISSING;
    if (lane < kSteps && n + lane < length) mark = p.marks ? p.marks[b * p.marks_sb + time_of(n + lane) * p.marks_st] : MF_MARK_SAMPLE;
  };
  auto forget = [&]() {
#pragma unroll
    for (int c = 0; c < CC; ++c)
#pragma unroll
      for (int r = 0; r < R / 2; ++r) s[c][r] = 0;
  };
  auto keep = [&](const Remains& left) {
#pragma unroll
    for (int c = 0; c < CC; ++c)
#pragma unroll
      for (int r = 0; r < R / 2; ++r) {
        const float2 v = parts(s[c][r]);
        s[c][r] = pair(left(v.x, 0.f), left(v.y, 0.f));
      }
  };
  const Remains full(log_decay, (float)kSteps);
  constexpr uint32_t kAll = (1u << kSteps) - 1;
  if (length > 0) load(0);
  auto step = [&](int64_t n, int j) {
    uint64_t zz[CC], o[CC][2];
#pragma unroll
    for (int c = 0; c < CC; ++c) {
      zz[c] = s_z[warp][j][(lane % kLanes) * CC + c];
      o[c][0] = o[c][1] = 0;
    }
#pragma unroll
    for (int r = 0; r < R; r += 4) {
      const ulonglong2 yy = *(const ulonglong2*)&s_y[warp][j][r0 + r];
#pragma unroll
      for (int c = 0; c < CC; ++c) {
        s[c][r / 2] = fma2(yy.x, zz[c], s[c][r / 2]);
        s[c][r / 2 + 1] = fma2(yy.y, zz[c], s[c][r / 2 + 1]);
      }
      if constexpr (!STATES) {
        const ulonglong2 xx = *(const ulonglong2*)&s_x[warp][j][r0 + r];
#pragma unroll
        for (int c = 0; c < CC; ++c) {
          o[c][0] = fma2(xx.x, s[c][r / 2], o[c][0]);
          o[c][1] = fma2(xx.y, s[c][r / 2 + 1], o[c][1]);
        }
      }
    }
    if constexpr (!STATES) {
      const float v = s_w[warp][1][j];
      T* const to = out + time_of(n + j) * p.out.st + c0;
#pragma unroll
      for (int c = 0; c < CC; ++c) {
        const float2 u = parts(o[c][0]), q = parts(o[c][1]);
        float sum = (u.x + u.y) + (q.x + q.y);
        if constexpr (G == 2) sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        if (group == 0 && n + j < length && c0 + c < p.dz) to[c] = from_f32<T>(sum * v);
      }
    }
  };
  float samples = 0.f;
  uint32_t carry_reset = 0, carry_decay = 0;
#pragma unroll 1
  for (int64_t n = 0; n < length; n += kSteps) {
    const uint32_t missing = __ballot_sync(0xffffffffu, mark == MF_MARK_MISSING) & kAll, begins = __ballot_sync(0xffffffffu, mark == MF_MARK_FIRST) & kAll;
    const int seen = kSteps - __popc(missing);
    samples = samples < 0.f || begins ? -1.f : samples + (float)seen;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int i = lane + 32 * k;
      const bool gone = missing >> (i / kRows) & 1;
      s_y[warp][0][i] = gone && !p.reverse ? 0.f : yr[k];
      if constexpr (!STATES) s_x[warp][0][i] = gone && p.reverse ? 0.f : xr[k];
    }
    if (lane < kSteps) {
      // samples since the block's start: with the step's own forward, without it in reverse
      const int e = fast ? 0 : __popc(~missing & (p.reverse ? (1u << lane) - 1 : (2u << lane) - 1));
      s_w[warp][0][lane] = exp2f(-l2 * (float)e) * p.alpha_src;
      s_w[warp][1][lane] = exp2f(l2 * (float)e) * p.alpha_row;
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kZLoads; ++k) {
      const int i = lane + 32 * k, j = i / kCols;
      const float v = (missing >> j & 1) && !p.reverse ? 0.f : zr[k] * s_w[warp][0][j];
      s_z[warp][0][i] = pair(v, v);
    }
    __syncwarp();
    if (n + kSteps < length) load(n + kSteps);
    // what happens to the state before each step: forward the step's own decay or reset, in reverse that of the step before
    const uint32_t resets = p.reverse ? begins << 1 | carry_reset : begins, decays = p.reverse ? ~missing << 1 | carry_decay : ~missing;
    if (!fast && !(resets & kAll)) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) step(n, j);
    } else {
#pragma unroll 1
      for (int j = 0; j < kSteps; ++j) {
        if (resets >> j & 1) forget();
        else if (fast && (decays >> j & 1)) keep(one);
        step(n, j);
      }
    }
    if (p.reverse) {
      carry_reset = begins >> (kSteps - 1) & 1;
      carry_decay = ~missing >> (kSteps - 1) & 1;
    }
    if (!fast) keep(seen == kSteps ? full : Remains(log_decay, (float)seen));
  }
  if (carry_reset) forget();
  else if (fast && carry_decay) keep(one);
  float* to = nullptr;
  if (STATES) to = p.local + (row * p.segs + seg) * p.dx * p.dz;
  else if (p.final_state && seg == (p.reverse ? 0 : p.segs - 1)) to = p.final_state + row * p.dx * p.dz;
  if (to)
#pragma unroll
    for (int c = 0; c < CC; ++c)
#pragma unroll
      for (int r = 0; r < R; r += 2) {
        const float2 v = parts(s[c][r / 2]);
        const int at0 = r0 + r;
        if (c0 + c >= p.dz) continue;
        if (at0 < p.dx) to[at0 * p.dz + c0 + c] = v.x;
        if (at0 + 1 < p.dx) to[(at0 + 1) * p.dz + c0 + c] = v.y;
      }
  if (STATES && block == 0 && lane == 0) p.seen[row * p.segs + seg] = samples;
}

template <typename T, int R, int CC, int G>
mf_status run(const AttendPass& p, int64_t rows, cudaStream_t s) {
  constexpr int kCols = CC * 32 / G;
  const int blocks = (p.dz + kCols - 1) / kCols;
  const int64_t units = rows * (p.local ? p.segs - 1 : p.segs) * blocks, grid = (units + kWarps - 1) / kWarps;
  if (!units) return MF_OK;
  if (grid > 0x7FFFFFFF) {
    set_error("mf_linear_attention: batch * heads is too large");
    return MF_EINVAL;
  }
  if (p.local) k_attend_scan<T, R, CC, G, true><<<(unsigned)grid, 32 * kWarps, 0, s>>>(p, units, blocks);
  else k_attend_scan<T, R, CC, G, false><<<(unsigned)grid, 32 * kWarps, 0, s>>>(p, units, blocks);
  MF_CUDA(cudaGetLastError());
  return MF_OK;
}

// Rows and columns of a warp: the fewest that hold dx rows, and 16 columns where dz has no more.
template <typename T>
mf_status run(const AttendPass& p, int64_t rows, cudaStream_t s) {
  const bool few = p.dz <= 16;
  if (p.dx <= 8) return few ? run<T, 4, 1, 2>(p, rows, s) : run<T, 8, 1, 1>(p, rows, s);
  if (p.dx <= 16) return few ? run<T, 8, 1, 2>(p, rows, s) : run<T, 16, 1, 1>(p, rows, s);
  if (p.dx <= 32) return few ? run<T, 16, 1, 2>(p, rows, s) : run<T, 32, 1, 1>(p, rows, s);
  if (p.dx <= 64) return few ? run<T, 32, 1, 2>(p, rows, s) : p.dz <= 32 ? run<T, 64, 1, 1>(p, rows, s) : run<T, 64, 2, 1>(p, rows, s);
  return few ? run<T, 64, 1, 2>(p, rows, s) : run<T, 64, 2, 2>(p, rows, s);
}

}  // namespace
}  // namespace mf
