// The passes of linear attention step by step, on the CUDA cores (attend.cuh has the formulas; a translation unit a type): S <- f S + y z^T,
// out = x S, with the state in registers.
//
// A warp takes a segment of a head and some columns of z; a lane holds R rows of a column of the state (G groups of lanes
// share a column's rows).  A step is one packed multiply-add for every two values of the state and one for every two of the result:
// the decay is taken out of the steps, S' = S f^-n over the n samples of a block of steps, so z comes times f^-n, the result leaves
// times f^n, and the state is brought up to date once a block.  (Where a block's decay passes 2^-20 the state is
// multiplied in each step instead, and where a block's values are so large that f^-n, up to 2^20, could carry a product out of
// fp32's range.)  x and y go through shared memory as fp32, the next block's
// on their way meanwhile.
//
// Bound by the FMA pipe (2 dx dz products a step, 128 a clock and SM: 64 clocks for 64 x 64), for small states by the
// issue of what is around them: 16 x 16 takes 45 instructions a step and warp, 8 of them products (states alone: 24).
// Measured, fp32, 8 x 86400 x 4 x 16 x 16 with marks: 350 us a call, 326 without the question whether a block's values allow it to pass without
// its decay (blocks of 8 steps instead of 16: 343 then).  (Chunks of 32 steps, 32 (dx + dz) + 2 dx dz products a step from operands
// in shared memory: 2300.)  8 x 4096 x 8 x 32 x 32, bf16, forward: 165, with values converted where they were loaded 250.
#pragma once

#include <type_traits>

#include "attend.cuh"

namespace mf {
namespace {

constexpr int kWarps = 4;

__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
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

// A lane's values of a block of W-wide steps, N in all: groups of kVector consecutive ones, 32 groups apart.
template <int N>
constexpr int kVector = N < 4 ? N : 4;

// Values as they were loaded: converted where they are used, so that no conversion waits for the load of a block ahead.
template <typename T, int N>
struct Raw {
  static constexpr bool k32 = sizeof(T) == 4;
  uint32_t w[k32 ? N : (N + 1) / 2];
  __device__ __forceinline__ float operator[](int k) const {
    if constexpr (k32) return __uint_as_float(w[k]);
    else if constexpr (std::is_same_v<T, __half>) return __half2float(__ushort_as_half((unsigned short)(k & 1 ? w[k / 2] >> 16 : w[k / 2])));
    else return __uint_as_float(k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
  }
  __device__ __forceinline__ void put(int k, uint32_t bits) {  // (in order)
    if constexpr (k32) w[k] = bits;
    else w[k / 2] = k & 1 ? w[k / 2] | bits << 16 : bits;
  }
};

// `at` is where the block's first step's first column lies, `stride` the way to the next step; vectors: groups are aligned and whole.
template <typename T, int W, int N>
__device__ __forceinline__ void fetch(Raw<T, N>& v, const T* at, int64_t stride, int width, int steps, bool vectors) {
  constexpr int kV = kVector<N>, kWords = kV * (int)sizeof(T) / 4;  // (no whole word: single 16-bit values)
  using Bits = std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t>;
  struct alignas(sizeof(T) * kV) Group {
    uint32_t w[kWords ? kWords : 1];
  };
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int m = 0; m < N / kV; ++m) {
    const int i = (lane + 32 * m) * kV, j = i / W, c = i % W;
    const T* const from = at + j * stride + c;
    if (kWords && vectors) {
      Group g;
#pragma unroll
      for (int k = 0; k < kWords; ++k) g.w[k] = 0u;
      if (c < width && j < steps) g = *(const Group*)from;
#pragma unroll
      for (int k = 0; k < kWords; ++k) v.w[m * kWords + k] = g.w[k];
    } else {
#pragma unroll
      for (int k = 0; k < kV; ++k) v.put(m * kV + k, c + k < width && j < steps ? (uint32_t)((const Bits*)from)[k] : 0u);
    }
  }
}
template <typename T>
__device__ __forceinline__ bool vectors_of(const AttendSeq& q, int dim, int values) {
  return !((uintptr_t)q.p & (sizeof(T) * values - 1)) && !((dim | q.sb | q.st | q.sh) & (values - 1));
}

// The largest magnitude, and that of a warp's finite values.  (A NaN counts as nothing.)
template <typename T, int N>
__device__ __forceinline__ float most_of(float m, const Raw<T, N>& v) {
#pragma unroll
  for (int k = 0; k < N; ++k) m = fmaxf(m, fabsf(v[k]));
  return m;
}
template <int N, typename V>
__device__ __forceinline__ float warp_most(const V& v) {
  float m = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) m = fmaxf(m, fabsf(v[k]) <= 3.4028235e38f ? fabsf(v[k]) : 0.f);
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
}

// STATES: a pass for the segments' own states.
template <typename T, int R, int G, bool STATES>
__global__ void __launch_bounds__(32 * kWarps, scan_warps(R * G) / kWarps) k_attend_scan(const __grid_constant__ AttendPass p, int64_t units, int blocks) {
  constexpr int kRows = R * G, kCols = 32 / G;  // of a warp
  constexpr int kSteps = kRows > 64 ? 4 : kRows > 16 ? 8 : 16;        // of a block
  constexpr int kLoads = kSteps * kRows / 32, kZLoads = kSteps * kCols / 32;  // values of x, of y and of z that a lane loads
  __shared__ __align__(16) float s_x[kWarps][STATES ? 1 : kSteps][STATES ? 4 : kRows], s_y[kWarps][kSteps][kRows];
  __shared__ __align__(16) uint64_t s_z[kWarps][kSteps][kCols];  // (each value twice)
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
  // (a NaN too; a state that grows by more than 2 a block as well: what comes times f^-n would lose its small values)
  const bool fast = !(fabsf(l2) * kSteps <= 20.f) || l2 * kSteps > 1.f;
  // for lane e: what e samples leave, and its inverse
  const Remains table(log_decay, fast ? 0.f : (float)lane);
  const float inverse = exp2f(fast ? 0.f : -l2 * (float)lane);
  const float alpha_src = p.alpha_src, alpha_row = p.alpha_row;

  const int group = lane / kCols, r0 = group * R, c0 = block * kCols + lane % kCols;
  uint64_t s[R / 2];
  const float* const from = STATES || !p.state ? nullptr : p.state + (row * p.state_segs + (p.state_segs > 1 ? seg : 0)) * p.dx * p.dz;
#pragma unroll
  for (int r = 0; r < R; r += 2) {
    float v[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const bool in = r0 + r + k < p.dx && c0 < p.dz;
      v[k] = from && in ? from[p.state_t ? c0 * p.dx + r0 + r + k : (r0 + r + k) * p.dz + c0] : 0.f;
      if (!STATES && p.save && in) p.save[row * p.dx * p.dz + (r0 + r + k) * p.dz + c0] = v[k];
    }
    s[r / 2] = pair(v[0], v[1]);
  }

  // Blocks of steps in the pass's order: step `pos` is the pos-th from the segment's first, or, in reverse, from its last.
  const int64_t first = (int64_t)seg * p.seg_chunks * kAttendScanChunk;
  const int64_t length = max((int64_t)0, min(p.time - first, (int64_t)p.seg_chunks * kAttendScanChunk));
  const int64_t origin = p.reverse ? first + length - 1 : first;
  const int64_t xs = p.reverse ? -p.x.st : p.x.st, ys = p.reverse ? -p.y.st : p.y.st, zs = p.reverse ? -p.z.st : p.z.st,
                os = p.reverse ? -p.out.st : p.out.st, ms = p.reverse ? -p.marks_st : p.marks_st;
  const T* xp = x + origin * p.x.st;
  const T* yp = y + origin * p.y.st;
  const T* zp = z + origin * p.z.st + block * kCols;
  T* op = out + origin * p.out.st + c0;
  const uint8_t* mp = p.marks ? p.marks + b * p.marks_sb + origin * p.marks_st + (lane < kSteps ? lane : 0) * ms : nullptr;
  const int zwidth = p.dz - block * kCols;
  Raw<T, STATES ? 1 : kLoads> xr;
  Raw<T, kLoads> yr;
  Raw<T, kZLoads> zr;
  int mark = MF_MARK_MISSING;
  const bool xv = !STATES && vectors_of<T>(p.x, p.dx, kVector<kLoads>), yv = vectors_of<T>(p.y, p.dx, kVector<kLoads>),
             zv = vectors_of<T>(p.z, p.dz, kVector<kZLoads>);
  auto load = [&](int64_t left) {  // the next block, of `left` steps or all of its own
    const int steps = (int)min(left, (int64_t)kSteps);
    fetch<T, kRows>(yr, yp, ys, p.dx, steps, yv);
    fetch<T, kCols>(zr, zp, zs, zwidth, steps, zv);
    yp += kSteps * ys;
    zp += kSteps * zs;
    if constexpr (!STATES) {
      fetch<T, kRows, kLoads>(xr, xp, xs, p.dx, steps, xv);
      xp += kSteps * xs;
    }
    mark = lane < steps ? (mp ? *mp : MF_MARK_SAMPLE) : MF_MARK_MISSING;
    if (mp) mp += kSteps * ms;
  };
  auto forget = [&]() {
#pragma unroll
    for (int r = 0; r < R / 2; ++r) s[r] = 0;
  };
  auto scale = [&](float factor) {
    const uint64_t f = pair(factor, factor);
#pragma unroll
    for (int r = 0; r < R / 2; ++r) s[r] = mul2(f, s[r]);
  };
  auto keep = [&](float factor, float lost) {  // (one rounding of what is nearly the state: Remains)
    if (!(factor >= 0.5f)) return scale(factor);
    const uint64_t f = pair(lost, lost);
#pragma unroll
    for (int r = 0; r < R / 2; ++r) s[r] = fma2(f, s[r], s[r]);
  };
  const int times = l2 > 120.f ? 3 : 1;  // (of a factor that may be no float32, its third root)
  const float fast_factor = times > 1 ? third_root(l2) : exp2f(l2), up = fast ? 0.f : fmaxf(1.f, exp2f(-l2 * kSteps)), grown = fmaxf(1.f, exp2f(l2 * kSteps));
  // A block passes without its decay where nothing can overflow.  Where no x, y and z is above 2^20 (one question a block), no
  // alpha_src above 2^10 and no state that came in above 2^80, sums of up to 2^31 steps stay below 2^82, times f^-n and x
  // below 2^126.  Else `most` bounds the state: what came in, what those blocks brought, and 2^82 for the others.
  constexpr bool kHalf = std::is_same_v<T, __half>;  // (never above 2^16)
  float most = 0x1p82f;
  bool usual;
  {
    float m = 0.f;
#pragma unroll
    for (int r = 0; r < R / 2; ++r) {
      const float v[2] = {parts(s[r]).x, parts(s[r]).y};
      m = fmaxf(m, warp_most<2>(v));
    }
    usual = m < 0x1p80f && fabsf(alpha_src) <= 1024.f && l2 <= 0.f;
    most += m;
  }
  auto decay = [&]() {
#pragma unroll 1
    for (int k = 0; k < times; ++k) scale(fast_factor);
  };
  constexpr uint32_t kAll = (1u << kSteps) - 1;
  if (length > 0) load(length);
  const bool owned = group == 0 && c0 < p.dz;
  auto step = [&](int j, float v, bool in) {  // v: the result's factor
    const uint64_t zz = s_z[warp][j][lane % kCols];
    uint64_t o[2] = {0, 0};
#pragma unroll
    for (int r = 0; r < R; r += 4) {
      const ulonglong2 yy = *(const ulonglong2*)&s_y[warp][j][r0 + r];
      s[r / 2] = fma2(yy.x, zz, s[r / 2]);
      s[r / 2 + 1] = fma2(yy.y, zz, s[r / 2 + 1]);
      if constexpr (!STATES) {
        const ulonglong2 xx = *(const ulonglong2*)&s_x[warp][j][r0 + r];
        o[0] = fma2(xx.x, s[r / 2], o[0]);
        o[1] = fma2(xx.y, s[r / 2 + 1], o[1]);
      }
    }
    if constexpr (!STATES) {
      const float2 u = parts(o[0]), q = parts(o[1]);
      float sum = (u.x + u.y) + (q.x + q.y);
#pragma unroll
      for (int w = kCols; w < 32; w <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
      if (in && owned) *op = from_f32<T>(sum * v);
      op += os;
    }
  };
  float samples = 0.f;
  uint32_t carry_reset = 0;
#pragma unroll 1
  for (int64_t n = 0; n < length; n += kSteps) {
    const uint32_t missing = __ballot_sync(0xffffffffu, mark == MF_MARK_MISSING) & kAll, begins = __ballot_sync(0xffffffffu, mark == MF_MARK_FIRST) & kAll;
    const int seen = kSteps - __popc(missing);
    samples = samples < 0.f || begins ? -1.f : samples + (float)seen;
    // samples since the block's start: with the step's own forward, without it in reverse
    const int e = __popc(~missing & kAll & (p.reverse ? (1u << (lane & 15)) - 1 : (2u << (lane & 15)) - 1));
    const float wz = __shfl_sync(0xffffffffu, inverse, e) * alpha_src;
    float wo = __shfl_sync(0xffffffffu, table.factor, e) * alpha_row;
    float m = 0.f;
    if constexpr (!kHalf) {
      m = most_of(most_of(0.f, yr), zr);
      if constexpr (!STATES) m = most_of(m, xr);
    }
    __syncwarp();
    constexpr int kV = kVector<kLoads>, kZV = kVector<kZLoads>;
#pragma unroll
    for (int m = 0; m < kLoads / kV; ++m) {
      struct alignas(4 * kV) Group {
        float v[kV];
      } g;
#pragma unroll
      for (int k = 0; k < kV; ++k) g.v[k] = yr[m * kV + k];
      *(Group*)&s_y[warp][0][(lane + 32 * m) * kV] = g;
      if constexpr (!STATES) {
#pragma unroll
        for (int k = 0; k < kV; ++k) g.v[k] = xr[m * kV + k];
        *(Group*)&s_x[warp][0][(lane + 32 * m) * kV] = g;
      }
    }
#pragma unroll
    for (int m = 0; m < kZLoads / kZV; ++m) {
      const int i = (lane + 32 * m) * kZV;
      const float w = __shfl_sync(0xffffffffu, wz, i / kCols);
#pragma unroll
      for (int k = 0; k < kZV; k += 2) {
        const float v0 = zr[m * kZV + k] * w, v1 = zr[m * kZV + k + (kZV > 1)] * w;
        if constexpr (kZV > 1) *(ulonglong2*)&s_z[warp][0][i + k] = make_ulonglong2(pair(v0, v0), pair(v1, v1));
        else s_z[warp][0][i] = pair(v0, v0);
      }
    }
    bool direct = fast;
    if (__any_sync(0xffffffffu, m > 0x1p20f) || !usual) {
      // (rare, and of values that are read again: the conversions of the registers' stay behind their loads)
      const int there = (int)min(length - n, (int64_t)kSteps);
      Raw<T, kLoads> v;
      Raw<T, kZLoads> u;
      float x_most = 0.f;
      if constexpr (!STATES) {
        fetch<T, kRows>(v, xp - kSteps * xs, xs, p.dx, there, false);
        x_most = kRows * warp_most<kLoads>(v);
      }
      fetch<T, kRows>(v, yp - kSteps * ys, ys, p.dx, there, false);
      fetch<T, kCols>(u, zp - kSteps * zs, zs, zwidth, there, false);
      const float y_most = warp_most<kLoads>(v), z_most = warp_most<kZLoads>(u) * fabsf(alpha_src), s_up = fmaf(kSteps * (z_most * up), y_most, most);
      direct = direct || !(z_most * up < 0x1p126f && s_up < 0x1p126f && x_most * s_up < 0x1p126f);
      most = fmaf(most, grown, kSteps * y_most * z_most);
      usual = usual && most < 0x1p84f;
      if (direct) {
        wo = alpha_row;
#pragma unroll
        for (int i = 0; i < kZLoads; ++i) {
          const int at = (lane + 32 * (i / kZV)) * kZV + i % kZV;
          s_z[warp][0][at] = pair(u[i] * alpha_src, u[i] * alpha_src);
        }
      }
    }
    __syncwarp();
    if (missing) {
      for (uint32_t m = missing; m; m &= m - 1) {
        const int j = __ffs(m) - 1;
        for (int c = lane; c < kRows; c += 32) {
          if (!p.reverse) s_y[warp][j][c] = 0.f;
          else if constexpr (!STATES) s_x[warp][j][c] = 0.f;
        }
        if (!p.reverse)
          for (int c = lane; c < kCols; c += 32) s_z[warp][j][c] = 0;
      }
      __syncwarp();
    }
    if (n + kSteps < length) load(length - n - kSteps);
    // what happens to the state before each step: forward the step's own decay or reset, in reverse that of the step before
    const uint32_t resets = p.reverse ? begins << 1 | carry_reset : begins, decays = p.reverse ? ~missing << 1 : ~missing;
    const int steps = (int)min(length - n, (int64_t)kSteps);
    if (!direct && !(resets & kAll) && steps == kSteps) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) step(j, __shfl_sync(0xffffffffu, wo, j), true);
    } else {
#pragma unroll 1
      for (int j = 0; j < kSteps; ++j) {
        if (resets >> j & 1) forget();
        else if (direct && (decays >> j & 1)) decay();
        step(j, __shfl_sync(0xffffffffu, wo, j), j < steps);
      }
    }
    if constexpr (!STATES) {
      // (a missing sample's row of x, k or v, has no gradient: not NaN either where the state or y is not finite)
      if (p.reverse && owned)
        for (uint32_t m = missing & ((1u << steps) - 1); m; m &= m - 1) op[(__ffs(m) - 1 - kSteps) * os] = from_f32<T>(0.f);
    }
    if (p.reverse) carry_reset = begins >> (kSteps - 1) & 1;
    if (direct) {
      if (p.reverse && !(missing >> (kSteps - 1) & 1)) decay();
    } else keep(__shfl_sync(0xffffffffu, table.factor, seen), __shfl_sync(0xffffffffu, table.lost, seen));
  }
  if (carry_reset) forget();
  float* to = nullptr;
  if (STATES) to = p.local + (row * p.segs + seg) * p.dx * p.dz;
  else if (p.final_state && seg == (p.reverse ? 0 : p.segs - 1)) to = p.final_state + row * p.dx * p.dz;
  if (to)
#pragma unroll
    for (int r = 0; r < R; r += 2) {
      const float2 v = parts(s[r / 2]);
      if (c0 >= p.dz) continue;
      if (r0 + r < p.dx) to[(r0 + r) * p.dz + c0] = v.x;
      if (r0 + r + 1 < p.dx) to[(r0 + r + 1) * p.dz + c0] = v.y;
    }
  if (STATES && block == 0 && lane == 0) p.seen[row * p.segs + seg] = samples;
}

template <typename T, int R, int G>
mf_status run(const AttendPass& p, int64_t rows, cudaStream_t s) {
  constexpr int kCols = 32 / G;
  const int blocks = (p.dz + kCols - 1) / kCols;
  const int64_t units = rows * (p.local ? p.segs - 1 : p.segs) * blocks, grid = (units + kWarps - 1) / kWarps;
  if (!units) return MF_OK;
  if (grid > 0x7FFFFFFF) {
    set_error("mf_linear_attention: batch * heads is too large");
    return MF_EINVAL;
  }
  if (p.local) k_attend_scan<T, R, G, true><<<(unsigned)grid, 32 * kWarps, 0, s>>>(p, units, blocks);
  else k_attend_scan<T, R, G, false><<<(unsigned)grid, 32 * kWarps, 0, s>>>(p, units, blocks);
  MF_CUDA(cudaGetLastError());
  return MF_OK;
}

// The fewest rows that hold dx, and scan_columns' columns.
template <typename T>
mf_status run(const AttendPass& p, int64_t rows, cudaStream_t s) {
  const int cols = scan_columns(p.dx, p.dz, p.few_warps);
  if (p.dx <= 8) return cols == 16 ? run<T, 4, 2>(p, rows, s) : run<T, 8, 1>(p, rows, s);
  if (p.dx <= 16) return cols == 16 ? run<T, 8, 2>(p, rows, s) : run<T, 16, 1>(p, rows, s);
  if (p.dx <= 32) return cols == 8 ? run<T, 8, 4>(p, rows, s) : cols == 16 ? run<T, 16, 2>(p, rows, s) : run<T, 32, 1>(p, rows, s);
  if (p.dx <= 64) return cols == 8 ? run<T, 16, 4>(p, rows, s) : cols == 16 ? run<T, 32, 2>(p, rows, s) : run<T, 64, 1>(p, rows, s);
  return cols == 8 ? run<T, 32, 4>(p, rows, s) : run<T, 64, 2>(p, rows, s);
}

}  // namespace
}  // namespace mf
