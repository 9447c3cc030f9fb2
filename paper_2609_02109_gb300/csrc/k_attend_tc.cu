// The passes of linear attention on the tensor cores, for bf16 and fp16 (attend.cuh has the formulas).
//
// A block takes a segment of a head, 128 steps at a time, and holds the state in registers: fp32, a row of x a lane.
// A chunk is four products with fp32 accumulators in tensor memory (tcgen05, 128 rows each):
//   P = x y^T          [steps][steps]   operands as they are
//   inter = x S        [steps][dz]      S in bf16 parts, written to shared memory behind the chunk before; times what is
//                                       left of the state at each step, in place
//   own = w^T z        [dx][dz]         w = y times what is left of each step at the chunk's end, in three bf16 parts
//   intra = P' z       [steps][dz]      P' = P times what is left between the steps, in bf16 parts from tensor memory; added
//                                       to inter
// bf16 has fp32's range, so no part needs a scale, and a value's bits do not depend on what stands beside it: a column of z
// 2^40 below another one, or a key that was last seen 100 half-lives ago, keeps its bits.  (Parts in fp16 did not.)  Three
// parts hold all 24 bits of fp32: the state's own products lose nothing to them.  Results of bf16 calls take S and P' in two
// (16 bits, up to 2^-16 of a term, where the results' own rounding is 2^-9: 0.4 % of results are rounded the other way; in three
// 0.04 %, for 941 us instead of 848 below), those of fp16 calls in three.  fp16's x and z are two bf16 parts each, which hold
// them; P is a product of x and y as they are.
// An infinity or a NaN in z is taken out (times a zero weight it would reach steps that do not see it) and added to the
// results that do see it, by reading z again; the rest of what is not finite takes the way of the products.
//
// The floor is memory (x, y and z read once, and y and z once more where a head is split into segments; results written
// once).  What bounds the kernel is a chunk's chain of steps, one block an SM: w in parts, P, P', state, results, each a third
// issue and two thirds latency.  Measured, bf16, dx = dz = 128: 65536 x 16 heads forward 562 us (floor 158); 8 x 4096 x 16 heads
// with gradients 842 (222): 207 a pass.  On the way (the latter): loads and stores by registers 1546, tensor copies 989, the next x and
// y as soon as they are read 953, P' in fp16, in one part, 877.  A seventeenth warp for products and copies left 120
// registers a thread (spills: 1227 instead of 1039); two issuing threads changed nothing.  One block takes all of an SM's
// shared memory for 128 x 128; 64 x 64 would let two in.
#include <cstddef>

#include "attend.cuh"
#include "tma.cuh"

namespace mf {
namespace {

constexpr int kC = kAttendTcChunk, kThreads = 512, kPanel = kC * 128;  // kPanel: 64 columns of 128 steps, 16 bits each
constexpr uint32_t kWaitTries = 4096;                                  // about a millisecond each

// ---- PTX wrappers --------------------------------------------------------------------------

// Operands of 64 columns a panel, rows of 128 bytes, 128-byte swizzle.  K-major: rows run along M or N; groups of 8 rows
// are 1024 bytes apart.  MN-major: rows run along K, the next 64 of M or N are `panel` bytes on.
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr, uint32_t panel) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(panel >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// kind::f16, fp32 accumulators, 128 rows.  bf: bf16 operands (else fp16); a_mn, b_mn: MN-major operands.
__host__ __device__ constexpr uint32_t idesc(int n, bool bf, bool a_mn, bool b_mn) {
  return 1u << 4 | (bf ? 1u << 7 | 1u << 10 : 0u) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 |
         (uint32_t)(128 >> 4) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t id, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a),
      "l"(b), "r"(id), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t id, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a),
      "l"(b), "r"(id), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_u32(bar)) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tmem_ask(uint32_t addr, uint32_t (&r)[16]) {  // (until tmem_wait)
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(addr) : "memory");
}
// The registers are tied to the wait, so no use of them is scheduled before it.
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :: "memory");
}
__device__ __forceinline__ void tmem_put(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ void tmem_put_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void put_shared(uint32_t addr, const uint4& v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__device__ __forceinline__ uint4 get_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

// ---- values ----------------------------------------------------------------------------------

template <typename T> struct Bits;
template <> struct Bits<__nv_bfloat16> {
  static constexpr bool bf = true;
  static constexpr uint32_t inf = 0x7F80;
  static __device__ __forceinline__ float2 floats(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *(const uint32_t*)&h;
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    const __nv_bfloat162 h = __hmax2_nan(*(const __nv_bfloat162*)&a, *(const __nv_bfloat162*)&b);
    return *(const uint32_t*)&h;
  }
};
template <> struct Bits<__half> {
  static constexpr bool bf = false;
  static constexpr uint32_t inf = 0x7C00;
  static __device__ __forceinline__ float2 floats(uint32_t w) { return __half22float2(*(const __half2*)&w); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *(const uint32_t*)&h;
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    const __half2 h = __hmax2_nan(*(const __half2*)&a, *(const __half2*)&b);
    return *(const uint32_t*)&h;
  }
};
using Bf = Bits<__nv_bfloat16>;

// A pair of fp32 values as bf16 parts: the first cut off (so that none overflows), the others rounded; three hold all 24 bits.
// `a` and `b` become what the parts so far do not hold.
__device__ __forceinline__ uint32_t take_first(float& a, float& b) {
  const uint32_t u = __float_as_uint(a), v = __float_as_uint(b);
  a -= __uint_as_float(u & 0xFFFF0000u);
  b -= __uint_as_float(v & 0xFFFF0000u);
  return __byte_perm(u, v, 0x7632);
}
__device__ __forceinline__ uint32_t take_next(float& a, float& b) {
  const uint32_t w = Bf::pack(a, b);
  const float2 f = Bf::floats(w);
  a -= f.x;
  b -= f.y;
  return w;
}
// Eight fp16 values as two bf16 parts, which hold all of them.
__device__ __forceinline__ void split_half(const uint4& p, uint4* hi, uint4* lo) {
  const uint32_t in[4] = {p.x, p.y, p.z, p.w};
  uint32_t h[4], l[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    float2 f = Bits<__half>::floats(in[w]);
    h[w] = take_next(f.x, f.y);
    l[w] = Bf::pack(f.x, f.y);
  }
  *hi = make_uint4(h[0], h[1], h[2], h[3]);
  *lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// The largest magnitude (as bits) of a row, N pieces of eight values on each of four neighbouring lanes.  A NaN counts as
// larger than all.
template <typename T, int N>
__device__ __forceinline__ uint32_t row_max(const uint4 (&p)[N]) {
  const uint32_t m = 0x7FFF7FFFu;
  uint32_t v = 0;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t u = Bits<T>::larger(Bits<T>::larger(p[k].x & m, p[k].y & m), Bits<T>::larger(p[k].z & m, p[k].w & m));
    v = k ? Bits<T>::larger(v, u) : u;
  }
  v = Bits<T>::larger(v, __shfl_xor_sync(0xffffffffu, v, 1));
  v = Bits<T>::larger(v, __shfl_xor_sync(0xffffffffu, v, 2));
  return max(v & 0xFFFFu, v >> 16);
}
// The values that are not finite as zeros.
template <typename T>
__device__ __forceinline__ uint32_t finite_part(uint32_t w) {
  if ((w & 0x7FFFu) >= Bits<T>::inf) w &= 0xFFFF0000u;
  if ((w >> 16 & 0x7FFFu) >= Bits<T>::inf) w &= 0x0000FFFFu;
  return w;
}
template <typename T>
__device__ __noinline__ uint4 finite_part(uint4 p) {
  return make_uint4(finite_part<T>(p.x), finite_part<T>(p.y), finite_part<T>(p.z), finite_part<T>(p.w));
}

// Eight values of a row, from column c on; zeros from `dim` on.  vec: values of a load (8 or 4, that dim is a multiple of).
template <typename T>
__device__ __forceinline__ uint4 load8(const T* row, int c, int dim, int vec) {
  uint4 r = make_uint4(0u, 0u, 0u, 0u);
  if (vec == 8) {
    if (c < dim) r = *(const uint4*)(row + c);
  } else {
    if (c < dim) *(uint2*)&r.x = *(const uint2*)(row + c);
    if (c + 4 < dim) *(uint2*)&r.z = *(const uint2*)(row + c + 4);
  }
  return r;
}
// Eight steps' rows of W columns, a value a lane at a time, to where the tensor copies would put them: `to` is the address of
// the first step's first column (of a multiple of eight steps), `at` the first step's row, `steps` the steps that there are.
template <int W>
__device__ __forceinline__ void copy_narrow(uint32_t to, const uint16_t* at, int64_t stride, int dim, int steps) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int r0 = 0; r0 < 8; r0 += 4) {
    uint16_t v[4][W / 32];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int k = 0; k < W / 32; ++k) {
        const int c = lane + 32 * k;
        v[r][k] = c < dim && r0 + r < steps ? at[(r0 + r) * stride + c] : (uint16_t)0;
      }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int k = 0; k < W / 32; ++k) {
        const int c = lane + 32 * k;
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + (c >> 6) * kPanel + (r0 + r) * 128 + ((((c & 63) >> 3) ^ (r0 + r)) << 4) + (c & 7) * 2),
                     "h"(v[r][k]) : "memory");
      }
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* row, int c, int dim, int vec, const uint4& v) {
  if (vec == 8) {
    if (c < dim) *(uint4*)(row + c) = v;
  } else {
    if (c < dim) *(uint2*)(row + c) = make_uint2(v.x, v.y);
    if (c + 4 < dim) *(uint2*)(row + c + 4) = make_uint2(v.z, v.w);
  }
}
// The way back, of eight steps' results.
template <int W>
__device__ __forceinline__ void store_narrow(uint16_t* at, int64_t stride, uint32_t from, int dim, int steps) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int r = 0; r < steps; ++r)
#pragma unroll
    for (int k = 0; k < W / 32; ++k) {
      const int c = lane + 32 * k;
      uint16_t v;
      asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(from + (c >> 6) * kPanel + r * 128 + ((((c & 63) >> 3) ^ r) << 4) + (c & 7) * 2) : "memory");
      if (c < dim) at[r * stride + c] = v;
    }
}
// Values of a load or store of these rows: 8, 4 or 1.
template <typename T>
__device__ __forceinline__ int vec_of(const AttendSeq& q, int dim) {
  const uintptr_t a = (uintptr_t)q.p;
  const int64_t s = (int64_t)dim | q.sb | q.st | q.sh;
  return !(a & 15) && !(s & 7) ? 8 : !(a & 7) && !(s & 3) ? 4 : 1;
}
// Shared memory.  Operands take turns: the second part of fp16's x and the first two of w; results that leave, the state's
// third part and those of w; the state's first parts, then the third of w and the second of fp16's z.
template <typename T, int DX, int DZ, bool STATES>
struct Layout {
  static constexpr bool bf = Bits<T>::bf;
  static constexpr int px = DX / 64 * kPanel, pz = DZ / 64 * kPanel, s_panel = DX * 128, ps = DZ / 64 * s_panel;
  static constexpr int most(int a, int b) { return a > b ? a : b; }
  static constexpr int x = 0, y = STATES ? 0 : px, z = y + px, z_next = z + pz;
  static constexpr int w = STATES ? z_next + pz : z_next, s3 = w + most(px, pz);
  static constexpr int s = most(w + 2 * px, STATES ? 0 : bf ? w + pz : s3 + ps), w3 = s, z2 = s + px;
  // (w's parts are read as 128 columns whatever dx: nothing uses the upper half's products)
  static constexpr int small = most(most(STATES ? 0 : s + 2 * ps, bf ? z2 : z2 + pz), w3 + 2 * kPanel);
  static __device__ __forceinline__ int w_part(int k) { return k < 2 ? w + k * px : w3; }
  static __device__ __forceinline__ int s_part(int k) { return k < 2 ? s + k * ps : s3; }
};
// What steps' values need beside them.
struct Small {
  uint64_t bar[7];               // P; own; all of the results; one that nothing completes; copies of x and y; inter; copies of z
  uint32_t missing[2][4], begins[2][4], bad[2][4];  // bits of a chunk's steps; bad: a z that is not finite
  uint32_t tmem;
  alignas(16) float column[kC];  // P' off the diagonal blocks: a column's factor
  alignas(16) float diagonal[kC];  // and on them, where the decay allows it
  float row[kC];                 // what is left at each step of the state before the chunk (-1: nothing)
  uint8_t seen[kC], trace[kC];   // samples, and traces begun, up to and with each step
};
static_assert(offsetof(Small, column) % 16 == 0 && offsetof(Small, diagonal) % 16 == 0, "read by vectors");
template <typename T, int DX, int DZ, bool STATES>
constexpr size_t smem_bytes() { return Layout<T, DX, DZ, STATES>::small + sizeof(Small); }
static_assert(smem_bytes<__nv_bfloat16, 128, 128, false>() <= 232448 && smem_bytes<__half, 128, 128, false>() <= 232448 &&
              smem_bytes<__half, 128, 128, true>() <= 232448, "shared memory of a block");

// Steps of the chunk that hold a sample, and traces begun, up to and with step i (from step 0 on).
__device__ __forceinline__ int upto(const uint32_t (&words)[4], int i, bool invert) {
  int n = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t w = invert ? ~words[k] : words[k];
    const int in = i - 32 * k;
    n += in >= 31 ? __popc(w) : in < 0 ? 0 : __popc(w & (0xffffffffu >> (31 - in)));
  }
  return n;
}

// N columns of a state's row from c0 on, four at a time where its rows allow.
template <int N>
__device__ __forceinline__ void load_row(float (&s)[N], const float* row, int c0, int dim) {
  const bool fours = !((uintptr_t)row & 15) && !(dim & 3);
#pragma unroll
  for (int c = 0; c < N; c += 4) {
    if (fours) {
      if (c0 + c < dim) *(float4*)&s[c] = *(const float4*)(row + c0 + c);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c0 + c + k < dim) s[c + k] = row[c0 + c + k];
    }
  }
}
template <int N>
__device__ __forceinline__ void store_row(const float (&s)[N], float* row, int c0, int dim) {
  const bool fours = !((uintptr_t)row & 15) && !(dim & 3);
#pragma unroll
  for (int c = 0; c < N; c += 4) {
    if (fours) {
      if (c0 + c < dim) *(float4*)(row + c0 + c) = make_float4(s[c], s[c + 1], s[c + 2], s[c + 3]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c0 + c + k < dim) row[c0 + c + k] = s[c + k];
    }
  }
}

// A segment step by step, for memories that grow: factors between the steps of a chunk may be no float32s, and what they
// meet nothing.  A thread has a row of x and 32 columns; a step's products are added up through shared memory.
template <typename T>
__device__ __noinline__ void grow_steps(const AttendPass& p, bool states, int64_t row, int seg, float* sm, float log_decay) {
  constexpr int kPitch = 129;
  float *const s_x = sm, *const s_y = sm + 128, *const s_z = sm + 256, *const s_sum = sm + 384;
  const int tid = threadIdx.x, r = tid & 127, c0 = tid >> 7 << 5;
  const int64_t b = row / p.heads;
  const int h = (int)(row - b * p.heads);
  const T* const x = (const T*)p.x.p + b * p.x.sb + h * p.x.sh;
  const T* const y = (const T*)p.y.p + b * p.y.sb + h * p.y.sh;
  const T* const z = (const T*)p.z.p + b * p.z.sb + h * p.z.sh;
  T* const out = (T*)p.out.p + b * p.out.sb + h * p.out.sh;
  const float third = third_root(log_decay * kLog2e);
  const float* const from = states || !p.state ? nullptr : p.state + (row * p.state_segs + (p.state_segs > 1 ? seg : 0)) * p.dx * p.dz;
  float s[32];
#pragma unroll
  for (int c = 0; c < 32; ++c) {
    const bool in = r < p.dx && c0 + c < p.dz;
    s[c] = from && in ? from[p.state_t ? (c0 + c) * p.dx + r : r * p.dz + c0 + c] : 0.f;
    if (!states && p.save && in) p.save[row * p.dx * p.dz + r * p.dz + c0 + c] = s[c];
  }
  const int64_t first = (int64_t)seg * p.seg_chunks * kC, length = min(p.time - first, (int64_t)p.seg_chunks * kC);
  float samples = 0.f;
#pragma unroll 1
  for (int64_t n = 0; n < length; ++n) {
    const int64_t t = first + (p.reverse ? length - 1 - n : n);
    const int mark = p.marks ? p.marks[b * p.marks_sb + t * p.marks_st] : MF_MARK_SAMPLE;
    const bool gone = mark == MF_MARK_MISSING, begins = mark == MF_MARK_FIRST, used = p.reverse || !gone;
    __syncthreads();
    if (tid < 128) s_x[r] = !states && r < p.dx ? to_f32(x[t * p.x.st + r]) : 0.f;
    else if (tid < 256) s_y[r] = used && r < p.dx ? to_f32(y[t * p.y.st + r]) : 0.f;
    else if (tid < 384) s_z[r] = used && r < p.dz ? to_f32(z[t * p.z.st + r]) * p.alpha_src : 0.f;
    __syncthreads();
    samples = samples < 0.f || begins ? -1.f : gone ? samples : samples + 1.f;
    const bool grows = !begins && !gone;
#pragma unroll
    for (int c = 0; c < 32; ++c) {
      if (!p.reverse) s[c] = begins ? 0.f : grows ? s[c] * third * third * third : s[c];
      if (used) s[c] = fmaf(s_y[r], s_z[c0 + c], s[c]);
      if (!states) s_sum[r * kPitch + c0 + c] = s_x[r] * s[c];
      if (p.reverse) s[c] = begins ? 0.f : grows ? s[c] * third * third * third : s[c];
    }
    if (states) continue;
    __syncthreads();
    if (tid < p.dz) {
      float sum = 0.f;
      for (int k = 0; k < p.dx; ++k) sum += s_sum[k * kPitch + tid];
      out[t * p.out.st + tid] = from_f32<T>(p.reverse && gone ? 0.f : sum * p.alpha_row);
    }
  }
  float* to = nullptr;
  if (states) to = p.local + (row * p.segs + seg) * p.dx * p.dz;
  else if (p.final_state && seg == (p.reverse ? 0 : p.segs - 1)) to = p.final_state + row * p.dx * p.dz;
  if (to)
#pragma unroll
    for (int c = 0; c < 32; ++c)
      if (r < p.dx && c0 + c < p.dz) to[r * p.dz + c0 + c] = s[c];
  if (states && tid == 0) p.seen[row * p.segs + seg] = samples;
}

struct Maps {
  CUtensorMap x, y, z, out;
};

// STATES: a pass for the segments' own states.  TMA: x, y and z come, and results leave, by tensor copies; else by loads and
// stores of the widths that their alignment allows.
template <typename T, int DX, int DZ, bool STATES, bool TMA>
__global__ void __launch_bounds__(kThreads, 1) k_attend_tc(const __grid_constant__ AttendPass p, const __grid_constant__ Maps maps) {
  using B = Bits<T>;
  using L = Layout<T, DX, DZ, STATES>;
  constexpr bool kBf = B::bf;
  constexpr int kXLoads = DX / 32, kZLoads = DZ / 32;  // 16-byte pieces of a thread
  constexpr int kCols = DZ / 4;                        // a thread's columns of results and state
  extern __shared__ __align__(1024) uint8_t sm[];
  const uint32_t base = shared_u32(sm);
  Small& a = *(Small*)(sm + L::small);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quarter = warp & 3, group = warp >> 2;

  const int segs = STATES ? p.segs - 1 : p.segs;
  const int64_t row = blockIdx.x / segs;
  const int seg = (int)(blockIdx.x - row * segs) + (STATES && p.reverse ? 1 : 0);
  const int64_t b = row / p.heads;
  const int h = (int)(row - b * p.heads);
  const T* const x = (const T*)p.x.p + b * p.x.sb + h * p.x.sh;
  const T* const y = (const T*)p.y.p + b * p.y.sb + h * p.y.sh;
  const T* const z = (const T*)p.z.p + b * p.z.sb + h * p.z.sh;
  T* const out = (T*)p.out.p + b * p.out.sb + h * p.out.sh;
  const int xv = STATES ? 1 : vec_of<T>(p.x, p.dx), yv = vec_of<T>(p.y, p.dx), zv = vec_of<T>(p.z, p.dz),
            ov = STATES || TMA ? 8 : vec_of<T>(p.out, p.dz);
  // rows that allow no loads of four values go through shared memory, value by value
  const bool narrow = !TMA && ((!STATES && xv == 1) || yv == 1 || zv == 1);
  const float log_decay = finite_log(p.log_decay[h]), l2 = log_decay * kLog2e;

  if (l2 > 0.5f) {  // (2^64 a chunk)
    static_assert(L::small >= (384 + 128 * 129) * (int)sizeof(float), "shared memory of grow_steps");
    grow_steps<T>(p, STATES, row, seg, (float*)sm, log_decay);
    return;
  }

  // the products of a block with itself: what is left between two steps as a quotient, unless the decay is too fast
  const bool inverse = fabsf(l2) <= 1.f;

  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_u32(&a.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 0) {
    for (int k = 0; k < 7; ++k) barrier_init(&a.bar[k], 1);
    barrier_init_fence();
  }
  if (tid < 4) a.bad[0][tid] = 0;
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = a.tmem;
  constexpr uint32_t kP = 0, kOut = 128, kOwn = 256, kP3 = 384;  // columns
  const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);

  // the state: row srow of x, kCols columns from c0 on
  const int srow = quarter * 32 + lane, c0 = group * kCols;
  float s[kCols];
  {
    const float* const from = STATES || !p.state ? nullptr : p.state + (row * p.state_segs + (p.state_segs > 1 ? seg : 0)) * p.dx * p.dz;
    float* const save = STATES || !p.save ? nullptr : p.save + row * p.dx * p.dz + srow * p.dz;
#pragma unroll
    for (int c = 0; c < kCols; ++c) s[c] = 0.f;
    if (from && srow < p.dx) {
      if (p.state_t) {
#pragma unroll
        for (int c = 0; c < kCols; ++c)
          if (c0 + c < p.dz) s[c] = from[(c0 + c) * p.dx + srow];
      } else {
        load_row<kCols>(s, from + srow * p.dz, c0, p.dz);
      }
    }
    if (save && srow < p.dx) store_row<kCols>(s, save, c0, p.dz);
  }

  const int first = seg * p.seg_chunks, end = min(p.chunks, first + p.seg_chunks), count = end - first;
  // A thread loads pieces (lane & 3) + 4 k of one step.  (Eight neighbouring lanes' stores: steps that differ by 4, so that
  // the swizzle puts them into different banks.)
  const int step = warp * 8 + ((lane >> 3) | (lane >> 2 & 1) << 2), col = (lane & 3) * 8;
  const uint32_t at0 = base + step * 128 + (((lane & 3) ^ (step & 7)) << 4);
  auto place = [&](int region, int k, const uint4& v) { put_shared((at0 ^ ((k & 1) << 6)) + region + (k >> 1) * kPanel, v); };
  auto get = [&](int region, int k) { return get_shared((at0 ^ ((k & 1) << 6)) + region + (k >> 1) * kPanel); };
  auto z_of = [&](int n) { return STATES && (n & 1) ? L::z_next : L::z; };
  const uint4 zeros = make_uint4(0u, 0u, 0u, 0u);
  uint4 xr[STATES || TMA ? 1 : kXLoads], yr[TMA ? 1 : kXLoads], zr[TMA ? 1 : kZLoads];
  int mark = MF_MARK_SAMPLE;
  auto chunk_at = [&](int n) { return (int64_t)(p.reverse ? end - 1 - n : first + n) * kC; };
  auto load = [&](int64_t lo) {
    const int64_t t = lo + step;
    if constexpr (!TMA) {
      const bool in = t < p.time && !narrow;
      const T* const xp = x + t * p.x.st;
      const T* const yp = y + t * p.y.st;
      const T* const zp = z + t * p.z.st;
#pragma unroll
      for (int k = 0; k < kXLoads; ++k) {
        if constexpr (!STATES) xr[k] = in ? load8(xp, col + 32 * k, p.dx, xv) : zeros;
        yr[k] = in ? load8(yp, col + 32 * k, p.dx, yv) : zeros;
      }
#pragma unroll
      for (int k = 0; k < kZLoads; ++k) zr[k] = in ? load8(zp, col + 32 * k, p.dz, zv) : zeros;
    }
    if (tid < kC) {
      mark = MF_MARK_MISSING;
      if (lo + tid < p.time) mark = p.marks ? p.marks[b * p.marks_sb + (lo + tid) * p.marks_st] : MF_MARK_SAMPLE;
    }
  };
  auto put_marks = [&](int which) {
    if (tid < kC) {
      const uint32_t missing = __ballot_sync(0xffffffffu, mark == MF_MARK_MISSING), begins = __ballot_sync(0xffffffffu, mark == MF_MARK_FIRST);
      if (lane == 0) {
        a.missing[which][warp] = missing;
        a.begins[which][warp] = begins;
      }
    }
  };

  // Copies of a chunk's x and y (of states y alone), and of its z (of states into two places in turn).
  auto copy_xy = [&](int n) {
    const int32_t lo = (int32_t)chunk_at(n);
    barrier_expect(&a.bar[4], (STATES ? 1 : 2) * L::px);
#pragma unroll
    for (int k = 0; k < DX / 64; ++k) {
      if constexpr (!STATES) tma_load_4d(base + L::x + k * kPanel, &maps.x, 64 * k, lo, h, (int32_t)b, &a.bar[4]);
      tma_load_4d(base + L::y + k * kPanel, &maps.y, 64 * k, lo, h, (int32_t)b, &a.bar[4]);
    }
  };
  auto copy_z = [&](int n) {
    barrier_expect(&a.bar[6], L::pz);
#pragma unroll
    for (int k = 0; k < DZ / 64; ++k)
      tma_load_4d(base + z_of(n) + k * kPanel, &maps.z, 64 * k, (int32_t)chunk_at(n), h, (int32_t)b, &a.bar[6]);
  };

  bool gave_up = false;
  auto wait = [&](int k, uint32_t parity) { gave_up = gave_up || !(barrier_polls(&a.bar[k], parity) || barrier_wait(&a.bar[k], parity, kWaitTries)); };
  if (p.tries) gave_up = !barrier_wait(&a.bar[3], 0, p.tries);  // (a test of the way out: nothing completes it)

  // The state as the operand of the next chunk, in bf16 parts.
  auto put_state = [&]() {
    if (DX == 128 || quarter < 2) {
#pragma unroll
      for (int c = 0; c < kCols; c += 8) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = s[c + k];
        const int piece = (c0 + c) / 8;
        const uint32_t to = base + (piece >> 3) * L::s_panel + srow * 128 + (((piece & 7) ^ (srow & 7)) << 4);
        put_shared(to + L::s_part(0), make_uint4(take_first(v[0], v[1]), take_first(v[2], v[3]), take_first(v[4], v[5]), take_first(v[6], v[7])));
        put_shared(to + L::s_part(1), make_uint4(take_next(v[0], v[1]), take_next(v[2], v[3]), take_next(v[4], v[5]), take_next(v[6], v[7])));
        if constexpr (!kBf) put_shared(to + L::s_part(2), make_uint4(Bf::pack(v[0], v[1]), Bf::pack(v[2], v[3]), Bf::pack(v[4], v[5]), Bf::pack(v[6], v[7])));
      }
    }
    fence_shared();
  };

  // Products and copies are issued by one thread, of a warp whose block of P' no step sees (so the others seldom wait for it).
  const bool issuer = tid == (p.reverse ? 3 : 12) * 32;
  auto make_p = [&]() {  // P = x y^T
    constexpr uint32_t id = idesc(kC, kBf, false, false);
#pragma unroll
    for (int k = 0; k < DX / 16; ++k) {
      const uint32_t at = (k >> 2) * kPanel + (k & 3) * 32;
      mma_ss(tmem + kP, desc_k(base + L::x + at), desc_k(base + L::y + at), id, k > 0);
    }
    commit(&a.bar[0]);
  };
  // (Of a product's parts the small ones first: each addition cuts what the sum has by then.  The last state of 2 x 1000 x
  // 4 x 128 x 128: 1.5e-7 off, with the large parts first 7e-7.)
  auto make_inter = [&]() {  // x S
    constexpr uint32_t id = idesc(DZ, true, false, true);
    auto product = [&](int xp, int sp, bool add) {
#pragma unroll
      for (int k = 0; k < DX / 16; ++k)
        mma_ss(tmem + kOut, desc_k(base + xp + (k >> 2) * kPanel + (k & 3) * 32), desc_mn(base + L::s_part(sp) + k * 2048, L::s_panel), id, add || k > 0);
    };
    if constexpr (!kBf) {
      product(L::x, 2, false);
      product(L::w, 1, true);
      product(L::w, 0, true);
    }
    product(L::x, 1, !kBf);
    product(L::x, 0, true);
    commit(&a.bar[5]);
  };
  auto make_own = [&](int zp) {  // w^T z.  (What the third part of w and the second of z make is 2^-24 of it.)
    constexpr uint32_t id = idesc(DZ, true, true, true);
    auto product = [&](int wp, int at, bool add) {
#pragma unroll
      for (int k = 0; k < kC / 16; ++k)
        mma_ss(tmem + kOwn, desc_mn(base + L::w_part(wp) + k * 2048, kPanel), desc_mn(base + at + k * 2048, kPanel), id, add || k > 0);
    };
    product(2, zp, false);
    product(1, zp, true);
    if constexpr (!kBf) {
      product(1, L::z2, true);
      product(0, L::z2, true);
    }
    product(0, zp, true);
    commit(&a.bar[1]);
  };
  auto make_intra = [&]() {  // P' z, added to what the state brings
    constexpr uint32_t id = idesc(DZ, true, false, true);
    auto product = [&](uint32_t pp, int at) {
#pragma unroll
      for (int k = 0; k < kC / 16; ++k) mma_ts(tmem + kOut, tmem + pp + k * 8, desc_mn(base + at + k * 2048, kPanel), id, true);
    };
    if constexpr (!kBf) {
      product(kP3, L::z);
      product(kP + 64, L::z2);
      product(kP, L::z2);
    }
    product(kP + 64, L::z);
    product(kP, L::z);
    commit(&a.bar[2]);
  };

  uint32_t phase = 0;
  int n = 0;
  bool xy_coming = false, z_coming = false;  // (of the issuer: copies of the next chunk are on their way)
  if (TMA && issuer && count > 0 && !gave_up) {
    copy_xy(0);
    copy_z(0);
    xy_coming = z_coming = true;
  }
  if (count > 0 && !gave_up) load(chunk_at(0));
  put_marks(0);
  if (!STATES && count > 0) put_state();

  float samples = 0.f;
  bool over = __syncthreads_or(gave_up);
  for (; n < count && !over; ++n, phase ^= 1) {
    const int64_t lo = chunk_at(n);
    const int now = n & 1;
    const bool more = n + 1 < count;
    if (tid < 4) a.bad[now ^ 1][tid] = 0;
    uint32_t missing[4], begins[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      missing[k] = a.missing[now][k];
      begins[k] = a.begins[now][k];
    }
    const int all = kC - (__popc(missing[0]) + __popc(missing[1]) + __popc(missing[2]) + __popc(missing[3]));
    const int traces = __popc(begins[0]) + __popc(begins[1]) + __popc(begins[2]) + __popc(begins[3]);
    // (a missing sample's row of x in reverse, k or v, has no gradient: not NaN either where the state or y is not finite)
    const bool no_row = p.reverse && (a.missing[now][quarter] >> lane & 1);

    // -- the step's weights, x and y
    const bool gone = missing[step >> 5] >> (step & 31) & 1;
    float weight;  // of the step's y z in the state
    {
      const bool plain = all == kC && traces == 0;  // (most chunks: a sample in each step, of one trace)
      const int seen = plain ? step + 1 : upto(missing, step, true), trace = plain ? 0 : upto(begins, step, false);
      const float head = trace ? -1.f : exp2f(l2 * (float)seen), tail = trace == traces ? exp2f(l2 * (float)(all - seen)) : -1.f;
      weight = p.reverse ? head : tail;
      if ((lane & 3) == 0) {
        a.seen[step] = (uint8_t)seen;
        a.trace[step] = (uint8_t)trace;
        a.row[step] = p.reverse ? tail : head;
      }
    }
    if constexpr (TMA) {
      wait(4, phase);
      xy_coming = false;
    } else if (narrow) {
      const int64_t t0 = lo + warp * 8;
      const int steps = (int)max((int64_t)0, min(p.time - t0, (int64_t)8));
      const uint32_t to = base + warp * 8 * 128;
      if constexpr (!STATES) copy_narrow<DX>(to + L::x, (const uint16_t*)x + t0 * p.x.st, p.x.st, p.dx, steps);
      copy_narrow<DX>(to + L::y, (const uint16_t*)y + t0 * p.y.st, p.y.st, p.dx, steps);
      copy_narrow<DZ>(to + z_of(n), (const uint16_t*)z + t0 * p.z.st, p.z.st, p.dz, steps);
      __syncwarp();  // (a warp copies its own steps' rows)
    } else {
#pragma unroll
      for (int k = 0; k < kXLoads; ++k) {
        if constexpr (!STATES) place(L::x, k, xr[k]);
        place(L::y, k, yr[k]);
      }
#pragma unroll
      for (int k = 0; k < kZLoads; ++k) place(z_of(n), k, zr[k]);
    }
    if (gone && !(STATES && p.reverse)) {
#pragma unroll
      for (int k = 0; k < kXLoads; ++k) place(p.reverse ? L::x : L::y, k, zeros);
    }

    // -- w: y times what is left of each step at the chunk's end, in three parts; z without what is not finite
    auto put_w_z = [&]() {
      if constexpr (TMA) {
        wait(6, phase);
        z_coming = false;
      }
      {
        uint4 v[kZLoads];
#pragma unroll
        for (int k = 0; k < kZLoads; ++k) v[k] = get(z_of(n), k);
        if (!p.reverse && gone) {
#pragma unroll
          for (int k = 0; k < kZLoads; ++k) {
            v[k] = zeros;
            if constexpr (kBf) place(z_of(n), k, v[k]);
          }
        }
        if (__any_sync(0xffffffffu, row_max<T>(v) >= B::inf)) {
          if (row_max<T>(v) >= B::inf && (lane & 3) == 0) atomicOr(&a.bad[now][step >> 5], 1u << (step & 31));
#pragma unroll
          for (int k = 0; k < kZLoads; ++k) {
            v[k] = finite_part<T>(v[k]);
            if constexpr (kBf) place(z_of(n), k, v[k]);
          }
        }
        if constexpr (!kBf) {
#pragma unroll
          for (int k = 0; k < kZLoads; ++k) {
            uint4 hi, lo2;
            split_half(v[k], &hi, &lo2);
            place(z_of(n), k, hi);
            place(L::z2, k, lo2);
          }
        }
      }
      const float f = weight * p.alpha_src;
      uint4 third[kXLoads];
#pragma unroll
      for (int k = 0; k < kXLoads; ++k) {
        // (nothing of a step whose weight is negative reaches the end, whatever it is)
        uint4 v = get(L::y, k);
        if (weight < 0.f) v = zeros;
        const uint32_t q[4] = {v.x, v.y, v.z, v.w};
        uint32_t p1[4], p2[4], p3[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float2 u = B::floats(q[w]);
          u.x *= f;
          u.y *= f;
          p1[w] = take_first(u.x, u.y);
          p2[w] = take_next(u.x, u.y);
          p3[w] = Bf::pack(u.x, u.y);
        }
        place(L::w_part(0), k, make_uint4(p1[0], p1[1], p1[2], p1[3]));
        place(L::w_part(1), k, make_uint4(p2[0], p2[1], p2[2], p2[3]));
        third[k] = make_uint4(p3[0], p3[1], p3[2], p3[3]);
      }
      if constexpr (!STATES && kBf) wait(5, phase);  // (the third part's place is the state's)
#pragma unroll
      for (int k = 0; k < kXLoads; ++k) place(L::w_part(2), k, third[k]);
    };

    // -- P' = P times what is left between its steps: a thread has step i, 32 columns; and what the state brings, times what is left
    auto put_p = [&]() {
      const int i = srow, j0 = group * 32;
      const bool none = p.reverse ? group < quarter : group > quarter;  // (blocks that no step of i's block sees)
      float v[32];
      wait(0, phase);
      fence_after();
      if (none) {
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = 0.f;
      } else {
        // which of the block's steps step i sees, and a factor of the row; the columns' are in shared memory
        const uint32_t here = begins[group], mine = 0xffffffffu >> (31 - lane);
        const int seen_i = a.seen[i], trace_i = a.trace[i];
        uint32_t sees;
        float f;  // (of the row)
        const float* table;
        if (group != quarter) {
          const int border = p.reverse ? j0 - 1 : j0 | 31;
          // forward: the steps from the block's last first sample on; reverse: those before its first one
          const uint32_t block = p.reverse ? (here ? (here & (0u - here)) - 1u : 0xffffffffu)
                                           : (here ? 0xffffffffu << (31 - __clz(here)) : 0xffffffffu);
          sees = a.trace[border] == trace_i ? block : 0u;
          f = exp2f(l2 * (float)abs(seen_i - a.seen[border]));
          table = a.column;
        } else {
          if (p.reverse) {
            const uint32_t later = here & ~mine;  // the first samples behind i
            sees = (later ? (later & (0u - later)) - 1u : 0xffffffffu) & (0xffffffffu << lane);
          } else {
            const uint32_t before = here & mine;  // those up to and with i
            sees = (before ? 0xffffffffu << (31 - __clz(before)) : 0xffffffffu) & mine;
          }
          const int far = p.reverse ? j0 | 31 : j0 - 1;
          f = inverse ? exp2f(l2 * (float)abs(seen_i - (far < 0 ? 0 : a.seen[far]))) : 1.f;
          table = a.diagonal;
        }
        if (no_row) sees = 0u;
        f *= p.alpha;
        const bool all_see = __all_sync(0xffffffffu, sees == 0xffffffffu);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t r[16];
          tmem_ask(lanes + kP + j0 + 16 * half, r);
          tmem_wait(r);
#pragma unroll
          for (int k = 0; k < 16; k += 4) {
            const float4 c = *(const float4*)(table + j0 + 16 * half + k);
            const float w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) v[16 * half + k + q] = __uint_as_float(r[k + q]) * (f * w[q]);
          }
        }
        if (!all_see)
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] = sees >> k & 1 ? v[k] : 0.f;
        if (group == quarter && !inverse) {
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (sees >> k & 1) v[k] *= exp2f(l2 * (float)abs(seen_i - a.seen[j0 + k]));
        }
      }
      // (the parts take the place of P, when all four warps of these lanes have read theirs)
      fence_before();
      asm volatile("bar.sync %0, %1;" ::"r"(1 + quarter), "r"(128) : "memory");
      fence_after();
      uint32_t part[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) part[k] = take_first(v[2 * k], v[2 * k + 1]);
      tmem_put(lanes + kP + group * 16, part);
#pragma unroll
      for (int k = 0; k < 16; ++k) part[k] = take_next(v[2 * k], v[2 * k + 1]);
      tmem_put(lanes + kP + 64 + group * 16, part);
      if constexpr (!kBf) {
#pragma unroll
        for (int k = 0; k < 16; ++k) part[k] = Bf::pack(v[2 * k], v[2 * k + 1]);
        tmem_put(lanes + kP3 + group * 16, part);
      }
      if constexpr (!kBf) wait(5, phase);  // (bf16's has been waited for)
      fence_after();
      const float w = a.row[i], left = w * p.alpha_row;
      const bool dark = w < 0.f || no_row;  // (of a trace that has ended nothing comes, whatever it was)
#pragma unroll
      for (int c = 0; c < kCols; c += 16) {
        uint32_t r[16];
        tmem_ask(lanes + kOut + c0 + c, r);
        tmem_wait(r);
#pragma unroll
        for (int k = 0; k < 16; ++k) r[k] = dark ? 0u : __float_as_uint(__uint_as_float(r[k]) * left);
        tmem_put(lanes + kOut + c0 + c, r);
      }
      tmem_put_wait();
    };

    if constexpr (!STATES) {
      // (the results before have left shared memory, where w goes)
      if (TMA && issuer) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
      fence_shared();
      fence_before();
      __syncthreads();
      if (issuer) {
        fence_after();
        make_p();
        if constexpr (kBf) make_inter();
      }
      __syncwarp();
      if (tid < kC) {
        // what is left of step j at its block's border on the side of the steps that see it, and the inverse from the
        // border on the other side
        const int near = p.reverse ? (tid & ~31) - 1 : tid | 31, far = p.reverse ? tid | 31 : (tid & ~31) - 1;
        const int seen = a.seen[tid], at = near < 0 ? 0 : a.seen[near], from = far < 0 ? 0 : a.seen[far];
        a.column[tid] = exp2f(l2 * (float)abs(seen - at));
        a.diagonal[tid] = inverse ? exp2f(-l2 * (float)abs(seen - from)) : 1.f;
      }
      if constexpr (!kBf) {
        // x as two bf16 parts
        wait(0, phase);
#pragma unroll
        for (int k = 0; k < kXLoads; ++k) {
          uint4 hi, lo2;
          split_half(get(L::x, k), &hi, &lo2);
          place(L::x, k, hi);
          place(L::w, k, lo2);
        }
        fence_shared();
        fence_before();
        __syncthreads();
        if (issuer) {
          fence_after();
          make_inter();
        }
        __syncwarp();
        put_p();
      }
    }
    put_w_z();
    fence_shared();
    fence_before();
    __syncthreads();
    if (issuer) {
      fence_after();
      make_own(z_of(n));
      if constexpr (!STATES && !kBf) make_intra();
      if (TMA && more && !gave_up) {  // (x and y have been read)
        copy_xy(n + 1);
        xy_coming = true;
        if constexpr (STATES) {
          copy_z(n + 1);
          z_coming = true;
        }
      }
    }
    __syncwarp();
    if constexpr (!STATES && kBf) {
      put_p();
      fence_before();
      __syncthreads();
      if (issuer) {
        fence_after();
        make_intra();
      }
      __syncwarp();
    }
    if (more) load(chunk_at(n + 1));

    // -- the state: what is left of it, and the chunk's own
    const bool any_bad = a.bad[now][0] | a.bad[now][1] | a.bad[now][2] | a.bad[now][3];
    const float chunk_samples = traces ? -1.f : (float)all;
    samples = samples < 0.f || traces ? -1.f : samples + (float)all;
    wait(1, phase);
    fence_after();
    if (DX == 128 || quarter < 2) {  // (rows of the state)
      // s' = left s + own as (keep + lost) s + own: one rounding of what is nearly s
      const Remains left(log_decay, chunk_samples);
      const float keep = left.factor >= 0.5f ? 1.f : 0.f, lost = left.factor >= 0.5f ? left.lost : left.factor;
      if (left.factor < 0.f) {
#pragma unroll
        for (int c = 0; c < kCols; ++c) s[c] = 0.f;
      }
#pragma unroll
      for (int c = 0; c < kCols; c += 16) {
        uint32_t r[16];
        tmem_ask(lanes + kOwn + c0 + c, r);
        tmem_wait(r);
#pragma unroll
        for (int k = 0; k < 16; ++k) s[c + k] = fmaf(keep, s[c + k], fmaf(lost, s[c + k], __uint_as_float(r[k])));
      }
      if (any_bad)
#pragma unroll 1
        for (int t = 0; t < kC; ++t) {
          if (!(a.bad[now][t >> 5] >> (t & 31) & 1) || a.trace[t] != (p.reverse ? 0 : traces)) continue;
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
            if (c0 + c >= p.dz || srow >= p.dx) continue;
            const float v = to_f32(z[(lo + t) * p.z.st + c0 + c]);
            if (!(fabsf(v) <= 3.4028235e38f)) s[c] = __int_as_float(0x7FC00000);
          }
        }
    }
    if constexpr (!STATES) {
      if (kBf && more) put_state();  // (w's third part has been read)
      // -- results
      const int i = srow, trace_i = a.trace[i];
      wait(2, phase);
      fence_after();
      if (TMA && issuer && more && !gave_up) {  // (z has been read)
        copy_z(n + 1);
        z_coming = true;
      }
      T* const to = out + (lo + i) * p.out.st;
#pragma unroll
      for (int c = 0; c < kCols; c += 16) {
        uint32_t u[16];
        tmem_ask(lanes + kOut + c0 + c, u);
        tmem_wait(u);
        float o[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) o[k] = __uint_as_float(u[k]);
        if (any_bad && !no_row)
#pragma unroll 1
          for (int t = p.reverse ? i : 0; t < (p.reverse ? kC : i + 1); ++t) {
            if (!(a.bad[now][t >> 5] >> (t & 31) & 1) || a.trace[t] != trace_i) continue;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              if (c0 + c + k >= p.dz) continue;
              const float g = to_f32(z[(lo + t) * p.z.st + c0 + c + k]);
              if (!(fabsf(g) <= 3.4028235e38f)) o[k] = __int_as_float(0x7FC00000);
            }
          }
        if (TMA || ov == 1) {
#pragma unroll
          for (int k = 0; k < 16; k += 8) {
            const int piece = (c0 + c + k) / 8;
            put_shared(base + L::w + (piece >> 3) * kPanel + i * 128 + (((piece & 7) ^ (i & 7)) << 4),
                       make_uint4(B::pack(o[k], o[k + 1]), B::pack(o[k + 2], o[k + 3]), B::pack(o[k + 4], o[k + 5]), B::pack(o[k + 6], o[k + 7])));
          }
        } else if (lo + i < p.time) {
#pragma unroll
          for (int k = 0; k < 16; k += 8) {
            const uint4 v = make_uint4(B::pack(o[k], o[k + 1]), B::pack(o[k + 2], o[k + 3]), B::pack(o[k + 4], o[k + 5]), B::pack(o[k + 6], o[k + 7]));
            store8(to, c0 + c + k, p.dz, ov, v);
          }
        }
      }
      if (!kBf && more) put_state();  // (z's second part has been read)
      if constexpr (TMA) fence_shared();
      fence_before();
    }
    put_marks(now ^ 1);
    over = __syncthreads_or(gave_up);
    if (!STATES && !TMA && ov == 1) {  // (a warp stores eight steps' rows; w's place is written again behind the next barrier)
      const int64_t t0 = lo + warp * 8;
      const int steps = (int)max((int64_t)0, min(p.time - t0, (int64_t)8));
      store_narrow<DZ>((uint16_t*)out + t0 * p.out.st, p.out.st, base + L::w + warp * 8 * 128, p.dz, steps);
    }
    if (!STATES && TMA && issuer && !over) {
#pragma unroll
      for (int k = 0; k < DZ / 64; ++k) tma_store_4d(&maps.out, 64 * k, (int32_t)lo, h, (int32_t)b, base + L::w + k * kPanel);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
  if (!over) {
    float* to = nullptr;
    if (STATES) to = p.local + (row * p.segs + seg) * p.dx * p.dz;
    else if (p.final_state && seg == (p.reverse ? 0 : p.segs - 1)) to = p.final_state + row * p.dx * p.dz;
    if (to && srow < p.dx) store_row<kCols>(s, to + srow * p.dz, c0, p.dz);
    if (STATES && tid == 0) p.seen[row * p.segs + seg] = samples;
  }
  if (TMA && issuer) {
    if (over && xy_coming) barrier_wait(&a.bar[4], n & 1, kWaitTries);  // (chunk n's, which nobody waits for)
    if (over && z_coming) barrier_wait(&a.bar[6], n & 1, kWaitTries);
    if (!STATES) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  if (over) {
    if (tid == 0 && p.status) atomicOr(p.status, kStatusTimeout);
    // products that may be in flight (all of them are in the phases of their barriers; bounded)
    if (n && warp == 0) {
      barrier_wait(&a.bar[1], phase ^ 1, kWaitTries);
      if (!STATES) {
        barrier_wait(&a.bar[0], phase ^ 1, kWaitTries);
        barrier_wait(&a.bar[2], phase ^ 1, kWaitTries);
        barrier_wait(&a.bar[5], phase ^ 1, kWaitTries);
      }
    }
  }
  fence_before();
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

template <typename T, int DX, int DZ, bool STATES, bool TMA>
mf_status run(const AttendPass& p, const Maps& maps, int64_t blocks, cudaStream_t s) {
  auto kernel = k_attend_tc<T, DX, DZ, STATES, TMA>;
  constexpr size_t smem = smem_bytes<T, DX, DZ, STATES>();
  MF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  kernel<<<(unsigned)blocks, kThreads, smem, s>>>(p, maps);
  MF_CUDA(cudaGetLastError());
  return MF_OK;
}

// A tensor's map, 64 columns of 128 steps of a head at a time; false if its address or strides do not allow one (a
// broadcast axis has none either).
template <typename T>
bool map_of(CUtensorMap* map, const AttendSeq& q, const AttendPass& p, int64_t rows, int dim) {
  const int64_t size[3] = {p.time, p.heads, rows / p.heads}, stride[3] = {q.st, q.sh, q.sb};
  cuuint64_t dims[4] = {(cuuint64_t)dim}, bytes[3];
  if ((uintptr_t)q.p & 15) return false;
  for (int k = 0; k < 3; ++k) {
    dims[k + 1] = (cuuint64_t)size[k];
    const int64_t b = size[k] > 1 ? stride[k] * 2 : (dim * 2 + 15) / 16 * 16;
    if (b <= 0 || b % 16 || b >= (int64_t(1) << 40)) return false;
    bytes[k] = (cuuint64_t)b;
  }
  const cuuint32_t box[4] = {64, kC, 1, 1};
  return tensor_map(map, Bits<T>::bf ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, q.p, dims, bytes, box,
                    CU_TENSOR_MAP_SWIZZLE_128B);
}

template <typename T, int DX, int DZ>
mf_status run(const AttendPass& p, int64_t rows, cudaStream_t s) {
  Maps maps{};
  const bool tma = map_of<T>(&maps.y, p.y, p, rows, p.dx) && map_of<T>(&maps.z, p.z, p, rows, p.dz) &&
                   (p.local || (map_of<T>(&maps.x, p.x, p, rows, p.dx) && map_of<T>(&maps.out, p.out, p, rows, p.dz)));
  if (p.local) return tma ? run<T, DX, DZ, true, true>(p, maps, rows * (p.segs - 1), s) : run<T, DX, DZ, true, false>(p, maps, rows * (p.segs - 1), s);
  return tma ? run<T, DX, DZ, false, true>(p, maps, rows * p.segs, s) : run<T, DX, DZ, false, false>(p, maps, rows * p.segs, s);
}

template <typename T>
mf_status run(const AttendPass& p, int64_t rows, cudaStream_t s) {
  if (p.dx <= 64) return p.dz <= 64 ? run<T, 64, 64>(p, rows, s) : run<T, 64, 128>(p, rows, s);
  return p.dz <= 64 ? run<T, 128, 64>(p, rows, s) : run<T, 128, 128>(p, rows, s);
}

}  // namespace

mf_status attend_tc(int type, const AttendPass& p, int64_t rows, cudaStream_t s) {
  return type == MF_TYPE_BF16 ? run<__nv_bfloat16>(p, rows, s) : run<__half>(p, rows, s);
}

}  // namespace mf
