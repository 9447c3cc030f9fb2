// The passes of linear attention on the tensor cores, for bf16 and fp16 (attend.cuh has the formulas).
//
// A block takes a segment of a head, 128 steps at a time, and holds the state in registers: fp32, a row of x a lane.
// A chunk is four products with fp32 accumulators in tensor memory (tcgen05, 128 rows each):
//   P = x y^T          [steps][steps]   operands as they are
//   inter = x S        [steps][dz]      S as two parts of x's type, written to shared memory behind the chunk before
//   own = w^T z        [dx][dz]         w = y times what is left of each step at the chunk's end, as two fp16 parts
//   intra = P' z       [steps][dz]      P' = P times what is left between the steps; fp16: one part for bf16 results, whose
//                                       own rounding is 8 times coarser, two for fp16 ones; from tensor memory
// Values that pass as fp16 are scaled by powers of two so that none leaves its range: z by each step's largest (bf16; fp16
// is as it is), P' by each row's largest, w by the chunk's largest, the state of fp16 calls by its largest.  What is lost
// lies 2^-39 or more below that.
// An infinity or a NaN in z is taken out (times a zero weight it would reach steps that do not see it) and added to the
// results that do see it, by reading z again; the rest of what is not finite takes the way of the products.
//
// The floor is memory (x, y and z read once, and y and z once more where a head is split into segments; results written
// once).  What bounds the kernel is a chunk's chain of steps, one block an SM: operands laid out and scaled, w, P, P', state,
// results, each a third issue and two thirds latency.  Measured, bf16, dx = dz = 128: about 13,000 clocks a chunk, where
// memory takes 5600 and the products 3100; 7000 a chunk for states alone.  65536 x 16 heads forward 593 us (floor 158); 8 x
// 4096 x 16 heads with gradients 877 (222): 216 a pass.  On the way (the latter): loads and stores by registers 1546,
// tensor copies 989, the next x and y as soon as they are read 953, no factor in two parts where one will do 877.  A
// seventeenth warp for products and copies left 120 registers a thread (spills: 1227 instead of 1039); two issuing
// threads changed nothing.  One block takes all of an SM's shared memory for 128 x 128; 64 x 64 would let two in.
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
  static __device__ __forceinline__ int exponent(uint32_t magnitude) { return (int)(magnitude >> 7) - 127; }
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
  static __device__ __forceinline__ int exponent(uint32_t magnitude) { return (int)(magnitude >> 10) - 15; }
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
using Half = Bits<__half>;

// 2^e; 0 and infinity outside the normal range.
__device__ __forceinline__ float pow2(int e) { return __int_as_float(e < -126 ? 0 : e > 127 ? 0x7F800000 : (e + 127) << 23); }
__device__ __forceinline__ int exponent_of(float v) { return (int)(__float_as_uint(v) >> 23 & 255) - 127; }
// 2^e of a product's sum, in one factor where that is a normal number (nearly always), else f and `more` first.
struct Power {
  float f, more;
  bool plain;
  __device__ __forceinline__ explicit Power(int e) {
    plain = e >= -120 && e <= 120;
    const int first = plain ? 0 : min(max(e, -252), 250) >> 1;
    more = pow2(first);
    f = pow2(plain ? e : min(max(e, -252), 250) - first);
  }
};
constexpr int kLeast = -125;  // exponents below count as this

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
__host__ __device__ __forceinline__ int vec_of(const AttendSeq& q, int dim) {
  const uintptr_t a = (uintptr_t)q.p;
  const int64_t s = (int64_t)dim | q.sb | q.st | q.sh;
  return !(a & 15) && !(s & 7) ? 8 : !(a & 7) && !(s & 3) ? 4 : 1;
}
template <int DX, int DZ>
struct Layout {
  static constexpr int x = 0, y = x + DX / 64 * kPanel, z = y + DX / 64 * kPanel, w = z + DZ / 64 * kPanel;
  static constexpr int w_part = DX / 64 * kPanel, s = w + 2 * w_part;
  static constexpr int s_panel = DX * 128, s_part = DZ / 64 * s_panel, small = s + 2 * s_part;
};
// What steps' values need beside them.
struct Small {
  uint64_t bar[6];               // P; own; intra; one that nothing completes; copies; inter
  uint32_t missing[2][4], begins[2][4], bad[2][4];  // bits of a chunk's steps; bad: a z that is not finite
  int most[2][3];                // largest exponents of a chunk: of w z, y z, z
  int largest[2];                // bits of the state's largest magnitude (fp16)
  uint32_t tmem;
  alignas(16) float column[kC];  // P' off the diagonal blocks: a column's factor
  alignas(16) float diagonal[kC];  // and on them, where the decay allows it
  float row[kC];                 // what is left at each step of the state before the chunk (-1: nothing)
  uint8_t seen[kC], trace[kC];   // samples, and traces begun, up to and with each step
  int8_t ze[kC];                 // z is what is in shared memory times 2^ze
  int8_t top[4][kC];             // exponents of the largest values of P' rows, of each block of 32 columns
};
static_assert(offsetof(Small, column) % 16 == 0 && offsetof(Small, diagonal) % 16 == 0, "read by vectors");
template <int DX, int DZ>
constexpr size_t smem_bytes() { return Layout<DX, DZ>::small + sizeof(Small); }
static_assert(smem_bytes<128, 128>() <= 232448, "shared memory of a block");

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

struct Maps {
  CUtensorMap x, y, z, out;
};

// STATES: a pass for the segments' own states.  TMA: x, y and z come, and results leave, by tensor copies; else by loads and
// stores of the widths that their alignment allows.
template <typename T, int DX, int DZ, bool STATES, bool TMA>
__global__ void __launch_bounds__(kThreads, 1) k_attend_tc(const __grid_constant__ AttendPass p, const __grid_constant__ Maps maps) {
  using B = Bits<T>;
  using L = Layout<DX, DZ>;
  constexpr int kXLoads = DX / 32, kZLoads = DZ / 32;  // 16-byte pieces of a thread
  constexpr int kCols = DZ / 4;                        // a thread's columns of results and state
  // z's copies go to where the lower part of w was, if that is as large (results leave from the upper part's place); of
  // states to where the state would be
  constexpr bool kZCopy = TMA && (STATES || DX >= DZ);
  constexpr int kZRaw = STATES ? L::s : L::w + L::w_part;
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
  // products of a decay above 1 grow by up to 2^(l2 kC)
  const int growth = l2 > 0.f ? (int)fminf(l2 * kC + 1.f, 200.f) : 0;

  // the products of a block with itself: what is left between two steps as a quotient, unless the decay is too fast
  const bool inverse = fabsf(l2) <= 1.f;

  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_u32(&a.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 0) {
    for (int k = 0; k < 6; ++k) barrier_init(&a.bar[k], k == 4 && !STATES && kZCopy ? 2 : 1);
    barrier_init_fence();
    a.most[0][0] = a.most[0][1] = a.most[0][2] = -1000;
    a.largest[0] = a.largest[1] = 0;
  }
  if (tid < 4) a.bad[0][tid] = 0;
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = a.tmem;
  constexpr uint32_t kP = 0, kIntra = 128, kInter = 256, kOwn = 384;  // columns
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
  uint4 xr[STATES || TMA ? 1 : kXLoads], yr[kXLoads], zr[kZLoads];
  int mark = MF_MARK_SAMPLE;
  auto chunk_at = [&](int n) { return (int64_t)(p.reverse ? end - 1 - n : first + n) * kC; };
  auto load = [&](int64_t lo) {
    const int64_t t = lo + step;
    const bool in = t < p.time && !narrow;
    const T* const zp = z + t * p.z.st;
    if constexpr (!TMA) {
      const T* const xp = x + t * p.x.st;
      const T* const yp = y + t * p.y.st;
#pragma unroll
      for (int k = 0; k < kXLoads; ++k) {
        if constexpr (!STATES) xr[k] = in ? load8(xp, col + 32 * k, p.dx, xv) : make_uint4(0u, 0u, 0u, 0u);
        yr[k] = in ? load8(yp, col + 32 * k, p.dx, yv) : make_uint4(0u, 0u, 0u, 0u);
      }
    }
    if constexpr (!kZCopy) {
#pragma unroll
      for (int k = 0; k < kZLoads; ++k) zr[k] = in ? load8(zp, col + 32 * k, p.dz, zv) : make_uint4(0u, 0u, 0u, 0u);
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

  // Copies of a chunk's x and y (for states of y, into the two operands' places in turn), and of its z.
  auto copy_xy = [&](int n) {
    const int32_t lo = (int32_t)chunk_at(n);
    barrier_expect(&a.bar[4], ((STATES ? 1 : 2) * (DX / 64) + (STATES ? DZ / 64 : 0)) * kPanel);
#pragma unroll
    for (int k = 0; k < DX / 64; ++k) {
      if constexpr (!STATES) tma_load_4d(base + L::x + k * kPanel, &maps.x, 64 * k, lo, h, (int32_t)b, &a.bar[4]);
      tma_load_4d(base + (STATES && (n & 1) ? L::x : L::y) + k * kPanel, &maps.y, 64 * k, lo, h, (int32_t)b, &a.bar[4]);
    }
  };
  auto copy_z = [&](int n) {
    if constexpr (kZCopy) {
      if constexpr (!STATES) barrier_expect(&a.bar[4], DZ / 64 * kPanel);  // (of states: copy_xy's)
#pragma unroll
      for (int k = 0; k < DZ / 64; ++k)
        tma_load_4d(base + kZRaw + k * kPanel, &maps.z, 64 * k, (int32_t)chunk_at(n), h, (int32_t)b, &a.bar[4]);
    }
  };

  bool gave_up = false;
  auto wait = [&](int k, uint32_t parity) { gave_up = gave_up || !(barrier_polls(&a.bar[k], parity) || barrier_wait(&a.bar[k], parity, kWaitTries)); };
  if (p.tries) gave_up = !barrier_wait(&a.bar[3], 0, p.tries);  // (a test of the way out: nothing completes it)

  // The state as the operand of the next chunk: two parts of T, fp16 ones scaled by 2^-se.
  int se = 0;
  auto put_state = [&](int which) {
    if constexpr (!B::bf) {
      float m = 0.f;
#pragma unroll
      for (int c = 0; c < kCols; ++c) m = fmaxf(m, fabsf(s[c]) <= 3.4028235e38f ? fabsf(s[c]) : 0.f);
      const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
      if (lane == 0) atomicMax(&a.largest[which], (int)top);
      __syncthreads();
      se = exponent_of(__int_as_float(a.largest[which])) - 14;
      if (tid == 0) a.largest[which ^ 1] = 0;
      se = max(se, -120);
    }
    const float scale = B::bf ? 1.f : pow2(-se);
    if (DX == 128 || quarter < 2) {
#pragma unroll
      for (int c = 0; c < kCols; c += 8) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float u = s[c + 2 * k] * scale, v = s[c + 2 * k + 1] * scale;
          hi[k] = B::pack(u, v);
          const float2 f = B::floats(hi[k]);
          lo[k] = B::pack(u - f.x, v - f.y);
        }
        const int piece = (c0 + c) / 8;
        const uint32_t to = base + L::s + (piece >> 3) * L::s_panel + srow * 128 + (((piece & 7) ^ (srow & 7)) << 4);
        put_shared(to, make_uint4(hi[0], hi[1], hi[2], hi[3]));
        put_shared(to + L::s_part, make_uint4(lo[0], lo[1], lo[2], lo[3]));
      }
    }
    fence_shared();
  };
  // Products and copies are issued by one thread, of a warp whose block of P' no step sees (so the others seldom wait for it).
  const bool issuer = tid == (p.reverse ? 3 : 12) * 32;
  auto first_products = [&]() {
    fence_after();
    if constexpr (!STATES) {
      constexpr uint32_t id_p = idesc(kC, B::bf, false, false), id_s = idesc(DZ, B::bf, false, true);
#pragma unroll
      for (int k = 0; k < DX / 16; ++k) {
        const uint32_t at = (k >> 2) * kPanel + (k & 3) * 32;
        mma_ss(tmem + kP, desc_k(base + L::x + at), desc_k(base + L::y + at), id_p, k > 0);
      }
      commit(&a.bar[0]);
#pragma unroll
      for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int k = 0; k < DX / 16; ++k)
          mma_ss(tmem + kInter, desc_k(base + L::x + (k >> 2) * kPanel + (k & 3) * 32),
                 desc_mn(base + L::s + part * L::s_part + k * 2048, L::s_panel), id_s, part + k > 0);
      commit(&a.bar[5]);
    }
    constexpr uint32_t id_w = idesc(DZ, false, true, true);
    // (dx of 64: the upper 64 rows of the product come from what lies behind, and nothing reads them)
#pragma unroll
    for (int part = 0; part < 2; ++part)
#pragma unroll
      for (int k = 0; k < kC / 16; ++k)
        mma_ss(tmem + kOwn, desc_mn(base + L::w + part * L::w_part + k * 2048, kPanel), desc_mn(base + L::z + k * 2048, kPanel), id_w,
               part + k > 0);
    commit(&a.bar[1]);
  };
  auto second_products = [&]() {
    fence_after();
    constexpr uint32_t id_z = idesc(DZ, false, false, true);
#pragma unroll
    for (int part = 0; part < (B::bf ? 1 : 2); ++part)
#pragma unroll
      for (int k = 0; k < kC / 16; ++k)
        mma_ts(tmem + kIntra, tmem + kP + part * 64 + k * 8, desc_mn(base + L::z + k * 2048, kPanel), id_z, part + k > 0);
    commit(&a.bar[2]);
  };

  uint32_t phase = 0;
  int n = 0;
  bool copying = false;  // (of the issuer: copies of the next chunk are on their way)
  if (TMA && issuer && count > 0 && !gave_up) {
    copy_xy(0);
    copy_z(0);
    copying = true;
  }
  if (count > 0 && !gave_up) load(chunk_at(0));
  put_marks(0);
  if (!STATES && count > 0) put_state(1);

  float samples = 0.f;
  bool over = __syncthreads_or(gave_up);
  for (; n < count && !over; ++n, phase ^= 1) {
    const int64_t lo = chunk_at(n);
    const int now = n & 1;
    if (tid == 0) a.most[now ^ 1][0] = a.most[now ^ 1][1] = a.most[now ^ 1][2] = -1000;
    if (tid < 4) a.bad[now ^ 1][tid] = 0;
    uint32_t missing[4], begins[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      missing[k] = a.missing[now][k];
      begins[k] = a.begins[now][k];
    }
    const int all = kC - (__popc(missing[0]) + __popc(missing[1]) + __popc(missing[2]) + __popc(missing[3]));
    const int traces = __popc(begins[0]) + __popc(begins[1]) + __popc(begins[2]) + __popc(begins[3]);

    // -- operands into shared memory
    const bool gone = missing[step >> 5] >> (step & 31) & 1;
    float weight;  // of the step's y z in the state
    int ze = 0;
    uint32_t ytop;
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
      if constexpr (TMA) {
        wait(4, phase);
#pragma unroll
        for (int k = 0; k < kXLoads; ++k) yr[k] = get(STATES && now ? L::x : L::y, k);
        if constexpr (kZCopy) {
#pragma unroll
          for (int k = 0; k < kZLoads; ++k) zr[k] = get(kZRaw, k);
        }
      }
      if constexpr (!TMA) {
        if (narrow) {
          const int64_t t0 = lo + warp * 8;
          const int steps = (int)max((int64_t)0, min(p.time - t0, (int64_t)8));
          const uint32_t to = base + warp * 8 * 128;
          if constexpr (!STATES) copy_narrow<DX>(to + L::x, (const uint16_t*)x + t0 * p.x.st, p.x.st, p.dx, steps);
          copy_narrow<DX>(to + L::y, (const uint16_t*)y + t0 * p.y.st, p.y.st, p.dx, steps);
          copy_narrow<DZ>(to + L::z, (const uint16_t*)z + t0 * p.z.st, p.z.st, p.dz, steps);
          __syncwarp();  // (a warp copies its own steps' rows)
#pragma unroll
          for (int k = 0; k < kXLoads; ++k) {
            if constexpr (!STATES) xr[k] = get(L::x, k);
            yr[k] = get(L::y, k);
          }
#pragma unroll
          for (int k = 0; k < kZLoads; ++k) zr[k] = get(L::z, k);
          __syncwarp();
        }
      }
      if (!p.reverse && gone) {
#pragma unroll
        for (int k = 0; k < kXLoads; ++k) yr[k] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int k = 0; k < kZLoads; ++k) zr[k] = make_uint4(0u, 0u, 0u, 0u);
      }
      if constexpr (!STATES) {
#pragma unroll
        for (int k = 0; k < kXLoads; ++k) {
          if constexpr (!TMA) {
            place(L::x, k, p.reverse && gone ? make_uint4(0u, 0u, 0u, 0u) : xr[k]);
            place(L::y, k, yr[k]);
          } else if (gone) {
            place(p.reverse ? L::x : L::y, k, make_uint4(0u, 0u, 0u, 0u));
          }
        }
      }
      uint32_t top = row_max<T>(zr);
      if (__any_sync(0xffffffffu, top >= B::inf)) {
        if (top >= B::inf && (lane & 3) == 0) atomicOr(&a.bad[now][step >> 5], 1u << (step & 31));
#pragma unroll
        for (int k = 0; k < kZLoads; ++k) zr[k] = finite_part<T>(zr[k]);
        top = row_max<T>(zr);
      }
      if constexpr (B::bf) {
        ze = max(B::exponent(top), -110) - 14;  // (below 2^15: fp16 holds 2^-39 of that)
        const float f = pow2(-ze);
#pragma unroll
        for (int k = 0; k < kZLoads; ++k) {
          uint32_t* const q = (uint32_t*)&zr[k];
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float2 u = B::floats(q[w]);
            q[w] = Half::pack(u.x * f, u.y * f);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kZLoads; ++k) place(L::z, k, zr[k]);
      if ((lane & 3) == 0) a.ze[step] = (int8_t)ze;
      // (nothing of a step whose weight is negative reaches the end, whatever it is)
      if (weight < 0.f) {
#pragma unroll
        for (int k = 0; k < kXLoads; ++k) yr[k] = make_uint4(0u, 0u, 0u, 0u);
      }
      ytop = row_max<T>(yr);
      if (__any_sync(0xffffffffu, ytop >= B::inf)) {
        uint4 finite[kXLoads];
#pragma unroll
        for (int k = 0; k < kXLoads; ++k) finite[k] = finite_part<T>(yr[k]);
        ytop = row_max<T>(finite);
      }
      weight = weight < 0.f || !ytop ? 0.f : weight * p.alpha_src;
    }
    {
      const int both = max(B::exponent(ytop), kLeast) + ze;
      const int w = __reduce_max_sync(0xffffffffu, ytop && weight != 0.f ? both + exponent_of(weight) : -1000);
      const int yz = __reduce_max_sync(0xffffffffu, ytop ? both : -1000), zz = __reduce_max_sync(0xffffffffu, ze);
      if (lane == 0) {
        atomicMax(&a.most[now][0], w);
        atomicMax(&a.most[now][1], yz);
        atomicMax(&a.most[now][2], zz);
      }
    }
    // (the results before have left shared memory, where w goes)
    if (!STATES && TMA && issuer) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncthreads();
    copying = false;
    if (STATES && TMA && issuer && n + 1 < count) {  // (the chunk's own copies have ended, and the place is that of the chunk before)
      copy_xy(n + 1);
      copy_z(n + 1);
      copying = true;
    }
    // (the second terms keep every factor in range)
    const int we = max(a.most[now][0], a.most[now][2] - 107), pe = max(a.most[now][1], a.most[now][2] - 80) + growth;
    {
      const float f = weight * pow2(ze - we + 13);  // y f: below 2^15
#pragma unroll
      for (int k = 0; k < kXLoads; ++k) {
        const uint32_t* const q = (const uint32_t*)&yr[k];
        uint32_t hi[4], lo4[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float2 u = B::floats(q[w]);
          const float v0 = u.x * f, v1 = u.y * f;
          hi[w] = Half::pack(v0, v1);
          const float2 g = Half::floats(hi[w]);
          lo4[w] = Half::pack(v0 - g.x, v1 - g.y);
        }
        place(L::w, k, make_uint4(hi[0], hi[1], hi[2], hi[3]));
        place(L::w + L::w_part, k, make_uint4(lo4[0], lo4[1], lo4[2], lo4[3]));
      }
    }
    if constexpr (!STATES) {
      if (tid < kC) {
        // what is left of step j at its block's border on the side of the steps that see it, and the inverse from the
        // border on the other side
        const int near = p.reverse ? (tid & ~31) - 1 : tid | 31, far = p.reverse ? tid | 31 : (tid & ~31) - 1;
        const int seen = a.seen[tid], at = near < 0 ? 0 : a.seen[near], from = far < 0 ? 0 : a.seen[far];
        const float f = pow2(a.ze[tid] - pe);
        a.column[tid] = exp2f(l2 * (float)abs(seen - at)) * f;
        a.diagonal[tid] = inverse ? exp2f(-l2 * (float)abs(seen - from)) * f : f;
      }
    }
    fence_shared();
    fence_before();
    __syncthreads();
    const bool more = n + 1 < count;
    if (issuer) {
      first_products();
      if (!STATES && TMA && more) {  // (P and inter have read x and y; the products' issue took as long)
        wait(5, phase);
        if (!gave_up) copy_xy(n + 1);
        copying = !gave_up;
      }
    }
    __syncwarp();
    int re = 0;  // P' is what is in tensor memory times 2^(re + pe)
    if constexpr (!STATES) {
      // -- P' = P times what is left between its steps: a thread has step i, 32 columns
      const int i = quarter * 32 + lane, j0 = group * 32;
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
      // scaled so that the row's largest lies below 2^15
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < 32; ++k) top = fmaxf(top, fabsf(v[k]));
      a.top[group][i] = (int8_t)min(max(exponent_of(top), -110), 126);
      // (the parts take the place of P, when all four warps of these lanes have read theirs)
      fence_before();
      asm volatile("bar.sync %0, %1;" ::"r"(1 + quarter), "r"(128) : "memory");
      fence_after();
      re = max(max(a.top[0][i], a.top[1][i]), max(a.top[2][i], a.top[3][i])) - 14;
      const float f = pow2(-re);
      uint32_t hi[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        v[2 * k] *= f;
        v[2 * k + 1] *= f;
        hi[k] = Half::pack(v[2 * k], v[2 * k + 1]);
      }
      tmem_put(lanes + kP + group * 16, hi);
      if constexpr (!B::bf) {
        uint32_t lo16[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float2 u = Half::floats(hi[k]);
          lo16[k] = Half::pack(v[2 * k] - u.x, v[2 * k + 1] - u.y);
        }
        tmem_put(lanes + kP + 64 + group * 16, lo16);
      }
      tmem_put_wait();
      fence_before();
      __syncthreads();
      if (issuer) second_products();
      __syncwarp();
    }
    if (more) load(chunk_at(n + 1));

    // -- the state: what is left of it, and the chunk's own
    const bool any_bad = a.bad[now][0] | a.bad[now][1] | a.bad[now][2] | a.bad[now][3];
    const float chunk_samples = traces ? -1.f : (float)all;
    samples = samples < 0.f || traces ? -1.f : samples + (float)all;
    wait(1, phase);
    fence_after();
    if (!STATES && TMA && issuer && copying) copy_z(n + 1);  // (w is read)
    const int used = se;              // (the scale of the operand that inter has)
    if (DX == 128 || quarter < 2) {  // (rows of the state)
      // s' = left s + own as (keep + lost) s + own: one rounding of what is nearly s
      const Remains left(log_decay, chunk_samples);
      const float keep = left.factor >= 0.5f ? 1.f : 0.f, lost = left.factor >= 0.5f ? left.lost : left.factor;
      const Power own_scale(we - 13);
      if (left.factor < 0.f) {
#pragma unroll
        for (int c = 0; c < kCols; ++c) s[c] = 0.f;
      }
#pragma unroll
      for (int c = 0; c < kCols; c += 16) {
        uint32_t r[16];
        tmem_ask(lanes + kOwn + c0 + c, r);
        tmem_wait(r);
        if (!own_scale.plain)
#pragma unroll
          for (int k = 0; k < 16; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * own_scale.more);
#pragma unroll
        for (int k = 0; k < 16; ++k) s[c + k] = fmaf(keep, s[c + k], fmaf(lost, s[c + k], __uint_as_float(r[k]) * own_scale.f));
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
      if (more) put_state(now);
      // -- results
      const int i = srow;
      const float w = a.row[i];
      const float fi = (B::bf ? 1.f : pow2(used)) * (w * p.alpha_row);
      const Power intra_scale(re + pe);
      const float fp = intra_scale.f * p.alpha;
      const bool all_plain = __all_sync(0xffffffffu, intra_scale.plain), state_seen = __all_sync(0xffffffffu, !(w < 0.f));
      const int trace_i = a.trace[i];
      // (a missing sample's row of x, k or v, has no gradient: not NaN either where the state or y is not finite)
      const bool no_row = p.reverse && (a.missing[now][quarter] >> lane & 1);
      wait(2, phase);
      fence_after();
      T* const to = out + (lo + i) * p.out.st;
#pragma unroll
      for (int c = 0; c < kCols; c += 16) {
        uint32_t u[16], v[16];
        tmem_ask(lanes + kIntra + c0 + c, u);
        tmem_ask(lanes + kInter + c0 + c, v);
        tmem_wait(u);
        tmem_wait(v);
        float o[16];
        if (!all_plain)
#pragma unroll
          for (int k = 0; k < 16; ++k) u[k] = __float_as_uint(__uint_as_float(u[k]) * intra_scale.more);
        if (!state_seen)  // (of a trace that has ended nothing comes, whatever it was)
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = w < 0.f ? 0u : v[k];
#pragma unroll
        for (int k = 0; k < 16; ++k) o[k] = fmaf(__uint_as_float(u[k]), fp, __uint_as_float(v[k]) * fi);
        if (any_bad)
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
        if (p.reverse)
#pragma unroll
          for (int k = 0; k < 16; ++k) o[k] = no_row ? 0.f : o[k];
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
    if (over && copying) barrier_wait(&a.bar[4], n & 1, kWaitTries);  // (chunk n's, which nobody waits for)
    if (!STATES) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  if (over) {
    if (tid == 0 && p.status) atomicOr(p.status, kStatusTimeout);
    // products that may be in flight (all of them are in the phases of their barriers; bounded)
    if (n && warp == 0)
      for (int k = STATES ? 1 : 0; k < (STATES ? 2 : 3); ++k) barrier_wait(&a.bar[k], phase ^ 1, kWaitTries);
  }
  fence_before();
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

template <typename T, int DX, int DZ, bool STATES, bool TMA>
mf_status run(const AttendPass& p, const Maps& maps, int64_t blocks, cudaStream_t s) {
  auto kernel = k_attend_tc<T, DX, DZ, STATES, TMA>;
  constexpr size_t smem = smem_bytes<DX, DZ>();
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
  // (where z comes by loads beside the others' copies, its rows have to allow loads of four values)
  const bool z_fits = !p.local && DX < DZ ? vec_of<T>(p.z, p.dz) > 1 : map_of<T>(&maps.z, p.z, p, rows, p.dz);
  const bool tma = z_fits && map_of<T>(&maps.y, p.y, p, rows, p.dx) &&
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
